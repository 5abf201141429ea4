// Pages of a cache: forking with copy of part pages, growing, trimming, compacting.
#include "../../include/arith_sampling.h"
#include "as_bounds.cuh"
#include "as_host.h"

namespace asx {

ASX_BOUNDS_READER(bounds_pages)

constexpr int PG_NT = 128;              // table kernels: one CTA per lane
constexpr int PL_NT = 1024;             // the planning CTA
constexpr int CP_NT = 256;              // page copies
constexpr int CP_CHUNK = CP_NT * 16 * 4;    // bytes a CTA copies at a time

// Scratch, in ints.
struct PageWork {
    int *child, *first, *eff;           // [lanes_in]: children of a lane, the first of them, its length (0 if unusable)
    int *off;                           // [lanes_out]: pages wanted by the lanes before this one
    int *free_page;                     // [n_pages]: free pages, lowest first
    int *src, *dst;                     // [n_pages]: pages to copy
    int *moves;                         // [1]: how many
};
static size_t work_ints(int lanes_in, int lanes_out, int n_pages) {
    return 64 + 3 * (size_t)lanes_in + (size_t)lanes_out + 3 * (size_t)n_pages;
}
static PageWork carve(void* p, int lanes_in, int lanes_out, int n_pages) {
    PageWork w;
    int* q = static_cast<int*>(p);
    w.moves = q; q += 64;
    w.child = q; q += lanes_in;
    w.first = q; q += lanes_in;
    w.eff = q; q += lanes_in;
    w.off = q; q += lanes_out;
    w.free_page = q; q += n_pages;
    w.src = q; q += n_pages;
    w.dst = q;
    return w;
}

struct ForkArgs {
    const int *parent, *table, *len, *ref;
    int *table_out, *len_out, *ref_out, *lane_status;
    int lanes_in, lanes_out, max_pages, page_size, n_pages;
};

__device__ __forceinline__ int pages_of(int len, int page_size) { return (len + page_size - 1) / page_size; }

// CTA j: how many lanes continue lane j and which is the first; whether its row is usable; its
// share of the copy of the reference counts.
__global__ void __launch_bounds__(PG_NT) fork_count_kernel(const ForkArgs a, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x;
    if (a.ref_out != a.ref)
        for (int i = blockIdx.x * PG_NT + tid; i < a.n_pages; i += gridDim.x * PG_NT) a.ref_out[i] = a.ref[i];
    __shared__ int n_child, first;
    for (int j = blockIdx.x; j < a.lanes_in; j += gridDim.x) {
        if (tid == 0) { n_child = 0; first = a.lanes_out; }
        __syncthreads();
        int n = 0, f = a.lanes_out;
        for (int i = tid; i < a.lanes_out; i += PG_NT)
            if (a.parent[i] == j) { ++n; f = min(f, i); }
        if (n) { atomicAdd(&n_child, n); atomicMin(&first, f); }
        const int len = a.len[j];
        bool bad = len < 0 || len > (long long)a.max_pages * a.page_size;
        if (!bad)
            for (int m = tid; m < pages_of(len, a.page_size); m += PG_NT) {
                const int g = a.table[(size_t)j * a.max_pages + m];
                bad |= g < 0 || g >= a.n_pages;
            }
        bad = __syncthreads_or(bad);
        if (tid == 0) { w.child[j] = n_child; w.first[j] = first; w.eff[j] = bad ? -1 : len; }
        __syncthreads();
    }
}

// CTA j: the change of the reference counts of lane j's pages, and row j of the new table.
__global__ void __launch_bounds__(PG_NT) fork_table_kernel(const ForkArgs a, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x;
    const int n = max(a.lanes_in, a.lanes_out);
    for (int j = blockIdx.x; j < n; j += gridDim.x) {
        if (j < a.lanes_in) {
            const int len = w.eff[j], c = w.child[j];
            const int* row = a.table + (size_t)j * a.max_pages;
            if (len > 0 && c != 1)
                for (int m = tid; m < pages_of(len, a.page_size); m += PG_NT) {
                    // a part page stays with one child, if there is any
                    const int change = (m + 1) * (long long)a.page_size > len ? min(c, 1) - 1 : c - 1;
                    if (change) atomicAdd(&a.ref_out[ASX_AT(row[ASX_AT(m, a.max_pages, 201)], a.n_pages, 202)], change);
                }
        }
        if (j < a.lanes_out) {
            const int p = a.parent[j];
            const int len = p >= 0 && p < a.lanes_in ? w.eff[p] : 0;
            const int full = len > 0 ? len / a.page_size : 0;
            const bool keeps = len > 0 && w.first[p] == j;
            const int held = keeps ? pages_of(len, a.page_size) : full;
            for (int m = tid; m < a.max_pages; m += PG_NT)
                a.table_out[(size_t)j * a.max_pages + m] = m < held ? a.table[(size_t)p * a.max_pages + m] : -1;
        }
    }
}

// Inclusive prefix sum over the planning CTA's threads, in thread order; total: the whole sum.
__device__ __forceinline__ int block_scan(int v, int* warp_sum, int& total) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                    // the last call's readers of warp_sum are done
    if (lane == 31) warp_sum[wid] = v;
    __syncthreads();
    int s = warp_sum[lane];             // 32 warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += u;
    }
    total = __shfl_sync(0xFFFFFFFFu, s, 31);
    const int before = __shfl_sync(0xFFFFFFFFu, s, wid > 0 ? wid - 1 : 0);
    return v + (wid > 0 ? before : 0);
}

// The first `want` pages i in [lo, hi) with (ref[i] > 0) == used, in order, into list; returns how many there are
// (at most want).  list has room for n_pages.
__device__ int collect(const int* ref, int lo, int hi, bool used, int want, int* list, int n_pages, int* warp_sum) {
    constexpr int PER = 16;
    int got = 0;
    for (int base = lo; base < hi && got < want; base += PL_NT * PER) {
        const int at = base + threadIdx.x * PER;
        unsigned bits = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (at + e < hi && (ref[ASX_AT(at + e, n_pages, 203)] > 0) == used) bits |= 1u << e;
        int total;
        int r = got + block_scan(__popc(bits), warp_sum, total) - __popc(bits);
        for (; bits; bits &= bits - 1, ++r)
            if (r < want) list[ASX_AT(r, n_pages, 204)] = at + __ffs(bits) - 1;
        got += total;
    }
    __syncthreads();
    return min(got, want);
}

// One CTA: which lanes need a page for a copy, and which page each gets.  One, because pages are given out in the order of
// the lanes and by number, which is a scan over both: latency (7 us for 256 lanes).
__global__ void __launch_bounds__(PL_NT) fork_plan_kernel(const ForkArgs a, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int warp_sum[32];
    const int tid = threadIdx.x;
    int wanted = 0;
    for (int base = 0; base < a.lanes_out; base += PL_NT) {
        const int i = base + tid;
        int need = 0;
        if (i < a.lanes_out) {
            const int p = a.parent[i];
            const int len = p >= 0 && p < a.lanes_in ? w.eff[p] : 0;
            need = len > 0 && len % a.page_size != 0 && w.first[p] != i;
        }
        int total;
        const int r = wanted + block_scan(need, warp_sum, total) - need;
        if (i < a.lanes_out) w.off[i] = need ? r : -1;
        wanted += total;
    }
    const int got = collect(a.ref_out, 0, a.n_pages, false, wanted, w.free_page, a.n_pages, warp_sum);
    for (int i = tid; i < a.lanes_out; i += PL_NT) {
        const int p = a.parent[i], r = w.off[i];
        const bool known = p >= 0 && p < a.lanes_in;
        const int eff = known ? w.eff[p] : 0;
        int len = max(eff, 0);
        int status = (p < -1 || p >= a.lanes_in || eff < 0) ? AS_ERR_INVALID_ARG : AS_OK;
        if (r >= 0 && r < got) {
            const int at = ASX_AT(r, a.n_pages, 205), m = ASX_AT(len / a.page_size, a.max_pages, 206), g = w.free_page[at];
            w.src[at] = a.table[(size_t)p * a.max_pages + m];
            w.dst[at] = g;
            a.table_out[(size_t)i * a.max_pages + m] = g;
            a.ref_out[ASX_AT(g, a.n_pages, 207)] = 1;
        } else if (r >= 0) {
            len -= len % a.page_size;
            status = AS_ERR_NO_PAGES;
        }
        a.len_out[i] = len;
        if (a.lane_status) a.lane_status[i] = status;
    }
    if (tid == 0) *w.moves = got;
}

// Copies pages src[r] to dst[r], r < *moves, of every plane.  Bound by HBM: 8 planes of about 256 pages of 72 KB in 27 to 47 us.
__global__ void __launch_bounds__(CP_NT)
copy_pages_kernel(const int* __restrict__ moves, const int* __restrict__ src, const int* __restrict__ dst, char* data, int planes,
                  long long plane_stride, long long page_bytes, int n_pages) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int per_page = (int)((page_bytes + CP_CHUNK - 1) / CP_CHUNK);
    const long long n = (long long)*moves * planes * per_page;
    for (long long i = blockIdx.x; i < n; i += gridDim.x) {
        const int c = (int)(i % per_page);
        const long long rest = i / per_page;
        const int plane = (int)(rest % planes), r = (int)(rest / planes);
        char* at = data + plane * plane_stride;
        const uint4* from = reinterpret_cast<const uint4*>(at + ASX_AT(src[ASX_AT(r, n_pages, 208)], n_pages, 209) * page_bytes);
        uint4* to = reinterpret_cast<uint4*>(at + ASX_AT(dst[r], n_pages, 210) * page_bytes);
        const long long vecs = page_bytes / 16, v0 = (long long)c * (CP_CHUNK / 16) + threadIdx.x;
        uint4 q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (v0 + e * CP_NT < vecs) q[e] = from[v0 + e * CP_NT];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (v0 + e * CP_NT < vecs) to[v0 + e * CP_NT] = q[e];
    }
}

struct GrowArgs {
    const int* add;
    int *table, *len, *ref, *lane_status;
    int lanes, max_pages, page_size, n_pages;
};

// One CTA: pages wanted by each lane, the free pages in order, and who gets which.
__global__ void __launch_bounds__(PL_NT) grow_kernel(const GrowArgs a, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int warp_sum[32];
    const int tid = threadIdx.x;
    const long long most = (long long)a.max_pages * a.page_size;
    int wanted = 0;
    for (int base = 0; base < a.lanes; base += PL_NT) {
        const int i = base + tid;
        int need = 0;
        bool bad = false;
        if (i < a.lanes) {
            const int len = a.len[i], add = a.add[i];
            bad = len < 0 || add < 0 || (long long)len + add > most;
            // (a part page that the lane has given up: its next token would have no place)
            if (!bad && add > 0 && len % a.page_size != 0) bad = a.table[(size_t)i * a.max_pages + ASX_AT(len / a.page_size, a.max_pages, 219)] < 0;
            if (!bad) need = pages_of(len + add, a.page_size) - pages_of(len, a.page_size);
        }
        int total;
        // (more than every page cannot be had: with at most 2^20 pages the sums stay within 32 bits)
        const int r = min(wanted, a.n_pages + 1) + block_scan(min(need, a.n_pages + 1), warp_sum, total) - min(need, a.n_pages + 1);
        if (i < a.lanes) w.off[i] = bad ? -1 : r;
        wanted = min(wanted + total, a.n_pages + 1);
    }
    const int got = collect(a.ref, 0, a.n_pages, false, min(wanted, a.n_pages), w.free_page, a.n_pages, warp_sum);
    for (int i = tid; i < a.lanes; i += PL_NT) {
        const int len = a.len[i], add = a.add[i], r = w.off[i];
        int status = AS_OK;
        if (r < 0) {
            status = AS_ERR_INVALID_ARG;
        } else {
            const int have = pages_of(len, a.page_size), need = pages_of(len + add, a.page_size) - have;
            if (need > 0 && r + need > got) {
                status = AS_ERR_NO_PAGES;
            } else {
                for (int m = 0; m < need; ++m) {
                    const int g = w.free_page[ASX_AT(r + m, a.n_pages, 211)];
                    a.table[(size_t)i * a.max_pages + ASX_AT(have + m, a.max_pages, 212)] = g;
                    a.ref[ASX_AT(g, a.n_pages, 213)] = 1;
                }
                a.len[i] = len + add;
            }
        }
        if (a.lane_status) a.lane_status[i] = status;
    }
}

struct TrimArgs {
    const int *keep, *gone, *table, *len, *ref;
    int *table_out, *len_out, *ref_out, *lane_status;
    int lanes, max_pages, page_size, n_pages;
};

// CTA j: lane j's new length (-1: it is left as it is), judged by the reference counts as they were; its share of the copy of those.  A
// kernel of its own, as the next one changes the counts that this one judges by.  Latency: 5 + 4 us for 1024 lanes of 125 pages, 8 + 7 for 512 of
// 469; a call is bound by the host (12 us).
__global__ void __launch_bounds__(PG_NT) trim_check_kernel(const TrimArgs a, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x;
    if (a.ref_out != a.ref)
        for (int i = blockIdx.x * PG_NT + tid; i < a.n_pages; i += gridDim.x * PG_NT) a.ref_out[i] = a.ref[i];
    for (int j = blockIdx.x; j < a.lanes; j += gridDim.x) {
        const int len = a.len[j], keep = a.keep ? a.keep[j] : len;
        bool bad = len < 0 || len > (long long)a.max_pages * a.page_size || keep < 0;
        const int left = min(len, keep);
        if (!bad) {
            const int* row = a.table + (size_t)j * a.max_pages;
            for (int m = tid; m < pages_of(len, a.page_size); m += PG_NT) {
                const int g = row[ASX_AT(m, a.max_pages, 217)];
                bad |= g < -1 || g >= a.n_pages;
                // the page that ends up as the lane's partly filled last one
                if (!bad && left < len && left % a.page_size != 0 && m == left / a.page_size && g >= 0) bad = a.ref[g] > 1;
            }
        }
        bad = __syncthreads_or(bad);
        if (tid == 0) w.eff[j] = bad ? -1 : left;
    }
}

// CTA j: row j of the new table, its length, and the reference counts of the pages it gives up.
__global__ void __launch_bounds__(PG_NT) trim_table_kernel(const TrimArgs a, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x;
    for (int j = blockIdx.x; j < a.lanes; j += gridDim.x) {
        const int left = w.eff[j], len = a.len[j];
        const int held = left < 0 ? 0 : pages_of(len, a.page_size);
        const int lo = a.gone ? a.gone[2 * j] : 0, hi = a.gone ? min(a.gone[2 * j + 1], left) : 0;
        for (int m = tid; m < a.max_pages; m += PG_NT) {
            const size_t at = (size_t)j * a.max_pages + m;
            int g = a.table[at];
            const long long from = (long long)m * a.page_size;
            if (left >= 0 && (from >= left || (from >= lo && from + a.page_size <= hi))) {
                if (m < held && g >= 0) atomicSub(&a.ref_out[ASX_AT(g, a.n_pages, 218)], 1);
                g = -1;
            }
            a.table_out[at] = g;
        }
        __syncthreads();                    // (every thread has read len)
        if (tid == 0) {
            a.len_out[j] = left < 0 ? len : left;
            if (a.lane_status) a.lane_status[j] = left < 0 ? AS_ERR_INVALID_ARG : AS_OK;
        }
    }
}

// One CTA: the number of pages in use, the holes below it and the pages to move there.  Two ordered scans over the reference
// counts, latency (7 us for 1024 pages).
__global__ void __launch_bounds__(PL_NT) compact_plan_kernel(const int* ref, int* ref_out, int n_pages, int* used_out, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int warp_sum[32];
    const int tid = threadIdx.x;
    int n = 0;
    for (int i = tid; i < n_pages; i += PL_NT) {
        const int r = ref[i];
        n += r > 0;
        w.free_page[i] = i;                             // (a page that does not move, or that nobody holds)
        if (ref_out != ref) ref_out[i] = r;
    }
    int used;
    block_scan(n, warp_sum, used);
    const int holes = collect(ref, 0, used, false, n_pages, w.dst, n_pages, warp_sum);
    const int late = collect(ref, used, n_pages, true, n_pages, w.src, n_pages, warp_sum);
    const int moves = min(holes, late);                 // (they are equal)
    for (int r = tid; r < moves; r += PL_NT) {
        const int s = ASX_AT(w.src[r], n_pages, 214), d = ASX_AT(w.dst[r], n_pages, 215);
        w.free_page[s] = d;                             // where page s went
        ref_out[d] = ref[s];
        ref_out[s] = 0;
    }
    if (tid == 0) { *w.moves = moves; *used_out = used; }
}

__global__ void __launch_bounds__(256)
compact_table_kernel(const int* table, int* table_out, long long n, int n_pages, const int* used, const PageWork w) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int u = *used;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int g = table[i];
        table_out[i] = g >= u && g < n_pages ? w.free_page[ASX_AT(g, n_pages, 216)] : g;
    }
}

static int check_work(const void* work, size_t bytes, int lanes_in, int lanes_out, int n_pages) {
    const size_t need = as_pages_work_bytes(lanes_in, lanes_out, n_pages);
    if (!work || bytes < need) return set_err(AS_ERR_INVALID_ARG, "d_work of %zu bytes is needed", need);
    if (reinterpret_cast<uintptr_t>(work) & 255) return set_err(AS_ERR_INVALID_ARG, "d_work is not 256-byte aligned");
    return AS_OK;
}

static int check_pool(const void* data, int planes, long long plane_stride, long long page_bytes, int n_pages) {
    if (!data) return AS_OK;
    if (planes < 0) return set_err(AS_ERR_INVALID_ARG, "planes = %d must be >= 0", planes);
    if (page_bytes < 16 || page_bytes % 16) return set_err(AS_ERR_INVALID_ARG, "page_bytes = %lld must be a positive multiple of 16", page_bytes);
    if (page_bytes > (1LL << 40) / n_pages) return set_err(AS_ERR_UNSUPPORTED, "a plane must not exceed 2^40 bytes");
    if (plane_stride % 16 || (planes > 1 && plane_stride < page_bytes * n_pages))
        return set_err(AS_ERR_INVALID_ARG, "plane_stride = %lld must be a multiple of 16 and hold n_pages pages", plane_stride);
    if (reinterpret_cast<uintptr_t>(data) & 15) return set_err(AS_ERR_INVALID_ARG, "d_data is not 16-byte aligned");
    return AS_OK;
}

static int check_shape(int lanes, int max_pages, int page_size, int n_pages) {
    if (lanes < 0) return set_err(AS_ERR_INVALID_ARG, "the number of lanes = %d must be >= 0", lanes);
    if (max_pages < 1 || page_size < 1 || n_pages < 1)
        return set_err(AS_ERR_INVALID_ARG, "max_pages = %d, page_size = %d and n_pages = %d must be >= 1", max_pages, page_size, n_pages);
    if ((long long)max_pages * page_size > (1LL << 30) || n_pages > (1 << 20))
        return set_err(AS_ERR_UNSUPPORTED, "max_pages * page_size must not exceed 2^30, n_pages not 2^20");
    return AS_OK;
}

static cudaError_t launch_copy(const PageWork& w, void* data, int planes, long long plane_stride, long long page_bytes, int n_pages, int sms, cudaStream_t st) {
    return launch_after(copy_pages_kernel, 8 * sms, CP_NT, 0, st, (const int*)w.moves, (const int*)w.src, (const int*)w.dst, static_cast<char*>(data), planes, plane_stride,
                        page_bytes, n_pages);
}

static unsigned lanes_grid(int n, int sms) { return (unsigned)(n < 16 * sms ? (n > 0 ? n : 1) : 16 * sms); }

}  // namespace asx

using namespace asx;

extern "C" {

size_t as_pages_work_bytes(int lanes_in, int lanes_out, int n_pages) {
    if (lanes_in < 0 || lanes_out < 0 || n_pages < 0) return 0;
    return (work_ints(lanes_in, lanes_out, n_pages) * sizeof(int) + 255) & ~(size_t)255;
}

int as_pages_fork(const int32_t* d_parent, int lanes_in, int lanes_out, int max_pages, int page_size, int n_pages, const int32_t* d_table,
                  const int32_t* d_len, const int32_t* d_ref, int32_t* d_table_out, int32_t* d_len_out, int32_t* d_ref_out, void* d_data,
                  int planes, long long plane_stride, long long page_bytes, int32_t* d_lane_status, void* d_work, size_t work_bytes,
                  void* stream) {
    int rc = check_shape(lanes_in < 0 ? lanes_in : lanes_out, max_pages, page_size, n_pages);
    if (rc != AS_OK) return rc;
    if ((rc = check_pool(d_data, planes, plane_stride, page_bytes, n_pages)) != AS_OK) return rc;
    if (!d_ref || !d_ref_out || (lanes_out > 0 && (!d_parent || !d_table_out || !d_len_out)) || (lanes_in > 0 && (!d_table || !d_len)))
        return set_err(AS_ERR_INVALID_ARG, "a table, length, reference or parent array is NULL");
    if (lanes_in > 0 && lanes_out > 0 && (d_table == d_table_out || d_len == d_len_out))
        return set_err(AS_ERR_INVALID_ARG, "d_table_out and d_len_out must not be d_table and d_len");
    if ((rc = check_work(d_work, work_bytes, lanes_in, lanes_out, n_pages)) != AS_OK) return rc;
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const PageWork w = carve(d_work, lanes_in, lanes_out, n_pages);
    ForkArgs a;
    a.parent = d_parent; a.table = d_table; a.len = d_len; a.ref = d_ref;
    a.table_out = d_table_out; a.len_out = d_len_out; a.ref_out = d_ref_out; a.lane_status = d_lane_status;
    a.lanes_in = lanes_in; a.lanes_out = lanes_out; a.max_pages = max_pages; a.page_size = page_size; a.n_pages = n_pages;
    cudaError_t e = launch_after(fork_count_kernel, lanes_grid(lanes_in, di->sms), PG_NT, 0, st, a, w);
    if (e == cudaSuccess) e = launch_after(fork_table_kernel, lanes_grid(lanes_in > lanes_out ? lanes_in : lanes_out, di->sms), PG_NT, 0, st, a, w);
    if (e == cudaSuccess) e = launch_after(fork_plan_kernel, 1, PL_NT, 0, st, a, w);
    if (e == cudaSuccess && d_data && planes > 0) e = launch_copy(w, d_data, planes, plane_stride, page_bytes, n_pages, di->sms, st);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "page fork kernel launch");
}

int as_pages_grow(const int32_t* d_add, int lanes, int max_pages, int page_size, int n_pages, int32_t* d_table, int32_t* d_len,
                  int32_t* d_ref, int32_t* d_lane_status, void* d_work, size_t work_bytes, void* stream) {
    int rc = check_shape(lanes, max_pages, page_size, n_pages);
    if (rc != AS_OK) return rc;
    if (lanes == 0) return AS_OK;
    if (!d_add || !d_table || !d_len || !d_ref) return set_err(AS_ERR_INVALID_ARG, "d_add, d_table, d_len or d_ref is NULL");
    if ((rc = check_work(d_work, work_bytes, lanes, lanes, n_pages)) != AS_OK) return rc;
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    GrowArgs a;
    a.add = d_add; a.table = d_table; a.len = d_len; a.ref = d_ref; a.lane_status = d_lane_status;
    a.lanes = lanes; a.max_pages = max_pages; a.page_size = page_size; a.n_pages = n_pages;
    const cudaError_t e = launch_after(grow_kernel, 1, PL_NT, 0, (cudaStream_t)stream, a, carve(d_work, lanes, lanes, n_pages));
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "page grow kernel launch");
}

int as_pages_compact(int lanes, int max_pages, int n_pages, const int32_t* d_table, const int32_t* d_ref, int32_t* d_table_out,
                     int32_t* d_ref_out, int32_t* d_used, void* d_data, int planes, long long plane_stride, long long page_bytes,
                     void* d_work, size_t work_bytes, void* stream) {
    int rc = check_shape(lanes, max_pages, 1, n_pages);
    if (rc != AS_OK) return rc;
    if ((rc = check_pool(d_data, planes, plane_stride, page_bytes, n_pages)) != AS_OK) return rc;
    if (!d_ref || !d_ref_out || !d_used || (lanes > 0 && (!d_table || !d_table_out)))
        return set_err(AS_ERR_INVALID_ARG, "d_table, d_ref, d_table_out, d_ref_out or d_used is NULL");
    if ((rc = check_work(d_work, work_bytes, lanes, lanes, n_pages)) != AS_OK) return rc;
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const PageWork w = carve(d_work, lanes, lanes, n_pages);
    cudaError_t e = launch_after(compact_plan_kernel, 1, PL_NT, 0, st, d_ref, d_ref_out, n_pages, d_used, w);
    const long long n = (long long)lanes * max_pages, blocks = (n + 255) / 256;
    if (e == cudaSuccess && n > 0)
        e = launch_after(compact_table_kernel, (unsigned)(blocks < 16 * di->sms ? blocks : 16 * di->sms), 256, 0, st, d_table, d_table_out, n, n_pages, d_used, w);
    if (e == cudaSuccess && d_data && planes > 0) e = launch_copy(w, d_data, planes, plane_stride, page_bytes, n_pages, di->sms, st);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "page compact kernel launch");
}

int as_pages_trim(const int32_t* d_keep, const int32_t* d_gone, int lanes, int max_pages, int page_size, int n_pages, const int32_t* d_table,
                  const int32_t* d_len, const int32_t* d_ref, int32_t* d_table_out, int32_t* d_len_out, int32_t* d_ref_out,
                  int32_t* d_lane_status, void* d_work, size_t work_bytes, void* stream) {
    int rc = check_shape(lanes, max_pages, page_size, n_pages);
    if (rc != AS_OK) return rc;
    if (!d_ref || !d_ref_out || (lanes > 0 && (!d_table || !d_len || !d_table_out || !d_len_out)))
        return set_err(AS_ERR_INVALID_ARG, "a table, length or reference array is NULL");
    if ((rc = check_work(d_work, work_bytes, lanes, lanes, n_pages)) != AS_OK) return rc;
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const PageWork w = carve(d_work, lanes, lanes, n_pages);
    TrimArgs a;
    a.keep = d_keep; a.gone = d_gone; a.table = d_table; a.len = d_len; a.ref = d_ref;
    a.table_out = d_table_out; a.len_out = d_len_out; a.ref_out = d_ref_out; a.lane_status = d_lane_status;
    a.lanes = lanes; a.max_pages = max_pages; a.page_size = page_size; a.n_pages = n_pages;
    cudaError_t e = launch_after(trim_check_kernel, lanes_grid(lanes, di->sms), PG_NT, 0, st, a, w);
    if (e == cudaSuccess) e = launch_after(trim_table_kernel, lanes_grid(lanes, di->sms), PG_NT, 0, st, a, w);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "page trim kernel launch");
}

}  // extern "C"
