// C-ABI entry points of the 4-bit cache and of attention over it.
#include "as_attend.cuh"
#include "as_attend_tc.cuh"
#include "as_cache4.cuh"
#include "as_units.h"

#include <cmath>

namespace asx {

ASX_BOUNDS_READER(bounds_cache4)

static int check_cache(const as_cache4* c) {
    if (!c) return set_err(AS_ERR_INVALID_ARG, "cache is NULL");
    if (c->n_pages < 1 || c->heads < 1) return set_err(AS_ERR_INVALID_ARG, "n_pages = %d and heads = %d must be >= 1", c->n_pages, c->heads);
    if (c->head_dim != 64 && c->head_dim != 128) return set_err(AS_ERR_UNSUPPORTED, "head_dim = %d is not 64 or 128", c->head_dim);
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return set_err(AS_ERR_UNSUPPORTED, "page_size = %d is not 16, 32, 64 or 128", c->page_size);
    if (!c->d_pages) return set_err(AS_ERR_INVALID_ARG, "d_pages is NULL");
    if (reinterpret_cast<uintptr_t>(c->d_pages) & 15) return set_err(AS_ERR_INVALID_ARG, "d_pages is not 16-byte aligned");
    return AS_OK;
}

static int check_lanes(int dtype, int lanes, int T, const void* table, int max_pages, const void* len, int page_size) {
    if (dtype != AS_F32 && dtype != AS_BF16) return set_err(AS_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (lanes < 0) return set_err(AS_ERR_INVALID_ARG, "lanes = %d must be >= 0", lanes);
    if (T < 1) return set_err(AS_ERR_INVALID_ARG, "T = %d must be >= 1", T);
    if (max_pages < 1) return set_err(AS_ERR_INVALID_ARG, "max_pages = %d must be >= 1", max_pages);
    if ((long long)max_pages * page_size > (1LL << 30) || (long long)lanes * T > (1LL << 30))
        return set_err(AS_ERR_UNSUPPORTED, "max_pages * page_size and lanes * T must not exceed 2^30");
    if (lanes > 0 && (!table || !len)) return set_err(AS_ERR_INVALID_ARG, "d_table or d_len is NULL");
    return AS_OK;
}

static CacheArgs cache_args(const as_cache4* c, int lanes, int T, const int* table, int max_pages, const int* len, int* status) {
    CacheArgs a;
    a.pages = static_cast<char*>(c->d_pages);
    a.n_pages = c->n_pages; a.heads = c->heads;
    a.page_shift = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
    a.k_scale = c->d_k_scale; a.v_scale = c->d_v_scale;
    a.table = table; a.max_pages = max_pages; a.len = len; a.lane_status = status;
    a.lanes = lanes; a.T = T;
    a.by_T.set(T);
    a.by_heads.set(c->heads);
    return a;
}

static int clear_status(int* status, int lanes, cudaStream_t st) {
    if (!status) return AS_OK;
    const cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int) * (size_t)lanes, st);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "lane status");
}

static unsigned grid_of(long long threads, int nt) {
    const long long n = (threads + nt - 1) / nt;
    return (unsigned)(n < (1 << 14) ? n : (1 << 14));       // (the kernels loop)
}

static unsigned block_grid(const CacheArgs& a, int D) { return grid_of((long long)a.lanes * a.T * 2 * a.heads * (D / 16), C4_NT); }
template <int DT, int D>
static void launch_append(const CacheArgs& a, const void* k, long long k_ld, const void* v, long long v_ld, bool vec, cudaStream_t st) {
    using E = typename Io<DT>::type;
    auto kern = vec ? append_kernel<DT, D, true> : append_kernel<DT, D, false>;
    kern<<<block_grid(a, D), C4_NT, 0, st>>>(a, static_cast<const E*>(k), k_ld, static_cast<const E*>(v), v_ld);
}
template <int DT, int D>
static void launch_load(const CacheArgs& a, void* k, void* v, cudaStream_t st) {
    using E = typename Io<DT>::type;
    load_kernel<DT, D><<<block_grid(a, D), C4_NT, 0, st>>>(a, static_cast<E*>(k), static_cast<E*>(v));
}

// ---------------------------------------------------------------------------
// attention: passes and scratch
// ---------------------------------------------------------------------------
enum Kernel { MMA_8, MMA_16, TC_128, TC_256 };      // rows of a tile and the kernel that takes it

struct AttendPlan {
    Kernel own_kernel, pre_kernel;  // of the lanes' own pass and of that over shared beginnings
    PassArgs own, pre;
    int* begin;
    size_t bytes;
};

// The smallest tile that holds an item's rows.  Measured on 32 or 128 lanes of up to 8192 tokens, this tile / the next
// one, us: 4 rows 179.5 / 254.8, 8 rows 183 / 257, 12 rows 89 / 173, 16 rows 84 / 166 (32 lanes) and 271 / 594 (128 lanes), 64 rows
// 165 / 248, 128 rows 156 / 257.  In 32 bits the rows stay with the 8-row kernel: TMEM's operands are f16, and q and P
// take two of them each.
static Kernel kernel_for(int dtype, int rows) {
    if (dtype == AS_F32) return MMA_8;
    return rows <= 8 ? MMA_8 : rows <= 16 ? MMA_16 : rows <= 128 ? TC_128 : TC_256;
}

// The shapes of the passes and where their scratch lies in d_work (sizes alone if d_work is null).
// Scratch for the pass over shared beginnings is there whenever N > 1.
static AttendPlan plan_attend(int dtype, int lanes, int T, int heads, int q_heads, int D, int N, void* d_work) {
    AttendPlan pl = {};
    const int g = q_heads / heads;
    char* base = static_cast<char*>(d_work);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* q = base ? base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return q;
    };
    pl.begin = reinterpret_cast<int*>(take(sizeof(int) * (size_t)(lanes / N)));
    auto pass = [&](PassArgs& p, Kernel& kernel, int n, int group, bool prefix) {
        p.n = n; p.group = group; p.prefix = prefix; p.N = N;
        p.rows = group * T * g;
        kernel = kernel_for(dtype, p.rows);
        const bool tc = kernel == TC_128 || kernel == TC_256;
        p.tile_rows = kernel == MMA_8 ? 8 : kernel == MMA_16 ? 16 : kernel == TC_128 ? 128 : 256;
        p.row_tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
        p.by_row_tiles.set(p.row_tiles);
        p.by_tile_rows.set(p.tile_rows);
        p.by_N.set(N);
        p.unit_shift = 7;               // TC_KV = 32 * AT_W tokens
        const size_t items = (size_t)n * heads * p.row_tiles;
        p.first_run = reinterpret_cast<int*>(take(sizeof(int) * items));
        p.last_run = reinterpret_cast<int*>(take(sizeof(int) * items));
        const size_t state = sizeof(float) * (size_t)p.tile_rows * (D + 2);
        p.part_run = reinterpret_cast<float*>(take(2 * (size_t)(tc ? TC_MAX_CTAS : AT_MAX_RUNS) * state));
        if (N > 1) p.part_item = reinterpret_cast<float*>(take(items * state));
    };
    pass(pl.own, pl.own_kernel, lanes, 1, false);
    if (N > 1) pass(pl.pre, pl.pre_kernel, lanes / N, N, true);
    pl.bytes = at;
    return pl;
}

template <int DT, int D, int NT, bool SOLO>
static cudaError_t launch_mma_runs(const AttendArgs& a, PassArgs& p, int sms, cudaStream_t st) {
    static int per_sm[64] = {0};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = attend_mma_kernel<DT, D, NT, SOLO>;
    if (per_sm[dev] == 0) {
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(AttendSmem<D>));
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, AT_NT, sizeof(AttendSmem<D>));
        if (e != cudaSuccess) return e;
        per_sm[dev] = n > 0 ? n : 1;
    }
    const int most = SOLO ? AT_MAX_RUNS / AT_W : AT_MAX_RUNS, ctas = per_sm[dev] * sms < most ? per_sm[dev] * sms : most;
    p.runs = SOLO ? ctas * AT_W : ctas;
    p.unit_shift = SOLO ? 5 : 7;                    // 32 tokens for a warp, 32 * AT_W for a CTA
    return launch_after(kern, ctas, AT_NT, sizeof(AttendSmem<D>), st, a, p);
}
template <int DT, int D, int NT>
static cudaError_t launch_mma(const AttendArgs& a, PassArgs& p, int sms, cudaStream_t st) {
    // A run for each warp where the items are many, or behind shared beginnings, where they are short; else a run for each
    // CTA, whose four warps share an item's tokens.  1024 items of up to 300 / 1000 / 8192 tokens: 26.5 / 41.9 / 179.7 us by
    // warps, 28.0 / 46.5 / 179.6 us by CTAs; few items leave most warps without a run of their own.
    const bool warps = runs_by_warps((long long)p.n * p.row_tiles, a.c.heads, (long long)a.c.max_pages << a.c.page_shift, p.begin && !p.prefix);
    return warps ? launch_mma_runs<DT, D, NT, true>(a, p, sms, st) : launch_mma_runs<DT, D, NT, false>(a, p, sms, st);
}

template <int D, bool DUAL>
static cudaError_t launch_tc(const AttendArgs& a, PassArgs& p, int sms, cudaStream_t st) {
    static bool attr_set[64] = {false};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = attend_tc_kernel<D, DUAL>;
    if (!attr_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc_smem_bytes<D, DUAL>());
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    p.runs = sms < TC_MAX_CTAS ? sms : TC_MAX_CTAS;
    p.wait_cycles = wait_cycles_now();
    return launch_after(kern, p.runs, TC_NT, tc_smem_bytes<D, DUAL>(), st, a, p);
}

template <int DT, int D>
static cudaError_t launch_pass(const AttendArgs& a, PassArgs& p, Kernel kernel, int sms, cudaStream_t st) {
    if constexpr (DT == AS_BF16) {
        if (kernel == TC_256) return launch_tc<D, true>(a, p, sms, st);
        if (kernel == TC_128) return launch_tc<D, false>(a, p, sms, st);
        if (kernel == MMA_16) return launch_mma<DT, D, 2>(a, p, sms, st);
    }
    return launch_mma<DT, D, 1>(a, p, sms, st);
}

template <int DT, int D>
static int launch_attend(const AttendArgs& a, int N, const int* shared, void* work, int sms, cudaStream_t st) {
    AttendPlan pl = plan_attend(DT, a.c.lanes, a.c.T, a.c.heads, a.q_heads, D, N, work);
    cudaError_t e = cudaSuccess;
    if (shared && N > 1) {
        attend_shared_kernel<<<a.c.lanes / N, 128, 0, st>>>(a.c, N, shared, pl.begin);
        pl.own.begin = pl.pre.begin = pl.begin;
        e = launch_pass<DT, D>(a, pl.pre, pl.pre_kernel, sms, st);
        if (e != cudaSuccess) return cuda_fail(e, "attention kernel launch (shared beginnings)");
    } else {
        pl.own.part_item = nullptr;
    }
    e = launch_pass<DT, D>(a, pl.own, pl.own_kernel, sms, st);
    if (e != cudaSuccess) return cuda_fail(e, "attention kernel launch");
    const long long items = (long long)pl.own.n * pl.own.row_tiles * a.c.heads;
    const dim3 grid((unsigned)(items < 64 * sms ? items : 64 * sms), (pl.own.tile_rows + JOIN_ROWS - 1) / JOIN_ROWS);
    e = launch_after(attend_join_kernel<DT, D>, grid, 128, 0, st, a, pl.own, pl.pre);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "attention join kernel launch");
}

}  // namespace asx

using namespace asx;

extern "C" {

size_t as_cache4_bytes(int n_pages, int heads, int head_dim, int page_size) {
    if (n_pages < 1 || heads < 1 || head_dim < 1 || page_size < 1) return 0;
    return (size_t)n_pages * heads * (page_size / 16) * 18 * head_dim;
}

int as_cache4_append(const as_cache4* cache, const void* d_k, long long k_ld, const void* d_v, long long v_ld, int dtype, int lanes,
                     int T, const int32_t* d_table, int max_pages, const int32_t* d_len, int32_t* d_lane_status, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    const long long row = (long long)cache->heads * cache->head_dim;
    if (k_ld < row || v_ld < row) return set_err(AS_ERR_INVALID_ARG, "k_ld = %lld or v_ld = %lld is smaller than heads * head_dim = %lld", k_ld, v_ld, row);
    if (lanes == 0) return AS_OK;
    if (!d_k || !d_v) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is NULL");
    const int es = dtype == AS_F32 ? 4 : 2;
    const uintptr_t at = reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_v);
    if (at % es) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is not element-aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = clear_status(d_lane_status, lanes, st)) != AS_OK) return rc;
    const bool vec = ((at | (uintptr_t)(k_ld * es) | (uintptr_t)(v_ld * es)) & 15) == 0;
    const CacheArgs a = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    if (dtype == AS_F32) {
        if (cache->head_dim == 64) launch_append<AS_F32, 64>(a, d_k, k_ld, d_v, v_ld, vec, st);
        else launch_append<AS_F32, 128>(a, d_k, k_ld, d_v, v_ld, vec, st);
    } else {
        if (cache->head_dim == 64) launch_append<AS_BF16, 64>(a, d_k, k_ld, d_v, v_ld, vec, st);
        else launch_append<AS_BF16, 128>(a, d_k, k_ld, d_v, v_ld, vec, st);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "cache append kernel launch");
}

int as_cache4_load(const as_cache4* cache, void* d_k, void* d_v, int dtype, int lanes, int T, const int32_t* d_table, int max_pages,
                   const int32_t* d_len, int32_t* d_lane_status, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    if (lanes == 0) return AS_OK;
    if (!d_k || !d_v) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is NULL");
    if ((reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_v)) & 15) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is not 16-byte aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = clear_status(d_lane_status, lanes, st)) != AS_OK) return rc;
    const CacheArgs a = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    if (dtype == AS_F32) {
        if (cache->head_dim == 64) launch_load<AS_F32, 64>(a, d_k, d_v, st);
        else launch_load<AS_F32, 128>(a, d_k, d_v, st);
    } else {
        if (cache->head_dim == 64) launch_load<AS_BF16, 64>(a, d_k, d_v, st);
        else launch_load<AS_BF16, 128>(a, d_k, d_v, st);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "cache load kernel launch");
}

size_t as_cache4_attend_work_bytes(const as_cache4* cache, int dtype, int lanes, int T, int q_heads, int N) {
    // (a shape that the call refuses may not even be planned: its rows may pass 32 bits)
    if (!cache || cache->heads < 1 || (cache->head_dim != 64 && cache->head_dim != 128) || (dtype != AS_F32 && dtype != AS_BF16)) return 0;
    if (lanes < 1 || T < 1 || q_heads < 1 || q_heads % cache->heads || N < 1 || lanes % N) return 0;
    if ((long long)lanes * T > (1LL << 30) || (long long)lanes * T * q_heads > 0x7FFFFFFFLL) return 0;
    return plan_attend(dtype, lanes, T, cache->heads, q_heads, cache->head_dim, N, nullptr).bytes;
}

int as_cache4_attend(const as_cache4* cache, const void* d_q, long long q_ld, int dtype, int lanes, int T, int q_heads,
                     const int32_t* d_table, int max_pages, const int32_t* d_len, double scale, int N, const int32_t* d_shared,
                     void* d_out, float* d_lse, int32_t* d_lane_status, void* d_work, size_t work_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    if (q_heads < 1 || q_heads % cache->heads) return set_err(AS_ERR_INVALID_ARG, "q_heads = %d must be a multiple of heads = %d", q_heads, cache->heads);
    if (q_ld < (long long)q_heads * cache->head_dim) return set_err(AS_ERR_INVALID_ARG, "q_ld = %lld is smaller than q_heads * head_dim", q_ld);
    if (!std::isfinite((float)scale)) return set_err(AS_ERR_INVALID_ARG, "scale = %g must be finite in binary32", scale);
    if (N < 1 || lanes % N) return set_err(AS_ERR_INVALID_ARG, "N = %d must be >= 1 and divide lanes = %d", N, lanes);
    // units of 128 tokens over all lanes, heads and tiles of 8 rows, and rows, are counted in 31 bits
    const long long tiles = ((long long)T * (q_heads / cache->heads) + 7) / 8;
    if ((long long)lanes * T * q_heads > 0x7FFFFFFFLL || !units_fit(lanes * tiles, cache->heads, (long long)max_pages * cache->page_size, 7))
        return set_err(AS_ERR_UNSUPPORTED, "lanes, T, q_heads and max_pages * page_size make more than 2^31 rows or units of work");
    if (lanes == 0) return AS_OK;
    if (!d_q || !d_out) return set_err(AS_ERR_INVALID_ARG, "d_q or d_out is NULL");
    const int es = dtype == AS_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(d_q) % es || (reinterpret_cast<uintptr_t>(d_out) & 15))
        return set_err(AS_ERR_INVALID_ARG, "d_q is not element-aligned or d_out not 16-byte aligned");
    const size_t need = as_cache4_attend_work_bytes(cache, dtype, lanes, T, q_heads, N);
    if (!d_work || work_bytes < need) return set_err(AS_ERR_INVALID_ARG, "d_work of %zu bytes is needed", need);
    if (reinterpret_cast<uintptr_t>(d_work) & 255) return set_err(AS_ERR_INVALID_ARG, "d_work is not 256-byte aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    AttendArgs a;
    a.c = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    a.q = d_q; a.q_ld = q_ld; a.q_heads = q_heads; a.scale = (float)scale; a.out = d_out; a.lse = d_lse;
    a.by_g.set(q_heads / cache->heads);
    a.by_Tg.set(T * (q_heads / cache->heads));
    if (d_lane_status) attend_status_kernel<<<grid_of(lanes, 256), 256, 0, st>>>(a.c);
    if (dtype == AS_F32) return cache->head_dim == 64 ? launch_attend<AS_F32, 64>(a, N, d_shared, d_work, di->sms, st) : launch_attend<AS_F32, 128>(a, N, d_shared, d_work, di->sms, st);
    return cache->head_dim == 64 ? launch_attend<AS_BF16, 64>(a, N, d_shared, d_work, di->sms, st) : launch_attend<AS_BF16, 128>(a, N, d_shared, d_work, di->sms, st);
}

}  // extern "C"
