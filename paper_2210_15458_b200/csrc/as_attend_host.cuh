// Host side of attention over the cache: which kernels run, on which shapes, with which scratch.
#pragma once
#include "as_attend.cuh"
#include "as_attend_tc.cuh"
#include "as_cache4_host.cuh"
#include "as_units.h"

#include <cmath>

namespace asx {

// ---------------------------------------------------------------------------
// attention: passes and scratch
// ---------------------------------------------------------------------------
enum Kernel { MMA_8, MMA_16, TC_128, TC_256 };      // rows of a tile and the kernel that takes it

struct AttendPlan {
    Kernel own_kernel, pre_kernel;  // of the lanes' own pass and of that over shared beginnings
    PassArgs own, pre;
    int* begin;
    int2* shortest;
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
    pl.shortest = reinterpret_cast<int2*>(take(sizeof(int2) * (size_t)(lanes / N)));    // (with a window)
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

template <int DT, int D, int NT, bool SOLO, bool WIN>
static cudaError_t launch_mma_runs(const AttendArgs& a, PassArgs& p, int sms, cudaStream_t st) {
    static int per_sm[64] = {0};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = attend_mma_kernel<DT, D, NT, SOLO, WIN>;
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
template <int DT, int D, int NT, bool WIN>
static cudaError_t launch_mma(const AttendArgs& a, PassArgs& p, int sms, cudaStream_t st) {
    // A run for each warp where the items are many, or behind shared beginnings, where they are short; else a run for each
    // CTA, whose four warps share an item's tokens.  1024 items of up to 300 / 1000 / 8192 tokens: 26.5 / 41.9 / 179.7 us by
    // warps, 28.0 / 46.5 / 179.6 us by CTAs; few items leave most warps without a run of their own.
    const bool warps = runs_by_warps((long long)p.n * p.row_tiles, a.c.heads, (long long)a.c.max_pages << a.c.page_shift, p.begin && !p.prefix);
    return warps ? launch_mma_runs<DT, D, NT, true, WIN>(a, p, sms, st) : launch_mma_runs<DT, D, NT, false, WIN>(a, p, sms, st);
}

template <int D, bool DUAL, bool WIN>
static cudaError_t launch_tc(const AttendArgs& a, PassArgs& p, int sms, cudaStream_t st) {
    static bool attr_set[64] = {false};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = attend_tc_kernel<D, DUAL, WIN>;
    if (!attr_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc_smem_bytes<D, DUAL>());
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    p.runs = sms < TC_MAX_CTAS ? sms : TC_MAX_CTAS;
    p.wait_cycles = wait_cycles_now();
    return launch_after(kern, p.runs, TC_NT, tc_smem_bytes<D, DUAL>(), st, a, p);
}

template <int DT, int D, bool WIN>
static cudaError_t launch_pass(const AttendArgs& a, PassArgs& p, Kernel kernel, int sms, cudaStream_t st) {
    if constexpr (DT == AS_BF16) {
        if (kernel == TC_256) return launch_tc<D, true, WIN>(a, p, sms, st);
        if (kernel == TC_128) return launch_tc<D, false, WIN>(a, p, sms, st);
        if (kernel == MMA_16) return launch_mma<DT, D, 2, WIN>(a, p, sms, st);
    }
    return launch_mma<DT, D, 1, WIN>(a, p, sms, st);
}

// Whether a pass over shared beginnings is worth its three kernels: windows that are small together each lane reads by itself, most of
// them from L2.  Lanes x 8 heads of 128, four query heads to each, contexts of 6000, own / shared, us: 128 lanes, windows of 512 (75 MB)
// 37 / 48..55, 1024 (151 MB) 54 / 53..56, 2048 84 / 62; 32 lanes, 2048 (75 MB) 34 / 48, 4096 49 / 53.
inline bool by_groups(const AttendArgs& a, int D, int window, int sinks) {
    const long long most = (long long)a.c.max_pages << a.c.page_shift, tokens = (long long)window + sinks;
    return window_groups_now() || (long long)a.c.lanes * a.c.heads * (tokens < most ? tokens : most) * (D * 18 / 16) > 1LL << 27;
}

template <int DT, int D, bool WIN>
static int launch_attend(const AttendArgs& a, int N, const int* shared, int window, int sinks, void* work, int sms, cudaStream_t st) {
    AttendPlan pl = plan_attend(DT, a.c.lanes, a.c.T, a.c.heads, a.q_heads, D, N, work);
    pl.own.window = pl.pre.window = window;
    pl.own.sinks = pl.pre.sinks = sinks;
    cudaError_t e = cudaSuccess;
    if (shared && N > 1 && (!WIN || by_groups(a, D, window, sinks))) {
        attend_shared_kernel<<<a.c.lanes / N, 128, 0, st>>>(a.c, N, shared, pl.begin, WIN ? pl.shortest : nullptr);
        pl.own.begin = pl.pre.begin = pl.begin;
        pl.pre.shortest = pl.shortest;
        e = launch_pass<DT, D, WIN>(a, pl.pre, pl.pre_kernel, sms, st);
        if (e != cudaSuccess) return cuda_fail(e, "attention kernel launch (shared beginnings)");
    } else {
        pl.own.part_item = nullptr;
    }
    e = launch_pass<DT, D, WIN>(a, pl.own, pl.own_kernel, sms, st);
    if (e != cudaSuccess) return cuda_fail(e, "attention kernel launch");
    const long long items = (long long)pl.own.n * pl.own.row_tiles * a.c.heads;
    const dim3 grid((unsigned)(items < 64 * sms ? items : 64 * sms), (pl.own.tile_rows + JOIN_ROWS - 1) / JOIN_ROWS);
    e = launch_after(attend_join_kernel<DT, D, WIN>, grid, 128, 0, st, a, pl.own, pl.pre);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "attention join kernel launch");
}

// What as_cache4_attend and as_cache4_weigh check alike.
inline int check_queries(const as_cache4* cache, const void* d_q, long long q_ld, int dtype, int lanes, int T, int q_heads, int max_pages, double scale) {
    if (q_heads < 1 || q_heads % cache->heads) return set_err(AS_ERR_INVALID_ARG, "q_heads = %d must be a multiple of heads = %d", q_heads, cache->heads);
    if (q_ld < (long long)q_heads * cache->head_dim) return set_err(AS_ERR_INVALID_ARG, "q_ld = %lld is smaller than q_heads * head_dim", q_ld);
    if (!std::isfinite((float)scale)) return set_err(AS_ERR_INVALID_ARG, "scale = %g must be finite in binary32", scale);
    // units of 128 tokens over all lanes, heads and tiles of 8 rows, and rows, are counted in 31 bits
    const long long tiles = ((long long)T * (q_heads / cache->heads) + 7) / 8;
    if ((long long)lanes * T * q_heads > 0x7FFFFFFFLL || !units_fit(lanes * tiles, cache->heads, (long long)max_pages * cache->page_size, 7))
        return set_err(AS_ERR_UNSUPPORTED, "lanes, T, q_heads and max_pages * page_size make more than 2^31 rows or units of work");
    return AS_OK;
}
inline int check_scratch(const void* d_work, size_t work_bytes, size_t need) {
    if (!d_work || work_bytes < need) return set_err(AS_ERR_INVALID_ARG, "d_work of %zu bytes is needed", need);
    if (reinterpret_cast<uintptr_t>(d_work) & 255) return set_err(AS_ERR_INVALID_ARG, "d_work is not 256-byte aligned");
    return AS_OK;
}

template <bool WIN>
static int attend(const as_cache4* cache, const void* d_q, long long q_ld, int dtype, int lanes, int T, int q_heads, const int32_t* d_table, int max_pages,
                  const int32_t* d_len, double scale, int N, const int32_t* d_shared, int window, int sinks, void* d_out, float* d_lse, int32_t* d_lane_status,
                  void* d_work, size_t work_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    if ((rc = check_queries(cache, d_q, q_ld, dtype, lanes, T, q_heads, max_pages, scale)) != AS_OK) return rc;
    if (N < 1 || lanes % N) return set_err(AS_ERR_INVALID_ARG, "N = %d must be >= 1 and divide lanes = %d", N, lanes);
    if (lanes == 0) return AS_OK;
    if (!d_q || !d_out) return set_err(AS_ERR_INVALID_ARG, "d_q or d_out is NULL");
    if (reinterpret_cast<uintptr_t>(d_q) % (dtype == AS_F32 ? 4 : 2) || (reinterpret_cast<uintptr_t>(d_out) & 15))
        return set_err(AS_ERR_INVALID_ARG, "d_q is not element-aligned or d_out not 16-byte aligned");
    if ((rc = check_scratch(d_work, work_bytes, as_cache4_attend_work_bytes(cache, dtype, lanes, T, q_heads, N))) != AS_OK) return rc;
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    AttendArgs a;
    a.c = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    a.q = d_q; a.q_ld = q_ld; a.q_heads = q_heads; a.scale = (float)scale; a.out = d_out; a.lse = d_lse;
    a.by_g.set(q_heads / cache->heads);
    a.by_Tg.set(T * (q_heads / cache->heads));
    if (d_lane_status) attend_status_kernel<<<grid_of(lanes, 256), 256, 0, st>>>(a.c);
    auto run = [&](auto go) { return go(a, N, d_shared, window, sinks, d_work, di->sms, st); };
    if (dtype == AS_F32) return cache->head_dim == 64 ? run(launch_attend<AS_F32, 64, WIN>) : run(launch_attend<AS_F32, 128, WIN>);
    return cache->head_dim == 64 ? run(launch_attend<AS_BF16, 64, WIN>) : run(launch_attend<AS_BF16, 128, WIN>);
}

}  // namespace asx
