// C-ABI entry point of the cached tokens' attention weights.
#include "as_attend_host.cuh"
#include "as_weigh.cuh"
#include "as_weigh_tc.cuh"

namespace asx {

ASX_BOUNDS_READER(bounds_weigh)

// bf16 rows beyond 48 go to the tensor cores' 128-row tiles; up to 48 are taken 16 at a time by the instructions on registers.  32 lanes of up to
// 8192 tokens, 8 heads, registers / tensor cores, us: 16 rows 53 / 283, 20 to 32 rows 151 / 271..292, 64 rows 297 / 275, 128 rows 653 / 301.  32-bit
// ones stay on registers whatever their number: an f16 operand holds half of one.
static bool many_rows(int dtype, int rows) { return dtype == AS_BF16 && rows > 48; }

struct WeighPlan {
    int *eff, *from, *begin, *steps;
    char* tiles;
    float* part;
    int4* info;
    size_t bytes;
};

// Where the scratch lies in d_work (sizes alone if it is null).
static WeighPlan plan_weigh(int dtype, int lanes, int T, int heads, int q_heads, int D, void* d_work) {
    WeighPlan pl = {};
    char* base = static_cast<char*>(d_work);
    auto take = [&](size_t bytes) {
        char* q = base ? base + pl.bytes : nullptr;
        pl.bytes += (bytes + 255) & ~(size_t)255;
        return q;
    };
    for (int** q : {&pl.eff, &pl.from, &pl.begin}) *q = reinterpret_cast<int*>(take(sizeof(int) * (size_t)lanes));
    const int rows = T * (q_heads / heads);
    if (many_rows(dtype, rows)) {
        pl.steps = reinterpret_cast<int*>(take(sizeof(int) * (size_t)lanes));
        pl.part = reinterpret_cast<float*>(take(sizeof(float) * 2 * WT_MAX_RUNS * TC_KV));
        pl.info = reinterpret_cast<int4*>(take(sizeof(int4) * WT_MAX_RUNS));
        pl.tiles = take((size_t)lanes * heads * ((rows + WT_ROWS - 1) / WT_ROWS) * (D == 128 ? WT_TILE<128> : WT_TILE<64>));
    }
    return pl;
}

// One CTA per lane: the length and beginning that the other kernels use, the lane's status, 0 for the places that no row looks at (in
// between the sinks and the first row's window) where sums are not added to older ones, and the lane's steps if the tensor cores are to
// take them (t.steps not null).  Latency, 3 to 5 us.
static __global__ void __launch_bounds__(128) weigh_start_kernel(const __grid_constant__ WeighTcArgs t, const CacheArgs c, const int* first, int* eff, int* from, int* begin, int* steps) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int sum;
    const WeighArgs& w = t.w;
    for (int b = blockIdx.x; b < c.lanes; b += gridDim.x) {
        bool bad;
        int len = lane_len(c, b, &bad);
        const int f = first ? first[b] : 0;
        bad = bad || len > w.weight_ld || f < 0 || f > len;
        if (bad) len = 0;
        if (threadIdx.x == 0) {
            eff[b] = len;
            from[b] = bad ? 0 : f;
            begin[b] = bad ? 0 : f & ~15;
            if (c.lane_status) c.lane_status[b] = bad ? AS_ERR_INVALID_ARG : AS_OK;
            sum = 0;
        }
        if (!w.add && !bad) {
            const int lo = max(f, w.p.sinks), hi = min(len, len - c.T + 1 - w.p.window);
            for (int h = 0; h < c.heads; ++h)
                for (int k = lo + threadIdx.x; k < hi; k += 128) w.weight[((size_t)b * c.heads + h) * w.weight_ld + k] = 0.f;
        }
        if (!steps) continue;
        __syncthreads();                    // (the lane's length and beginning are read again)
        const WeighLane l(w, b);
        int mine = 0;
        for (int i = threadIdx.x; i < l.tiles(); i += 128) mine += l.row_span(w, i).y;
        atomicAdd(&sum, mine);
        __syncthreads();
        if (threadIdx.x == 0) steps[b] = sum;
        __syncthreads();
    }
}

template <int DT, int D, int NT, bool MANY>
static cudaError_t launch_weigh_mma(WeighArgs& wa, int sms, cudaStream_t st) {
    static int per_sm[64] = {0};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = weigh_mma_kernel<DT, D, NT, MANY>;
    if (per_sm[dev] == 0) {
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(WeighSmem<D>));
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, WG_NT, sizeof(WeighSmem<D>));
        if (e != cudaSuccess) return e;
        per_sm[dev] = n > 0 ? n : 1;
    }
    const int ctas = per_sm[dev] * sms;
    wa.p.runs = ctas * WG_W;
    wa.p.unit_shift = 5;
    return launch_after(kern, ctas, WG_NT, sizeof(WeighSmem<D>), st, wa);
}

template <int D>
static cudaError_t launch_weigh_tc(const WeighArgs& wa, const WeighPlan& pl, int sms, cudaStream_t st) {
    static bool attr_set[64] = {false};
    int dev = 0;
    cudaGetDevice(&dev);
    if (!attr_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(weigh_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)weigh_tc_smem<D>());
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    WeighTcArgs t;
    t.w = wa;
    t.w.p.wait_cycles = wait_cycles_now();
    t.tiles = pl.tiles; t.steps = pl.steps; t.part = pl.part; t.info = pl.info;
    t.row_tiles = (wa.p.rows + WT_ROWS - 1) / WT_ROWS;
    t.runs = sms < WT_MAX_RUNS ? sms : WT_MAX_RUNS;
    const int lanes = wa.a.c.lanes;
    const long long items = (long long)lanes * wa.a.c.heads * t.row_tiles;
    cudaError_t e = launch_after(weigh_rows_kernel<D>, (unsigned)(items < 64 * sms ? items : 64 * sms), 256, 0, st, t);
    if (e == cudaSuccess) e = launch_after(weigh_tc_kernel<D>, t.runs, WT_NT, weigh_tc_smem<D>(), st, t);
    if (e == cudaSuccess) e = launch_after(weigh_join_kernel, t.runs, TC_KV, 0, st, t);
    return e;
}

template <int DT, int D>
static int launch_weigh(WeighArgs& wa, const WeighPlan& pl, int sms, cudaStream_t st) {
    cudaError_t e;
    if (many_rows(DT, wa.p.rows)) e = launch_weigh_tc<D>(wa, pl, sms, st);
    else if (DT == AS_BF16 && wa.p.rows > 16) e = launch_weigh_mma<DT, D, DT == AS_BF16 ? 2 : 1, true>(wa, sms, st);
    else if (DT == AS_BF16 && wa.p.rows > 8) e = launch_weigh_mma<DT, D, DT == AS_BF16 ? 2 : 1, false>(wa, sms, st);
    else if (DT == AS_F32 && wa.p.rows > 8) e = launch_weigh_mma<DT, D, 1, DT == AS_F32>(wa, sms, st);
    else e = launch_weigh_mma<DT, D, 1, false>(wa, sms, st);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "weigh kernel launch");
}

}  // namespace asx

using namespace asx;

extern "C" {

size_t as_cache4_weigh_work_bytes(const as_cache4* cache, int dtype, int lanes, int T, int q_heads) {
    if (!cache || cache->heads < 1 || (cache->head_dim != 64 && cache->head_dim != 128) || (dtype != AS_F32 && dtype != AS_BF16)) return 0;
    if (lanes < 1 || T < 1 || q_heads < 1 || q_heads % cache->heads) return 0;
    if ((long long)lanes * T > (1LL << 30) || (long long)lanes * T * q_heads > 0x7FFFFFFFLL) return 0;
    return plan_weigh(dtype, lanes, T, cache->heads, q_heads, cache->head_dim, nullptr).bytes;
}

int as_cache4_weigh(const as_cache4* cache, const void* d_q, long long q_ld, int dtype, int lanes, int T, int q_heads, const float* d_lse,
                    const int32_t* d_table, int max_pages, const int32_t* d_len, double scale, int window, int sinks, int add,
                    const int32_t* d_first, float* d_weight, long long weight_ld, int32_t* d_lane_status, void* d_work, size_t work_bytes,
                    void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    if ((rc = check_queries(cache, d_q, q_ld, dtype, lanes, T, q_heads, max_pages, scale)) != AS_OK) return rc;
    if (window < 0 || sinks < 0) return set_err(AS_ERR_INVALID_ARG, "window = %d and sinks = %d must be >= 0", window, sinks);
    if (weight_ld < 1) return set_err(AS_ERR_INVALID_ARG, "weight_ld = %lld must be >= 1", weight_ld);
    // (the keys of 32 tokens are a warp's unit of work)
    if (!units_fit(lanes, cache->heads, (long long)max_pages * cache->page_size, 5)) return set_err(AS_ERR_UNSUPPORTED, "lanes, heads and max_pages * page_size make more than 2^31 units of work");
    if (lanes == 0) return AS_OK;
    if (!d_q || !d_lse || !d_weight) return set_err(AS_ERR_INVALID_ARG, "d_q, d_lse or d_weight is NULL");
    if (reinterpret_cast<uintptr_t>(d_q) % (dtype == AS_F32 ? 4 : 2) || (reinterpret_cast<uintptr_t>(d_lse) | reinterpret_cast<uintptr_t>(d_weight)) % 4)
        return set_err(AS_ERR_INVALID_ARG, "d_q, d_lse or d_weight is not element-aligned");
    if ((rc = check_scratch(d_work, work_bytes, as_cache4_weigh_work_bytes(cache, dtype, lanes, T, q_heads))) != AS_OK) return rc;
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    constexpr int most = 1 << 30;                   // (a lane has at most 2^30 positions)
    const WeighPlan pl = plan_weigh(dtype, lanes, T, cache->heads, q_heads, cache->head_dim, d_work);
    WeighArgs wa = {};
    wa.a.c = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    const int g = q_heads / cache->heads, win = window == 0 || window > most ? most : window, sk = sinks < most ? sinks : most;
    wa.a.c.len = pl.eff;
    wa.a.q = d_q; wa.a.q_ld = q_ld; wa.a.q_heads = q_heads; wa.a.scale = (float)scale;
    wa.a.by_g.set(g);
    wa.a.by_Tg.set(T * g);
    PassArgs& p = wa.p;
    p.n = lanes; p.group = 1; p.N = 1; p.begin = pl.begin;
    p.rows = p.tile_rows = T * g;
    p.row_tiles = 1;
    p.by_row_tiles.set(1); p.by_tile_rows.set(p.tile_rows); p.by_N.set(1);
    p.window = win; p.sinks = sk;
    wa.lse = d_lse; wa.first = pl.from; wa.weight = d_weight; wa.weight_ld = weight_ld; wa.add = add != 0;
    WeighTcArgs t = {};
    t.w = wa;
    const cudaError_t e = launch_after(weigh_start_kernel, (unsigned)(lanes < 16 * di->sms ? lanes : 16 * di->sms), 128, 0, st, t,
                                       cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status), (const int*)d_first, pl.eff, pl.from, pl.begin, pl.steps);
    if (e != cudaSuccess) return cuda_fail(e, "weigh start kernel launch");
    if (dtype == AS_F32) return cache->head_dim == 64 ? launch_weigh<AS_F32, 64>(wa, pl, di->sms, st) : launch_weigh<AS_F32, 128>(wa, pl, di->sms, st);
    return cache->head_dim == 64 ? launch_weigh<AS_BF16, 64>(wa, pl, di->sms, st) : launch_weigh<AS_BF16, 128>(wa, pl, di->sms, st);
}

}  // extern "C"
