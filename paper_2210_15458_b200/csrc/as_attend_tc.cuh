// Attention over the 4-bit cache for many query rows on the same tokens (a chunk of a prompt, the lanes
// of a group on their shared beginning): products on the tensor cores with accumulators in TMEM.
#pragma once
#include "as_attend.cuh"

#include <type_traits>

namespace asx {

constexpr int TC_MAX_CTAS = 160;            // one on each SM
constexpr int TC_KV = 128;                  // tokens of a tile
// Threads, in this order: a warp that issues (and three that are not used: a group's first warp reads the first lanes of
// TMEM), a group of 128 that fills in keys (and queries), one that fills in values, two softmax groups.  Their loops run side by side on each quarter of the SM and together have to fit its instruction cache: they
// are kept short, rare parts are calls (unrolled whole, the kernel was instruction-bound and half as fast).
constexpr int TC_SOFT = 256, TC_FILL = 128, TC_FIRST = 128, TC_NT = TC_FIRST + 2 * TC_FILL + TC_SOFT;

__device__ __forceinline__ void tc_bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void tc_bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A wait for a phase of a barrier, bounded: false when the bound has run out here or in another warp.
__device__ __forceinline__ bool tc_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
static __device__ __noinline__ bool tc_wait_long(uint32_t bar, uint32_t parity, long long limit, volatile int* failed) {
    const long long start = clock64();
#pragma unroll 1
    while (!tc_try(bar, parity)) {
        if (*failed) return false;
        if (clock64() - start > limit) { *failed = 1; return false; }
    }
    return true;
}
__device__ __forceinline__ bool tc_wait(uint32_t bar, uint32_t parity, long long limit, volatile int* failed) {
    return tc_try(bar, parity) || tc_wait_long(bar, parity, limit, failed);
}

#define TC_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define TC_W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
__device__ __forceinline__ bool tc_elect() {
    uint32_t e;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e;
}
// 32 columns of the warp's 32 lanes of TMEM: thread = lane
__device__ __forceinline__ void tc_ld32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : TC_R8(r, 0), TC_R8(r, 8), TC_R8(r, 16), TC_R8(r, 24) : "r"(at));
}
__device__ __forceinline__ void tc_st16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::TC_W8(r, 0), TC_W8(r, 8), "r"(at) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : TC_R8(r, 0), TC_R8(r, 8) : "r"(at));
}
// two floats side by side in a 64-bit register, and arithmetic on both
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ float2 unpair(uint64_t x) {
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(x));
    return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// columns at .. at + 16 n of the warp's lanes, each thread's times f: 32-bit sums, or pairs of f16 weights
static __device__ __noinline__ void tc_scale_sums(uint32_t at, int n, float f) {
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        uint32_t o[16];
        tc_ld16(at + 16 * i, o);
        tc_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
        tc_st16(at + 16 * i, o);
    }
}
static __device__ __noinline__ void tc_scale_weights(uint32_t at, int n, float f) {
    tc_wait_st();
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        uint32_t o[16];
        tc_ld16(at + 16 * i, o);
        tc_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float2 h = unpack_f16(o[e]);
            o[e] = pack_f16(h.x * f, h.y * f);
        }
        tc_st16(at + 16 * i, o);
    }
}
// D[tmem] (+)= A x B, f16 in, f32 accumulators; A from shared memory or from TMEM, B from shared memory
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// Matrices lie in shared memory as blocks of 64 columns: rows of 128 bytes, 16-byte pieces swizzled by
// the row's number mod 8 (128-byte swizzle), 8 rows = 1024 bytes.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, uint32_t block_bytes) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)((block_bytes >> 4) & 0x3FFF) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__host__ __device__ constexpr uint32_t tc_idesc(int M, int N, bool b_rows_are_k) {
    return 1u << 4 | (b_rows_are_k ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}
__device__ __forceinline__ uint32_t tc_at(int row, int chunk) { return row * 128 + ((chunk ^ (row & 7)) << 4); }     // 16-byte piece of a block

// 32 elements of a query row, which may start off a 16-byte boundary or not be there
__device__ __forceinline__ void tc_read_row(const uint16_t* from, bool there, bool wide, uint4 (&q)[4]) {
    if (there && wide) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = reinterpret_cast<const uint4*>(from)[i];
        return;
    }
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = there ? from[2 * i] | (uint32_t)from[2 * i + 1] << 16 : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

struct TcSmem {
    unsigned long long k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[2][2], p_full[2][2], pv_done[2], q_full[2], q_empty[2], o_full, o_empty, ml_full, fin;
    uint32_t tmem;
    int failed;
    RunSmem run;
    float up[2][256];                       // factor by which a query row was scaled down, by parity of the item
    float ml[2][2][2][128];                 // [parity][group][m, l][row]
};

template <int D, bool DUAL> constexpr size_t tc_smem_bytes() { return 1024 + (size_t)6 * TC_KV * D * 2 + (size_t)TC_KV * D + sizeof(TcSmem); }

// An item's rows stand in one tile of 128 (DUAL: two).  Filling threads turn 128 tokens at a time into
// f16 keys and values in shared memory, two buffers; the issuing thread runs S = Q K^T into TMEM and
// O += P V with P taken from TMEM; two groups of 128 softmax threads, a thread to a row, turn S into P in
// place.  DUAL: each group has a row tile and takes every tile of tokens; else the groups take the
// tiles of tokens in turn, each with its own m, l and O, joined at the end, and the next item's queries have
// a buffer of their own.  DUAL takes a tile in two pieces of 64 tokens, each with columns of its own: while
// the weights of one are formed, the products of the other run (2 x 2048 tokens over up to 8192: 498 -> 465 us;
// 460 to 480 us in all runs, 848 to 885 TFLOP/s; nothing is busy for more than half of it, waiting is spread over softmax, filling and products).
// The other form waits for the filling, and pieces cost it more than they give (8 x 32 codes behind shared tokens: 89.2 -> 90.1 us).
template <int D, bool DUAL, bool WIN>
__global__ void __launch_bounds__(TC_NT, 1) attend_tc_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ PassArgs p) {
    using Ti = Tile4<D>;
    constexpr int FILL = TC_FIRST / 32, SOFT = FILL + 2 * TC_FILL / 32;     // first warps of the groups
    constexpr int MAT = TC_KV * D * 2, BLK = TC_KV * 128, CHUNKS = D / 8, KSTEPS = D / 16;
    constexpr int PIECES = DUAL ? 2 : 1, PIECE = TC_KV / PIECES;            // of a tile's tokens
    extern __shared__ char raw[];
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(raw) + 1023) & ~1023u;
    const uint32_t q_s = base, k_s = q_s + 2 * MAT, v_s = k_s + 2 * MAT, raw_s = v_s + 2 * MAT;
    TcSmem& sm = *reinterpret_cast<TcSmem*>(raw + (raw_s + TC_KV * D - (uint32_t)__cvta_generic_to_shared(raw)));
    auto bar = [](const unsigned long long& b) { return (uint32_t)__cvta_generic_to_shared(&b); };
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            tc_bar_init(bar(sm.k_full[i]), TC_FILL / 32); tc_bar_init(bar(sm.v_full[i]), TC_FILL / 32);
            tc_bar_init(bar(sm.k_empty[i]), 1); tc_bar_init(bar(sm.v_empty[i]), 1);
            for (int h = 0; h < 2; ++h) { tc_bar_init(bar(sm.s_full[i][h]), 1); tc_bar_init(bar(sm.p_full[i][h]), 4); }
            tc_bar_init(bar(sm.pv_done[i]), 1);
            tc_bar_init(bar(sm.q_full[i]), (DUAL ? 2 : 1) * TC_FILL / 32); tc_bar_init(bar(sm.q_empty[i]), 1 + TC_SOFT / 32);
        }
        tc_bar_init(bar(sm.o_full), 1); tc_bar_init(bar(sm.o_empty), TC_SOFT / 32);
        tc_bar_init(bar(sm.ml_full), TC_SOFT / 32); tc_bar_init(bar(sm.fin), 1);
        sm.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    Cursor<WIN> cu;
    const int run = find_run<TC_NT, 1, WIN>(a, p, sm.run, cu);      // units of the CTA
    if (run == 0) return;
    if (w == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    constexpr uint32_t s_t = 0, o_t = 256;      // TMEM columns: S of group 0, 1 (P in its place), then O of group 0, 1
    const uint32_t tmem = sm.tmem;              // (all 512 columns: 0)
    const long long limit = p.wait_cycles;
    volatile int* failed = &sm.failed;
    bool ok = true;
    int x = 0;                                  // units behind
    // the query buffer of an item, and how often it has been used before
    auto q_buf = [](int item) { return DUAL ? 0 : item & 1; };
    auto q_use = [](int item) { return (uint32_t)(DUAL ? item : item >> 1); };
    auto wait_warp = [&](const unsigned long long& b, uint32_t parity) { return __all_sync(0xFFFFFFFFu, tc_wait(bar(b), parity, limit, failed)); };

    if (w >= SOFT) {
        // ------------------------------------------------ weights ------------------------------------------------
        const int s = (w - SOFT) >> 2, r = tid & 127;
        const uint32_t mine = (uint32_t)(w & 3) << 21;              // the warp's 32 lanes of TMEM
        const uint32_t st = s_t + 128 * s + mine, ot = o_t + 128 * s + mine;
        uint32_t steps = 0;                                         // of this group, ever
#pragma unroll 1
        for (int item = 0; x < run && ok; ++item) {
            const int tiles = min(cu.nu - cu.u, run - x);
            const int row = cu.row0 + (DUAL ? 128 * s : 0) + r;
            int lim, low = 0;                                       // (low: of the row's window)
            if constexpr (WIN) {
                const int rl = row < p.rows ? row_limit(a, cu.lane0, row) : 0;
                lim = row < p.rows ? min(rl - cu.hole.skip, cu.hi) : 0;
                low = max(rl - p.window, 0) - cu.hole.skip;
            } else {
                lim = row < p.rows ? min(row_limit(a, cu.lane0, row), cu.hi) : 0;
            }
            const float vg = c.v_scale ? c.v_scale[cu.head] : 1.f;
            ok = wait_warp(sm.q_full[q_buf(item)], q_use(item) & 1);
            if (!ok) break;
            float k2 = sm.up[item & 1][ASX_AT((DUAL ? 128 * s : 0) + r, 256, 151)] * fabsf(a.scale) * (c.k_scale ? c.k_scale[cu.head] : 1.f) * 1.44269504088896f;
            k2 = fmaxf(k2, 1e-37f);         // (a scale of 0: -inf x k2 stays -inf)
            __syncwarp();
            if (lane == 0) tc_bar_arrive(bar(sm.q_empty[q_buf(item)]));          // (so that no group falls two items behind the filling)
            float m = -INFINITY, mu = 0.f, l = 0.f;
            bool first = true;
#pragma unroll 1
            for (int j = DUAL ? 0 : s; j < tiles && ok; j += DUAL ? 1 : 2, ++steps) {
#pragma unroll 1
              for (int hf = 0; hf < PIECES; ++hf) {
                ok = wait_warp(sm.s_full[s][hf], steps & 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t sh = st + PIECE * hf;
                const int left = lim - (cu.lo + (cu.u + j) * TC_KV + PIECE * hf);   // visible tokens of the piece
                const bool cut = __any_sync(0xFFFFFFFFu, left < PIECE);
                // places [hide, show) of the piece lie in front of the row's window and behind the sinks
                int hide = 0, show = 0;
                bool front = false;
                if constexpr (WIN) {
                    const int at = lim - left;
                    hide = p.sinks - at;
                    show = low - at;
                    front = __any_sync(0xFFFFFFFFu, hide < PIECE && show > 0);
                }
                bool settled = false;
                // One pass over the row, 32 columns at a time.  The running maximum hardly ever rises after the first tiles;
                // where it does, what was written with the old one is scaled.
#pragma unroll 1
                for (int ch = 0; ch < PIECE / 32; ++ch) {
                    uint32_t v[32];
                    tc_ld32(sh + ASX_AT(128 * s + PIECE * hf + 32 * ch, 225, 152) - (128 * s + PIECE * hf), v);
                    tc_wait_ld();
                    if (cut) {
                        const int have = left - 32 * ch;
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = e < have ? v[e] : 0xFF800000u;
                    }
                    if (WIN && front) {
                        const int from = hide - 32 * ch, to = show - 32 * ch;
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = e >= from && e < to ? 0xFF800000u : v[e];
                    }
                    float tops[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        tops[i] = fmaxf(__uint_as_float(v[8 * i]), __uint_as_float(v[8 * i + 1]));
#pragma unroll
                        for (int e = 2; e < 8; e += 2) tops[i] = fmaxf(fmaxf(tops[i], __uint_as_float(v[8 * i + e])), __uint_as_float(v[8 * i + e + 1]));
                    }
                    const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * k2;
                    const bool rise = top > m + AT_RISE<AS_BF16>;
                    if (__any_sync(0xFFFFFFFFu, rise)) {
                        float f = 1.f;
                        if (rise) {
                            mu = top - AT_BELOW<AS_BF16>;
                            f = ex2(m - mu);
                            m = mu;
                            l *= f;
                        }
                        if (!first) {
                            // (the products of the piece before may still be adding to the sums)
                            if (PIECES > 1 && !settled) ok = wait_warp(sm.pv_done[s], (2 * steps + hf - 1) & 1);
                            if (!ok) break;
                            settled = true;
                            tc_scale_sums(ot, D / 16, f);
                        }
                        if (ch > 0) tc_scale_weights(sh, ch, f);
                    }
                    const uint64_t kk = pair(k2, k2), mm = pair(-mu, -mu);
                    uint64_t sum[2] = {0, 0};
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float2 w = unpair(fma2(pair(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), kk, mm));
                        w = make_float2(ex2(w.x), ex2(w.y));
                        sum[e / 2 & 1] = add2(sum[e / 2 & 1], pair(w.x, w.y));
                        pk[e / 2] = pack_f16(w.x, w.y);
                    }
                    const float2 total = unpair(add2(sum[0], sum[1]));
                    l += total.x + total.y;
                    tc_st16(sh + ASX_AT(16 * ch, PIECE / 2 - 15, 157), pk);
                }
                if (!ok) break;
                first = false;
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) tc_bar_arrive(bar(sm.p_full[s][hf]));
              }
              if (!ok) break;
            }
            if (!ok) break;
            // ---- the end of an item or of the run ----
            if (!DUAL) {
                sm.ml[item & 1][ASX_AT(s, 2, 158)][0][r] = m;
                sm.ml[item & 1][s][1][r] = l;
                __syncwarp();
                if (lane == 0) tc_bar_arrive(bar(sm.ml_full));
                ok = wait_warp(sm.ml_full, item & 1);
                if (!ok) break;
            }
            ok = wait_warp(sm.o_full, item & 1);
            if (!ok) break;
            tc_fence_after();
            const bool whole = cu.u == 0 && tiles == cu.nu;
            const size_t at_item = ASX_AT((size_t)cu.entry * c.heads + cu.head, (long long)p.n * p.row_tiles * c.heads, 153);
            if (tid == TC_NT - 1) {
                if (cu.u == 0) p.first_run[at_item] = blockIdx.x;
                if (cu.u + tiles == cu.nu) p.last_run[at_item] = blockIdx.x;
            }
            float* part = nullptr;
            if (!whole) part = p.part_run + (size_t)ASX_AT(2 * blockIdx.x + (cu.u == 0), 2 * TC_MAX_CTAS, 154) * state_floats<D>(p.tile_rows);
            else if (p.part_item) part = p.part_item + at_item * state_floats<D>(p.tile_rows);
            // DUAL: a thread writes its row; else the two groups' states of a row join, and each group writes half of it
            float M = m, L = l, f0 = 1.f, f1 = 0.f;
            if (!DUAL) {
                const float ma = sm.ml[item & 1][0][0][r], mb = sm.ml[item & 1][1][0][r];
                M = fmaxf(ma, mb);
                f0 = ma == -INFINITY ? 0.f : ex2(ma - M);
                f1 = mb == -INFINITY ? 0.f : ex2(mb - M);
                L = f0 * sm.ml[item & 1][0][1][r] + f1 * sm.ml[item & 1][1][1][r];
            }
            const int tr = (DUAL ? 128 * s : 0) + r;
            const size_t orow = row < p.rows ? out_row(a, cu.lane0, cu.head, row) : 0;
            const float inv = L == 0.f ? 0.f : vg / L;
#pragma unroll 1
            for (int ch = 0; ch < (DUAL ? D / 32 : D / 64); ++ch) {
                const int col = ASX_AT((DUAL ? 0 : s * (D / 2)) + 32 * ch, D - 31, 155);
                uint32_t v[32], u[32];
                tc_ld32((DUAL ? ot : o_t + mine) + col, v);
                if (!DUAL) tc_ld32(o_t + 128 + mine + col, u);
                tc_wait_ld();
                float y[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    y[e] = __uint_as_float(v[e]);
                    // (a group that had no tile, or saw nothing, has left no sums of its own)
                    if (!DUAL) y[e] = (f0 > 0.f ? f0 * y[e] : 0.f) + (f1 > 0.f ? f1 * __uint_as_float(u[e]) : 0.f);
                    else if (m == -INFINITY) y[e] = 0.f;
                }
                if (part) {
                    float* at = part + (size_t)ASX_AT(tr, p.tile_rows, 156) * D + col;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(at + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
                } else if (row < p.rows) {
                    __nv_bfloat16* at = static_cast<__nv_bfloat16*>(a.out) + orow * D + col;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t h[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 b2 = __floats2bfloat162_rn(y[e + 2 * i] * inv, y[e + 2 * i + 1] * inv);
                            h[i] = *reinterpret_cast<const uint32_t*>(&b2);
                        }
                        *reinterpret_cast<uint4*>(at + e) = make_uint4(h[0], h[1], h[2], h[3]);
                    }
                }
            }
            if (DUAL || s == 0) {
                if (part) {
                    part[(size_t)p.tile_rows * D + tr] = M;
                    part[(size_t)p.tile_rows * (D + 1) + tr] = L;
                } else if (row < p.rows && a.lse) {
                    a.lse[orow] = L == 0.f ? -INFINITY : 0.693147180559945f * (M + log2f(L));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(bar(sm.o_empty));
            x += tiles;
            if (cu.u + tiles < cu.nu) cu.u += tiles;
            else cu.next_item(a, p);
        }
    } else if (w >= FILL) {
        // ------------------------------------------------ filling ------------------------------------------------
        auto fill = [&](auto which) {
            constexpr bool keys = decltype(which)::value;
            const int r = tid & 127, t = r & 15;                        // token of a tile of 128, row of a query tile
            const int page_mask = (1 << c.page_shift) - 1, tiles_per_page = 1 << (c.page_shift - 4);
            // Each thread takes its token's codes into registers a tile before they are widened, and the page's id a tile
            // before that.  They are widened from the thread's own place in shared memory, by a loop.
            Cursor<WIN> ahead = cu;
            int looked = 0;
            int page = 0, next_lane = 0;
            uint4 code[D / 32];
            uint2 scale = make_uint2(0, 0);                         // keys' scales; values' are bytes apart
            uint32_t byte[KSTEPS];
            bool next_real = false, real = false;
            const char* next_base = c.pages;                        // the token's place within page 0 of its head
            const uint32_t own = raw_s + (keys ? 0 : TC_KV * (D / 2)) + r * 16;
            auto load = [&]() {
                if (next_real && (page < 0 || page >= c.n_pages)) {
#pragma unroll 1
                    for (int j = 0; j < p.group; ++j) flag_lane(c.lane_status, next_lane + j, AS_ERR_INVALID_ARG);
                    page = 0;
                }
                // tokens behind the last one count as zeros: their scales do (any code is finite)
                const char* src = next_real ? next_base + (size_t)page * c.heads * tiles_per_page * Ti::BYTES : c.pages;
                if constexpr (keys) {
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) code[i] = __ldg(reinterpret_cast<const uint4*>(src + Ti::k_code(t, 2 * i)));
                    if constexpr (D == 128) scale = __ldg(reinterpret_cast<const uint2*>(src + Ti::k_scale(t, 0)));
                    else scale.x = __ldg(reinterpret_cast<const uint32_t*>(src + Ti::k_scale(t, 0)));
                } else {
                    uint32_t b1[KSTEPS];
#pragma unroll
                    for (int i = 0; i < KSTEPS; ++i) {
                        const uint2 q = __ldg(reinterpret_cast<const uint2*>(src + Ti::v_code(t, i)));
                        if (i & 1) { code[i / 2].z = q.x; code[i / 2].w = q.y; }
                        else { code[i / 2].x = q.x; code[i / 2].y = q.y; }
                        b1[i] = __ldg(reinterpret_cast<const unsigned char*>(src + Ti::v_scale(t, i)));
                    }
#pragma unroll
                    for (int i = 0; i < KSTEPS; ++i) byte[i] = b1[i];
                }
                real = next_real;
                next_real = false;
                if (looked < run) {
                    int pos = ahead.lo + ahead.u * TC_KV + r;
                    bool seen = pos < ahead.hi;
                    if constexpr (WIN) {
                        seen = seen && !(pos >= p.sinks && pos < ahead.hole.low);
                        pos = ahead.hole.real(pos);
                    }
                    if (seen) {
                        page = c.table[(size_t)ASX_AT(ahead.hole.holder(ahead.lane0), c.lanes, 159) * c.max_pages + ASX_AT(pos >> c.page_shift, c.max_pages, 160)];
                        next_base = c.pages + ((size_t)ASX_AT(ahead.head, c.heads, 161) * tiles_per_page + ((pos & page_mask) >> 4)) * Ti::BYTES;
                        next_lane = ahead.lane0;
                        next_real = true;
                    }
                    ++looked;
                    ahead.step(a, p);
                }
            };
            // 8 codes x scale -> 16 bytes of f16
            auto widen = [](uint32_t codes, uint32_t scale2) {
                uint32_t f[4];
                codes_f16x2(codes, f);
                return make_uint4(mul_f16(f[0], scale2), mul_f16(f[1], scale2), mul_f16(f[2], scale2), mul_f16(f[3], scale2));
            };
            auto put = [](uint32_t at, const uint4& v) { asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); };
            auto filled = [&](uint32_t b) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) tc_bar_arrive(b);
            };
#pragma unroll 1
            for (int i = 0; i < 2; ++i) load();                         // (the first time round only the page id is fetched)
            uint32_t n = 0;                                             // tiles filled
#pragma unroll 1
            for (int item = 0; x < run && ok; ++item) {
                const int tiles = min(cu.nu - cu.u, run - x);
                Cursor<WIN> next = cu;
                if (x + tiles < run) next.next_item(a, p);
                if constexpr (keys || DUAL) {
                    // ---- the item's queries, scaled by a power of two into f16's range; a negative scale goes in here ----
                    if (q_use(item) > 0) ok = wait_warp(sm.q_empty[q_buf(item)], (q_use(item) - 1) & 1);
                    if (!ok) break;
                    {
                        constexpr int h = keys ? 0 : 1;             // (the values' group takes the second row tile)
                        const int row = cu.row0 + 128 * h + r;
                        const bool there = row < p.rows;
                        const uint16_t* from = there ? reinterpret_cast<const uint16_t*>(query_row<AS_BF16, D>(a, cu.lane0, cu.head, row)) : nullptr;
                        const bool wide = (reinterpret_cast<uintptr_t>(from) & 15) == 0;
                        uint32_t top = 0;                               // largest magnitude's bits
                        // (twice over the row, 4 pieces of 8 elements at a time: code that runs once an item is fetched anew each
                        // time, so that a short loop is faster than straight code)
#pragma unroll 1
                        for (int i = 0; i < CHUNKS; i += 4) {
                            uint4 q[4];
                            tc_read_row(from + 8 * i, there, wide, q);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                top = max(max(max(q[e].x & 0x7FFFu, q[e].x >> 16 & 0x7FFFu), max(q[e].y & 0x7FFFu, q[e].y >> 16 & 0x7FFFu)),
                                          max(max(max(q[e].z & 0x7FFFu, q[e].z >> 16 & 0x7FFFu), max(q[e].w & 0x7FFFu, q[e].w >> 16 & 0x7FFFu)), top));
                        }
                        int ex = (int)(top >> 7) - 127;
                        ex = ex > 126 ? 126 : ex < -126 ? -126 : ex;
                        const float down = __uint_as_float((uint32_t)(127 - ex) << 23 | (a.scale < 0.f ? 0x80000000u : 0u));
                        sm.up[item & 1][ASX_AT(128 * h + r, 256, 162)] = __uint_as_float((uint32_t)(127 + ex) << 23);
                        const uint32_t to_q = q_s + (DUAL ? h : q_buf(item)) * MAT;
                        auto both = [&](uint32_t z) { return pack_f16(__uint_as_float(z << 16) * down, __uint_as_float(z & 0xFFFF0000u) * down); };
#pragma unroll 1
                        for (int i = 0; i < CHUNKS; i += 4) {
                            uint4 q[4];
                            tc_read_row(from + 8 * i, there, wide, q);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                put(q_s + ASX_AT(to_q - q_s + (i / 8) * BLK + tc_at(r, (i & 4) + e), 2 * MAT - 15, 163), make_uint4(both(q[e].x), both(q[e].y), both(q[e].z), both(q[e].w)));
                        }
                    }
                    filled(bar(sm.q_full[q_buf(item)]));
                    // the next item's, into L1 meanwhile
                    const int row = next.row0 + 128 * (keys ? 0 : 1) + r;
                    if (x + tiles < run && row < p.rows) {
                        const __nv_bfloat16* from = query_row<AS_BF16, D>(a, next.lane0, next.head, row);
                        asm volatile("prefetch.global.L1 [%0];" ::"l"(from));
                        if (D == 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(from + 64));
                    }
                }
                // ---- its keys or values ----
                const uint32_t to = (keys ? k_s : v_s) + r * 128;
#pragma unroll 1
                for (int j = 0; j < tiles && ok; ++j, ++n) {
                    const int b = n & 1;
                    if (n >= 2) ok = wait_warp(keys ? sm.k_empty[b] : sm.v_empty[b], ((n >> 1) & 1) ^ 1);
                    if (!ok) break;
                    // piece i of a token's codes lies TC_KV * 16 bytes behind piece i - 1: threads side by side, 16 bytes each
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) put(raw_s + ASX_AT(own - raw_s + i * (TC_KV * 16), TC_KV * D - 15, 164), code[i]);
                    if constexpr (!keys) {
                        scale.x = byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24;
                        if constexpr (D == 128) scale.y = byte[KSTEPS - 4] | byte[KSTEPS - 3] << 8 | byte[KSTEPS - 2] << 16 | byte[KSTEPS - 1] << 24;
                    }
                    const uint32_t sc_lo = real ? scale.x : 0u, sc_hi = real ? scale.y : 0u;
                    load();
#pragma unroll 1
                    for (int i = 0; i < D / 32; ++i) {
                        const uint4 q = lds<uint4>(raw_s + ASX_AT(own - raw_s + i * (TC_KV * 16), TC_KV * D - 15, 165));
                        const uint32_t two = e4m3_f16x2(((D == 128 && i >= 2 ? sc_hi : sc_lo) >> (16 * (i & 1))) & 0xFFFFu);
                        const uint32_t sa = __byte_perm(two, two, 0x1010), sb = __byte_perm(two, two, 0x3232);
                        const uint32_t at = (keys ? k_s : v_s) + ASX_AT(to - (keys ? k_s : v_s) + b * MAT + (i >> 1) * BLK, 2 * MAT - 127, 166);
                        const int cx = (4 * (i & 1)) ^ (r & 7);
                        put(at + ((cx ^ 0) << 4), widen(q.x, sa));
                        put(at + ((cx ^ 1) << 4), widen(q.y, sa));
                        put(at + ((cx ^ 2) << 4), widen(q.z, sb));
                        put(at + ((cx ^ 3) << 4), widen(q.w, sb));
                    }
                    filled(bar(keys ? sm.k_full[b] : sm.v_full[b]));
                }
                x += tiles;
                cu = next;                                          // (an item ends, or the run does)
            }
        };
        if (w < FILL + TC_FILL / 32) fill(std::true_type{});
        else fill(std::false_type{});
    } else {
        // ------------------------------------------------ issuing ------------------------------------------------
        if (w == 0 && tc_elect()) {
            // One thread walks the steps.  (Chosen by elect.sync, not by its number: 8 products then take 512 cycles in place of
            // 920 beside the other groups' warps.  TMEM, allocated whole, starts at 0.)
            constexpr uint32_t ID_S = tc_idesc(128, PIECE, false), ID_O = tc_idesc(128, D, true);
            constexpr int HALF = (PIECE * 128) >> 4, QS = DUAL ? 4 : 1, AHEAD = DUAL ? 1 : 2;   // QS: pieces (group, half) of a tile
            const uint64_t q_d = tc_desc(q_s, 0), k_d = tc_desc(k_s, 0), v_d = tc_desc(v_s, BLK);
            uint32_t n0 = 0, seen[2] = {0, 0};                      // tiles before this item; tiles of weights taken, by group
#pragma unroll 1
            for (int item = 0; x < run && ok; ++item) {
                const int tiles = min(cu.nu - cu.u, run - x);
                ok = tc_wait(bar(sm.q_full[q_buf(item)]), q_use(item) & 1, limit, failed);
                // scores of piece z of tile j, into the columns that the piece has
                auto scores = [&](int j, int z) {
                    const int s = DUAL ? z & 1 : j & 1, hf = DUAL ? z >> 1 : 0;
                    const uint32_t n = n0 + j, b = n & 1;
                    if (z == 0) {
                        ok = tc_wait(bar(sm.k_full[b]), (n >> 1) & 1, limit, failed);
                        if (!ok) return;
                        tc_fence_after();
                    }
                    const uint64_t qa = q_d + (DUAL ? s : q_buf(item)) * (MAT >> 4), ka = k_d + b * (MAT >> 4) + hf * HALF;
#pragma unroll
                    for (int k = 0; k < KSTEPS; ++k) {
                        const uint32_t at = (k / 4) * (BLK >> 4) + (k % 4) * 2;
                        tc_mma_ss(s_t + 128 * s + PIECE * hf, qa + at, ka + at, ID_S, k > 0);
                    }
                    tc_commit(bar(sm.s_full[s][hf]));
                    if (z == QS - 1) {
                        tc_commit(bar(sm.k_empty[b]));
                        if (j + 1 == tiles) tc_commit(bar(sm.q_empty[q_buf(item)]));
                    }
                };
#pragma unroll 1
                for (int z = 0; z < QS * AHEAD && ok; ++z)
                    if (z / QS < tiles) scores(z / QS, z % QS);
#pragma unroll 1
                for (int j = 0; j < tiles && ok; ++j) {
                    const uint32_t n = n0 + j, b = n & 1;
                    if (j == 0 && item > 0) ok = tc_wait(bar(sm.o_empty), (item - 1) & 1, limit, failed);
                    if (ok) ok = tc_wait(bar(sm.v_full[b]), (n >> 1) & 1, limit, failed);
#pragma unroll 1
                    for (int z = 0; z < QS && ok; ++z) {
                        const int s = DUAL ? z & 1 : j & 1, hf = DUAL ? z >> 1 : 0;
                        ok = tc_wait(bar(sm.p_full[s][hf]), (s ? seen[1] : seen[0]) & 1, limit, failed);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t va = v_d + b * (MAT >> 4) + hf * HALF;
                        const bool add = j >= AHEAD || hf > 0;
#pragma unroll
                        for (int k = 0; k < PIECE / 16; ++k)
                            tc_mma_ts(o_t + 128 * s, s_t + 128 * s + PIECE * hf + 8 * k, va + k * (2048 >> 4), ID_O, k > 0 || add);
                        if constexpr (PIECES > 1) tc_commit(bar(sm.pv_done[s]));
                        if (z == QS - 1) {
                            tc_commit(bar(sm.v_empty[b]));
                            if (j + 1 == tiles) tc_commit(bar(sm.o_full));
                        }
                        if (hf == PIECES - 1) { if (s) ++seen[1]; else ++seen[0]; }
                        if (j + AHEAD < tiles) scores(j + AHEAD, z);
                    }
                }
                if (!ok) break;
                n0 += tiles;
                x += tiles;
                if (cu.u + tiles < cu.nu) cu.u += tiles;
                else cu.next_item(a, p);
            }
            // whatever is still in flight ends before TMEM is freed
            tc_commit(bar(sm.fin));
            const long long start = clock64();
#pragma unroll 1
            while (!tc_try(bar(sm.fin), 0) && clock64() - start < 2000000000LL) {}     // (whatever the bound on the other waits)
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (sm.failed && tid == 0) {
#pragma unroll 1
        for (int j = 0; j < c.lanes; ++j) flag_lane(c.lane_status, j, AS_ERR_TIMEOUT);
    }
    if (w == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

}  // namespace asx
