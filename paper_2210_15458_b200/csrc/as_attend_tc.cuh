// Attention over the 4-bit cache for many query rows on the same tokens (a chunk of a prompt, the lanes
// of a group on their shared beginning): products on the tensor cores with accumulators in TMEM.
#pragma once
#include "as_attend.cuh"

namespace asx {

constexpr int TC_MAX_CTAS = 160;            // one on each SM
constexpr int TC_KV = 128;                  // tokens of a tile
constexpr int TC_SOFT = 256, TC_FILL = 128; // threads: two softmax groups, one filling group, one warp that issues
constexpr int TC_NT = TC_SOFT + TC_FILL + 32;

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
__device__ __forceinline__ bool tc_wait(uint32_t bar, uint32_t parity, long long limit, volatile int* failed) {
    long long start = 0;
    for (int spin = 0;; ++spin) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if (*failed) return false;
        if (spin == 0) start = clock64();
        else if (clock64() - start > limit) { *failed = 1; return false; }
    }
}

#define TC_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define TC_W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the warp's 32 lanes of TMEM: thread = lane
__device__ __forceinline__ void tc_ld32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : TC_R8(r, 0), TC_R8(r, 8), TC_R8(r, 16), TC_R8(r, 24) : "r"(at));
}
__device__ __forceinline__ void tc_st32(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 ::TC_W8(r, 0), TC_W8(r, 8), TC_W8(r, 16), TC_W8(r, 24), "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::TC_W8(r, 0), TC_W8(r, 8), "r"(at) : "memory");
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

struct TcSmem {
    unsigned long long k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[2], p_full[2], q_full, q_empty, o_full, o_empty, ml_full, fin;
    uint32_t tmem;
    int failed;
    RunSmem run;
    float up[2][256];                       // factor by which a query row was scaled down, by parity of the item
    float ml[2][2][2][128];                 // [parity][group][m, l][row]
};

template <int D, bool DUAL> constexpr size_t tc_smem_bytes() { return 1024 + (size_t)(DUAL ? 6 : 5) * TC_KV * D * 2 + sizeof(TcSmem); }

// An item's rows stand in one tile of 128 (DUAL: two).  Filling threads turn 128 tokens at a time into
// f16 keys and values in shared memory, two buffers; the issuing thread runs S = Q K^T into TMEM and
// O += P V with P taken from TMEM; two groups of 128 softmax threads, a thread to a row, turn S into P in
// place.  DUAL: each group has a row tile and takes every tile of tokens; else the groups take the
// tiles of tokens in turn, each with its own m, l and O, joined at the end.  Either way step i belongs to
// group i % 2, so that one group's products run while the other's weights are formed.
template <int D, bool DUAL>
__global__ void __launch_bounds__(TC_NT, 1) attend_tc_kernel(const AttendArgs a, const PassArgs p) {
    using Ti = Tile4<D>;
    constexpr int MAT = TC_KV * D * 2, BLK = TC_KV * 128, CHUNKS = D / 8, KSTEPS = D / 16;
    extern __shared__ char raw[];
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(raw) + 1023) & ~1023u;
    const uint32_t q_s = base, k_s = q_s + (DUAL ? 2 : 1) * MAT, v_s = k_s + 2 * MAT;
    TcSmem& sm = *reinterpret_cast<TcSmem*>(raw + (v_s + 2 * MAT - (uint32_t)__cvta_generic_to_shared(raw)));
    auto bar = [](const unsigned long long& b) { return (uint32_t)__cvta_generic_to_shared(&b); };
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, g = a.q_heads / c.heads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            tc_bar_init(bar(sm.k_full[i]), TC_FILL / 32); tc_bar_init(bar(sm.v_full[i]), TC_FILL / 32);
            tc_bar_init(bar(sm.k_empty[i]), 1); tc_bar_init(bar(sm.v_empty[i]), 1);
            tc_bar_init(bar(sm.s_full[i]), 1); tc_bar_init(bar(sm.p_full[i]), 4);
        }
        tc_bar_init(bar(sm.q_full), TC_FILL / 32); tc_bar_init(bar(sm.q_empty), 1 + TC_SOFT / 32);
        tc_bar_init(bar(sm.o_full), 1); tc_bar_init(bar(sm.o_empty), TC_SOFT / 32);
        tc_bar_init(bar(sm.ml_full), TC_SOFT / 32); tc_bar_init(bar(sm.fin), 1);
        sm.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    long long x0, x1;
    Cursor cu;
    if (!find_run<TC_NT>(c, p, g, sm.run, x0, x1, cu)) return;
    if (w == TC_NT / 32 - 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem, s_t = tmem, o_t = tmem + 256;    // columns: S of group 0, 1 (P in its place), then O of group 0, 1
    const long long limit = p.wait_cycles;
    volatile int* failed = &sm.failed;
    bool ok = true;
    long long x = x0;
    auto wait_warp = [&](const unsigned long long& b, uint32_t parity) { return __all_sync(0xFFFFFFFFu, tc_wait(bar(b), parity, limit, failed)); };

    if (w < TC_SOFT / 32) {
        // ------------------------------------------------ weights ------------------------------------------------
        const int s = w >> 2, r = tid & 127;
        const uint32_t mine = (uint32_t)(w & 3) << 21;              // the warp's 32 lanes of TMEM
        const uint32_t st = s_t + 128 * s + mine, ot = o_t + 128 * s + mine;
        uint32_t steps = 0;                                         // of this group, ever
        for (int item = 0; x < x1 && ok; ++item) {
            const int tiles = (int)min((long long)(cu.nu - cu.u), x1 - x);
            const int row = (cu.entry % p.row_tiles) * p.tile_rows + (DUAL ? 128 * s : 0) + r;
            const int lane0 = cu.row_of_table(p);
            const int ln = lane0 + row / (c.T * g), t = row / g % c.T;
            const int lim = row < p.rows ? min(lane_len(c, ln) - c.T + 1 + t, cu.hi) : 0;
            const float vg = c.v_scale ? c.v_scale[cu.head] : 1.f;
            ok = wait_warp(sm.q_full, item & 1);
            if (!ok) break;
            const float k2 = sm.up[item & 1][(DUAL ? 128 * s : 0) + r] * fabsf(a.scale) * (c.k_scale ? c.k_scale[cu.head] : 1.f) * 1.44269504088896f;
            __syncwarp();
            if (lane == 0) tc_bar_arrive(bar(sm.q_empty));          // (so that no group falls two items behind the filling)
            float m = -INFINITY, mu = 0.f, l = 0.f;
            bool first = true;
            for (int j = DUAL ? 0 : s; j < tiles && ok; j += DUAL ? 1 : 2, ++steps) {
                ok = wait_warp(sm.s_full[s], steps & 1);
                if (!ok) break;
                tc_fence_after();
                const int left = lim - (cu.lo + (cu.u + j) * TC_KV);        // visible tokens of the tile
                const bool cut = __any_sync(0xFFFFFFFFu, left < TC_KV);
                float top = -INFINITY;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    uint32_t v[32];
                    tc_ld32(st + 32 * ch, v);
                    tc_wait_ld();
                    if (cut) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * ch + e < left) top = fmaxf(top, __uint_as_float(v[e]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) top = fmaxf(top, __uint_as_float(v[e]));
                    }
                }
                top = top == -INFINITY ? top : top * k2;
                const bool rise = top > m + AT_LAZY;
                if (__any_sync(0xFFFFFFFFu, rise)) {
                    float f = 1.f;
                    if (rise) {
                        f = ex2(m - top);
                        m = mu = top;
                        l *= f;
                    }
                    if (!first) {
#pragma unroll
                        for (int ch = 0; ch < D / 32; ++ch) {
                            uint32_t v[32];
                            tc_ld32(ot + 32 * ch, v);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                            tc_st32(ot + 32 * ch, v);
                        }
                    }
                }
                first = false;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    uint32_t v[32], pk[16];
                    tc_ld32(st + 32 * ch, v);
                    tc_wait_ld();
                    float l0 = 0.f, l1 = 0.f;
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float p0 = ex2(fmaf(__uint_as_float(v[e]), k2, -mu)), p1 = ex2(fmaf(__uint_as_float(v[e + 1]), k2, -mu));
                        if (cut) {
                            if (32 * ch + e >= left) p0 = 0.f;
                            if (32 * ch + e + 1 >= left) p1 = 0.f;
                        }
                        l0 += p0; l1 += p1;
                        pk[e / 2] = pack_f16(p0, p1);
                    }
                    l += l0 + l1;
                    tc_st16(st + 16 * ch, pk);
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) tc_bar_arrive(bar(sm.p_full[s]));
            }
            if (!ok) break;
            // ---- the end of an item or of the run ----
            if (!DUAL) {
                sm.ml[item & 1][s][0][r] = m;
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
            float* part = nullptr;
            if (!whole) part = p.part_cta + (size_t)(2 * blockIdx.x + (cu.u == 0)) * state_floats<D>(p.tile_rows);
            else if (p.part_item) part = p.part_item + ((size_t)cu.entry * c.heads + cu.head) * state_floats<D>(p.tile_rows);
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
            const size_t orow = ((size_t)ln * c.T + t) * a.q_heads + cu.head * g + row % g;
            const float inv = L > 0.f ? vg / L : 0.f;
#pragma unroll
            for (int ch = 0; ch < (DUAL ? D / 32 : D / 64); ++ch) {
                const int col = (DUAL ? 0 : s * (D / 2)) + 32 * ch;
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
                    float* at = part + (size_t)tr * D + col;
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
                    a.lse[orow] = L > 0.f ? 0.693147180559945f * (M + log2f(L)) : -INFINITY;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(bar(sm.o_empty));
            x += tiles;
            if (cu.u + tiles < cu.nu) cu.u += tiles;
            else cu.next_item(c, p, g);
        }
    } else if (w < (TC_SOFT + TC_FILL) / 32) {
        // ------------------------------------------------ filling ------------------------------------------------
        const int r = tid - TC_SOFT;                                // token of a tile, row of a query tile
        const int page_mask = (1 << c.page_shift) - 1, tiles_per_page = 1 << (c.page_shift - 4);
        Cursor ahead = cu;
        long long looked = x0;
        bool real = false;
        const char* src = nullptr;                                  // the thread's token under `ahead`
        auto look = [&]() {
            real = false;
            if (looked >= x1) return;
            const int pos = ahead.lo + ahead.u * TC_KV + r;
            if (pos < ahead.hi) {
                const int l0 = ahead.row_of_table(p);
                int page = c.table[(size_t)l0 * c.max_pages + (pos >> c.page_shift)];
                if (page < 0 || page >= c.n_pages) {
                    for (int j = 0; j < p.group; ++j) flag_lane(c.lane_status, l0 + j, AS_ERR_INVALID_ARG);
                    page = 0;
                }
                src = c.pages + (((size_t)page * c.heads + ahead.head) * tiles_per_page + ((pos & page_mask) >> 4)) * Ti::BYTES;
                real = true;
            }
            ++looked;
            ahead.step(c, p, g);
        };
        uint32_t kc[CHUNKS], vc[CHUNKS], ksc[CHUNKS / 8 + (CHUNKS % 8 != 0)], vsc[KSTEPS];
        const int t = r & 15;
        auto load_k = [&]() {
#pragma unroll
            for (int i = 0; i < CHUNKS; i += 4) {
                const uint4 q = real ? *reinterpret_cast<const uint4*>(src + Ti::k_code(t, 0) + 4 * i) : make_uint4(0, 0, 0, 0);
                kc[i] = q.x; kc[i + 1] = q.y; kc[i + 2] = q.z; kc[i + 3] = q.w;
            }
#pragma unroll
            for (int i = 0; i < KSTEPS / 4; ++i) ksc[i] = real ? *reinterpret_cast<const uint32_t*>(src + Ti::k_scale(t, 4 * i)) : 0u;
        };
        auto load_v = [&]() {
#pragma unroll
            for (int b = 0; b < KSTEPS; ++b) {
                const uint2 q = real ? *reinterpret_cast<const uint2*>(src + Ti::v_code(t, b)) : make_uint2(0, 0);
                vc[2 * b] = q.x; vc[2 * b + 1] = q.y;
                vsc[b] = real ? (uint32_t)(uint8_t)src[Ti::v_scale(t, b)] : 0u;
            }
        };
        // 8 codes x scale -> 16 bytes of f16
        auto widen = [](uint32_t codes, uint32_t scale2) {
            return make_uint4(mul_f16(codes_f16x2(codes), scale2), mul_f16(codes_f16x2(codes >> 8), scale2), mul_f16(codes_f16x2(codes >> 16), scale2),
                              mul_f16(codes_f16x2(codes >> 24), scale2));
        };
        auto put = [](uint32_t at, const uint4& v) { asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); };
        auto filled = [&](uint32_t b) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc_bar_arrive(b);
        };
        look();
        load_k();
        load_v();
        uint32_t n = 0;                                             // tiles filled
        for (int item = 0; x < x1 && ok; ++item) {
            const int tiles = (int)min((long long)(cu.nu - cu.u), x1 - x);
            // ---- the item's queries, scaled by a power of two into f16's range; a negative scale goes in here ----
            if (item > 0) ok = wait_warp(sm.q_empty, (item - 1) & 1);
            if (!ok) break;
#pragma unroll
            for (int h = 0; h < (DUAL ? 2 : 1); ++h) {
                const int row = (cu.entry % p.row_tiles) * p.tile_rows + 128 * h + r;
                uint4 q[CHUNKS];
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) q[i] = make_uint4(0, 0, 0, 0);
                if (row < p.rows) {
                    const int ln = cu.row_of_table(p) + row / (c.T * g), tt = row / g % c.T;
                    const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(a.q) + ((long long)ln * c.T + tt) * a.q_ld + (cu.head * g + row % g) * D;
                    if ((reinterpret_cast<uintptr_t>(from) & 15) == 0) {
#pragma unroll
                        for (int i = 0; i < CHUNKS; ++i) q[i] = reinterpret_cast<const uint4*>(from)[i];
                    } else {
                        const uint16_t* e = reinterpret_cast<const uint16_t*>(from);
#pragma unroll
                        for (int i = 0; i < CHUNKS; ++i)
                            q[i] = make_uint4(e[8 * i] | (uint32_t)e[8 * i + 1] << 16, e[8 * i + 2] | (uint32_t)e[8 * i + 3] << 16,
                                              e[8 * i + 4] | (uint32_t)e[8 * i + 5] << 16, e[8 * i + 6] | (uint32_t)e[8 * i + 7] << 16);
                    }
                }
                uint32_t top = 0;                                   // largest magnitude's bits
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) {
                    const uint32_t z[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = max(top, max(z[e] & 0x7FFFu, z[e] >> 16 & 0x7FFFu));
                }
                int ex = (int)(top >> 7) - 127;
                ex = ex > 126 ? 126 : ex < -126 ? -126 : ex;
                const float down = __uint_as_float((uint32_t)(127 - ex) << 23 | (a.scale < 0.f ? 0x80000000u : 0u));
                sm.up[item & 1][128 * h + r] = __uint_as_float((uint32_t)(127 + ex) << 23);
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) {
                    const uint32_t z[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
                    uint32_t f[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = pack_f16(__uint_as_float(z[e] << 16) * down, __uint_as_float(z[e] & 0xFFFF0000u) * down);
                    put(q_s + h * MAT + (i / 8) * BLK + tc_at(r, i % 8), make_uint4(f[0], f[1], f[2], f[3]));
                }
            }
            filled(bar(sm.q_full));
            // ---- its keys and values ----
            for (int j = 0; j < tiles && ok; ++j, ++n) {
                const int b = n & 1;
                const uint32_t turn = (n >> 1) & 1;
                if (n >= 2) ok = wait_warp(sm.k_empty[b], turn ^ 1);
                if (!ok) break;
                uint32_t sc[KSTEPS];
#pragma unroll
                for (int i = 0; i < KSTEPS; i += 2) {
                    const uint32_t two = e4m3_f16x2(ksc[i / 4] >> (8 * (i & 2)) & 0xFFFFu);
                    sc[i] = __byte_perm(two, two, 0x1010);
                    sc[i + 1] = __byte_perm(two, two, 0x3232);
                }
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) put(k_s + b * MAT + (i / 8) * BLK + tc_at(r, i % 8), widen(kc[i], sc[i / 2]));
                filled(bar(sm.k_full[b]));
                if (n >= 2) ok = wait_warp(sm.v_empty[b], turn ^ 1);
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < KSTEPS; ++i) {
                    const uint32_t one = e4m3_f16x2(vsc[i]);
                    sc[i] = __byte_perm(one, one, 0x1010);
                }
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) put(v_s + b * MAT + (i / 8) * BLK + tc_at(r, i % 8), widen(vc[i], sc[i / 2]));
                filled(bar(sm.v_full[b]));
                look();
                load_k();
                load_v();
            }
            x += tiles;
            if (cu.u + tiles < cu.nu) cu.u += tiles;
            else cu.next_item(c, p, g);
        }
    } else if (lane == 0) {
        // ------------------------------------------------ issuing ------------------------------------------------
        constexpr uint32_t ID_S = tc_idesc(128, TC_KV, false), ID_O = tc_idesc(128, D, true);
        uint32_t n0 = 0, p_seen[2] = {0, 0};                        // tiles before this item; weights taken, by group
        for (int item = 0; x < x1 && ok; ++item) {
            const int tiles = (int)min((long long)(cu.nu - cu.u), x1 - x), steps = DUAL ? 2 * tiles : tiles;
            ok = tc_wait(bar(sm.q_full), item & 1, limit, failed);
            if (!ok) break;
            for (int i = 0; i <= steps && ok; ++i) {
                if (i < steps) {
                    const int j = DUAL ? i >> 1 : i, s = i & 1;
                    const uint32_t n = n0 + j, b = n & 1;
                    if (!DUAL || s == 0) ok = tc_wait(bar(sm.k_full[b]), (n >> 1) & 1, limit, failed);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < KSTEPS; ++k) {
                        const uint32_t at = (k / 4) * BLK + (k % 4) * 32;
                        tc_mma_ss(s_t + 128 * s, tc_desc(q_s + (DUAL ? s * MAT : 0) + at, 0), tc_desc(k_s + b * MAT + at, 0), ID_S, k > 0);
                    }
                    tc_commit(bar(sm.s_full[s]));
                    if (!DUAL || s == 1) tc_commit(bar(sm.k_empty[b]));
                    if (i + 1 == steps) tc_commit(bar(sm.q_empty));
                }
                if (i > 0) {
                    const int i2 = i - 1, j = DUAL ? i2 >> 1 : i2, s = i2 & 1;
                    const uint32_t n = n0 + j, b = n & 1;
                    if (i2 == 0 && item > 0) ok = tc_wait(bar(sm.o_empty), (item - 1) & 1, limit, failed);
                    if (ok && (!DUAL || s == 0)) ok = tc_wait(bar(sm.v_full[b]), (n >> 1) & 1, limit, failed);
                    if (ok) ok = tc_wait(bar(sm.p_full[s]), p_seen[s] & 1, limit, failed);
                    if (!ok) break;
                    ++p_seen[s];
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < TC_KV / 16; ++k)
                        tc_mma_ts(o_t + 128 * s, s_t + 128 * s + 8 * k, tc_desc(v_s + b * MAT + k * 2048, BLK), ID_O, k > 0 || (DUAL ? j > 0 : j > 1));
                    if (!DUAL || s == 1) tc_commit(bar(sm.v_empty[b]));
                }
            }
            if (!ok) break;
            tc_commit(bar(sm.o_full));
            n0 += tiles;
            x += tiles;
            if (cu.u + tiles < cu.nu) cu.u += tiles;
            else cu.next_item(c, p, g);
        }
        // whatever is still in flight ends before TMEM is freed
        tc_commit(bar(sm.fin));
        for (long long start = clock64(); clock64() - start < limit;) {
            uint32_t done;
            asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar(sm.fin)) : "memory");
            if (done) break;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (sm.failed && tid == 0) {
        for (int j = 0; j < c.lanes; ++j) flag_lane(c.lane_status, j, AS_ERR_TIMEOUT);
    }
    if (w == TC_NT / 32 - 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

}  // namespace asx
