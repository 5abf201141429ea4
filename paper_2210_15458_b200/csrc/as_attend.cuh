// Attention over the 4-bit cache.
//
// For a query row: o = sum_t softmax_t(scale q.k_t) v_t, taken tile by tile (16 tokens) with a running
// maximum m and sum l:  o <- o 2^(m-m') + sum_t 2^(s_t-m') v_t, l likewise, scores s in units of log 2.
// Two such states over different tokens join into one the same way, so the tokens of a row may be
// split over warps, CTAs and passes.
#pragma once
#include "as_cache4.cuh"

namespace asx {

constexpr int AT_W = 4;                     // warps of a CTA; a unit of work is 2 tiles of 16 tokens for each
constexpr int AT_NT = 32 * AT_W;
constexpr int AT_STAGES = 2;                // pairs of tiles that a warp has in flight or in use
constexpr int AT_MAX_RUNS = 2560;           // CTAs, or warps where each has a run of its own
// Weights are 2^(s - m).  They become f16 for the products with the values, off by up to 2^-25 however small they are, while
// their place in the sum is exact: so they are formed large, the largest of a row at least 2^AT_TOP, and never above 2^15 (f16 ends at
// 2^16).  What a token loses is then at most 2^(-25 - AT_TOP) of the largest weight.  m is set anew when a score passes it by
// 15 - AT_TOP; that lag saves scalings of the sums: a lag of 8 / 4 / 0 takes 462 / 500 / 733 us for a chunk of 2 x 2048 tokens, 87 /
// 92 / 110 us behind shared beginnings; in 32 bits one of 8 / 3 / 0 takes 313 / 313 / 319 us for 2 x 300 tokens over 4096.
// Eleven bits are enough for bf16 outputs: the 64-bit result is missed by 1.67e-3 instead of 1.66e-3, nearly all of it the output's
// own 8 bits.  In 32 bits a weight goes in as two f16.
// bf16: m itself stands AT_TOP below the largest score.  32 bits: s - m would lose digits there (12 x 30001 tokens: 3.8e-7 in place
// of 3.1e-7 off the 64-bit result), so the weights are multiplied after the exponential and the outputs by the inverse.
template <int DT> constexpr float AT_TOP = DT == AS_F32 ? 12.f : 7.f;
template <int DT> constexpr float AT_BELOW = DT == AS_F32 ? 0.f : AT_TOP<DT>;                   // m below the largest score
template <int DT> constexpr float AT_RISE = 15.f - AT_TOP<DT> + AT_BELOW<DT>;                   // a score this far above m sets it anew
template <int DT> constexpr float AT_UP = DT == AS_F32 ? 4096.f : 1.f;                          // on weights
template <int DT> constexpr float AT_DOWN = 1.f / AT_UP<DT>;                                    // on outputs

struct AttendArgs {
    CacheArgs c;
    const void* q;
    long long q_ld;
    int q_heads;
    float scale;
    void* out;
    float* lse;
    Divisor by_g, by_Tg;                    // query heads of a key head, rows of a lane
};

// One pass over the cache.  An item is a set of query rows that read the same tokens of one head: the
// rows of `group` lanes (1, or all N lanes of a group for their shared beginning) x T tokens x the
// query heads of a key head, cut into row tiles of tile_rows.  Items are ordered by entry (lane or
// group, row tile), then head; their units (2^unit_shift tokens each) are dealt out in equal
// contiguous runs, one for each CTA (or warp).  (The host holds the number of units below 2^31, at either size.)
struct PassArgs {
    int n;                                  // lanes, or groups
    int group;                              // lanes of an item
    bool prefix;                            // tokens [0, begin[b]) of group b, else [begin[b / N], len) of lane b
    int N;
    const int* begin;                       // [lanes / N] usable shared lengths, or null (0)
    int rows, tile_rows, row_tiles, unit_shift;
    Divisor by_row_tiles, by_tile_rows, by_N;
    int *first_run, *last_run;              // [items] the runs that have an item's first and last units, written by them
    float* part_item;                       // states of items that one run saw whole; null: it writes the output itself
    float* part_run;                        // [2 * runs] states of the others: a run's first and last item
    int runs;
    long long wait_cycles;
};

__device__ __forceinline__ int lane_len(const CacheArgs& c, int lane, bool* bad = nullptr) {
    const int len = c.len[ASX_AT(lane, c.lanes, 121)];
    const bool b = len < 0 || len > ((long long)c.max_pages << c.page_shift);
    if (bad) *bad = b;
    return b ? 0 : len;
}
// the tokens [lo, hi) that the rows of an entry read; behind a tile's last row nothing is seen
__device__ __forceinline__ void token_range(const AttendArgs& a, const PassArgs& p, int entry, int b, int& lo, int& hi) {
    const int s = p.begin ? p.begin[ASX_AT(p.prefix ? b : p.by_N.div(b), a.c.lanes / p.N, 122)] : 0;
    lo = p.prefix ? 0 : s;
    hi = p.prefix ? s : lane_len(a.c, b);
    if (!p.prefix && a.c.T > 1) {
        const int last = min(p.rows, (entry - b * p.row_tiles + 1) * p.tile_rows) - 1;
        hi = max(lo, hi - a.c.T + 1 + a.by_g.div(last));
    }
}
__device__ __forceinline__ int units_of(const PassArgs& p, int lo, int hi) { return (hi - lo + (1 << p.unit_shift) - 1) >> p.unit_shift; }
// Positions that a row may see, and where its output goes.
__device__ __forceinline__ int row_limit(const AttendArgs& a, int lane0, int row) {
    const int ln = a.by_Tg.div(row), t = a.by_g.div(row) - ln * a.c.T;
    return lane_len(a.c, lane0 + ln) - a.c.T + 1 + t;
}
__device__ __forceinline__ size_t out_row(const AttendArgs& a, int lane0, int head, int row) {
    const int tok = a.by_g.div(row), g = (int)a.by_g.d;
    return ASX_AT(((size_t)lane0 * a.c.T + tok) * a.q_heads + head * g + row - tok * g, (long long)a.c.lanes * a.c.T * a.q_heads, 123);
}

// The first entry from `entry` on that has tokens: (entry, lo, hi, lane or group).  A call: it is rare, and inlined it
// would swell every loop that moves on through the units beyond the instruction caches.
__device__ __noinline__ int4 find_entry(const AttendArgs& a, const PassArgs& p, int entry) {
    int b = 0, lo = 0, hi = 0;
#pragma unroll 1
    for (; entry < p.n * p.row_tiles; ++entry) {
        b = p.by_row_tiles.div(entry);
        token_range(a, p, entry, b, lo, hi);
        if (hi > lo) break;
    }
    return make_int4(entry, lo, hi, b);
}

// Where a CTA stands in its run of units.
struct Cursor {
    int entry, head, u, nu, lo, hi, lane0, row0;    // row0: the tile's first row
    __device__ __forceinline__ void enter(const AttendArgs& a, const PassArgs& p) {
        const int4 e = find_entry(a, p, entry);
        entry = e.x; lo = e.y; hi = e.z;
        nu = units_of(p, lo, hi);
        lane0 = p.prefix ? e.w * p.N : e.w;
        row0 = (entry - e.w * p.row_tiles) * p.tile_rows;
    }
    __device__ __forceinline__ void next_item(const AttendArgs& a, const PassArgs& p) {
        u = 0;
        if (++head < a.c.heads) return;
        head = 0;
        ++entry;
        enter(a, p);
    }
    __device__ __forceinline__ void step(const AttendArgs& a, const PassArgs& p) {
        if (++u == nu) next_item(a, p);
    }
};

// The run of the thread's CTA (WORKERS = 1) or warp (one of WORKERS): how many units it has, and where it starts; called
// by all NT threads.  0: it has none.
struct RunSmem {
    int warp_sum[32];
    int start[4][3];
};
__device__ __noinline__ int entry_units(const AttendArgs& a, const PassArgs& p, int entry) {
    int lo, hi;
    token_range(a, p, entry, p.by_row_tiles.div(entry), lo, hi);
    return units_of(p, lo, hi);
}
template <int NT, int WORKERS = 1>
__device__ __forceinline__ int find_run(const AttendArgs& a, const PassArgs& p, RunSmem& sm, Cursor& cu) {
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, n = p.n * p.row_tiles;
    const int per = (n + NT - 1) / NT, j0 = min(tid * per, n), j1 = min(j0 + per, n);
    int mine = 0;
#pragma unroll 1
    for (int j = j0; j < j1; ++j) mine += entry_units(a, p, j);
    int incl = mine;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) sm.warp_sum[w] = incl;
    __syncthreads();
    int before = incl - mine, total = 0;
#pragma unroll 1
    for (int i = 0; i < NT / 32; ++i) {
        const int v = sm.warp_sum[i];
        before += i < w ? v : 0;
        total += v;
    }
    // U = q G + r units in G equal shares, none of them empty
    const unsigned U = (unsigned)total * a.c.heads, G = min((unsigned)p.runs, U);
    const unsigned first = blockIdx.x * WORKERS;
    if (first >= G) return 0;
    const unsigned q = U / G, r = U - q * G;
    auto start = [&](unsigned k) { return q * k + r * k / G; };
    unsigned at = (unsigned)before * a.c.heads;
    const unsigned end = at + (unsigned)mine * a.c.heads;
    if (start(first) < end && start(min(first + WORKERS, G)) > at) {
#pragma unroll 1
        for (int j = j0; j < j1; ++j) {
            const unsigned nu = entry_units(a, p, j), all = nu * a.c.heads;
#pragma unroll 1
            for (int k = 0; k < WORKERS; ++k) {
                const unsigned x = start(first + k) - at;
                if (first + k < G && start(first + k) >= at && x < all) {
                    (void)ASX_AT(k, 4, 124);
                    sm.start[k][0] = j;
                    sm.start[k][1] = (int)(x / nu);
                    sm.start[k][2] = (int)(x % nu);
                }
            }
            at += all;
        }
    }
    __syncthreads();
    const unsigned k = WORKERS == 1 ? 0 : w;
    if (first + k >= G) return 0;
    cu.entry = sm.start[k][0]; cu.head = sm.start[k][1]; cu.u = sm.start[k][2];
    cu.enter(a, p);
    return (int)(start(first + k + 1) - start(first + k));
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
__device__ __forceinline__ uint32_t mul_f16(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t e4m3_f16x2(uint32_t two) {
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((unsigned short)two));
    return d;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <class V> __device__ __forceinline__ V lds(uint32_t at);
template <> __device__ __forceinline__ uint4 lds<uint4>(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
template <> __device__ __forceinline__ uint2 lds<uint2>(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
template <> __device__ __forceinline__ uint32_t lds<uint32_t>(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
template <> __device__ __forceinline__ unsigned short lds<unsigned short>(uint32_t at) {
    unsigned short v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
    return v;
}
template <> __device__ __forceinline__ unsigned char lds<unsigned char>(uint32_t at) {
    unsigned short v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=h"(v) : "r"(at));
    return (unsigned char)v;
}

// row = (lane of the group x T + token) x g + query head
template <int DT, int D>
__device__ __forceinline__ const typename Io<DT>::type* query_row(const AttendArgs& a, int lane0, int head, int row) {
    const int tok = a.by_g.div(row), g = (int)a.by_g.d;
    return static_cast<const typename Io<DT>::type*>(a.q) + ASX_AT((long long)lane0 * a.c.T + tok, (long long)a.c.lanes * a.c.T, 125) * a.q_ld + ASX_AT(head * g + row - tok * g, a.q_heads, 126) * D;
}

template <int D> struct AttendSmem {
    char ring[AT_W][AT_STAGES][2 * Tile4<D>::BYTES];
    float join[AT_W][8][D + 20];            // the warps' sums (the pitch spreads rows over the banks)
    float join_m[AT_W][8], join_l[AT_W][8];
    RunSmem run;
};

// A state as it is kept in scratch: rows x D sums, then m and l of each row.
// l = 0: the row saw nothing (zeros, lse -inf).  A NaN in the row's query or scores, or a score of +inf, makes l NaN whatever m
// is, and 1 / l carries it into the output and lse.
template <int D> __host__ __device__ __forceinline__ constexpr int state_floats(int rows) { return rows * (D + 2); }

// Each warp takes every fourth pair of tiles of the CTA's run; SOLO: every pair of a run of its own, so that nothing is
// joined within the CTA (for many items of few tokens).  Scores are formed transposed, S^T = K q^T (tokens
// x rows, so that 16 x 16 keys go through one instruction whatever the number of rows up to 8), and
// so is the output, O^T = V^T P^T.  Keys and values become f16 in registers: code x scale is exact
// there; queries are scaled by a power of two to lie in f16's range (bf16: exact down to 2^-17 of the row's largest, below that
// within 2^-25 of it) or split in two f16 (32 bits).  Which dimension of a tile goes to which index of the products is free, and chosen so that a
// thread's keys are 16 neighbouring bytes and its values the 16 dimensions of one block, which share
// their scale.  The tensor cores cut sums off instead of rounding them: with 32-bit queries (one row tile) chains of products
// are kept to two and joined by additions (12 x 30001 tokens: 3.0e-6 off otherwise, from the bias alone; a bf16 output is rounded by a
// thousand times that, and its chains stay long).  Token l of the
// products is token 4 (l / 2 mod 4) + (l mod 2) + 2 (l / 8) of the tile.
// Bound by issue slots: 364 instructions for a tile of 16 tokens at head dimension 128, conversions and products mostly
// (60 % of the slots, ALU pipe 54 %, DRAM 52 %: no unit is full, 3.5 warps a scheduler do not hide every wait).  128 lanes of up to 8192 tokens, 32 heads on 8: 178 to 194 us (4.2 to 4.6 TB/s); in 32
// bits, 12 lanes of up to 30001: 95 us (3.1 TB/s).
template <int DT, int D, int NT, bool SOLO>
__global__ void __launch_bounds__(AT_NT) attend_mma_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ PassArgs p) {
    using Ti = Tile4<D>;
    constexpr bool F32 = DT == AS_F32;
    constexpr int PARTS = F32 ? 2 : 1;
    constexpr int KS = D / 16;                      // steps of 16 dimensions
    extern __shared__ __align__(16) char at_smem[];
    AttendSmem<D>& sm = *reinterpret_cast<AttendSmem<D>*>(at_smem);
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, r = lane >> 2, cc = lane & 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    Cursor cu, ahead;
    int left = find_run<AT_NT, SOLO ? AT_W : 1>(a, p, sm.run, cu), to_issue = left;
    if (left == 0) return;
    ahead = cu;

    // ---- copies: half a warp brings in one of its two tiles; the page id is fetched a unit before ----
    const int half = lane >> 4, hl = lane & 15;
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(&sm.ring[w][0][0]);
    const int page_mask = (1 << c.page_shift) - 1, tiles_per_page = 1 << (c.page_shift - 4);
    int page = 0;
    auto look = [&]() {                             // page id of the half-warp's tile under `ahead`
        const int pos = ahead.lo + ((SOLO ? ahead.u : ahead.u * AT_W + w) * 2 + half) * 16;
        if (pos < ahead.hi) page = c.table[(size_t)ASX_AT(ahead.lane0, c.lanes, 127) * c.max_pages + ASX_AT(pos >> c.page_shift, c.max_pages, 128)];
    };
    auto issue = [&](int stage) {
        const int pos = ahead.lo + ((SOLO ? ahead.u : ahead.u * AT_W + w) * 2 + half) * 16;
        if (pos < ahead.hi) {
            if (page < 0 || page >= c.n_pages) {
                if (hl == 0) {
#pragma unroll 1
                    for (int j = 0; j < p.group; ++j) flag_lane(c.lane_status, ahead.lane0 + j, AS_ERR_INVALID_ARG);
                }
                page = 0;
            }
            const char* src = c.pages + (((size_t)page * c.heads + ASX_AT(ahead.head, c.heads, 129)) * tiles_per_page + ((pos & page_mask) >> 4)) * Ti::BYTES + hl * 16;
            const uint32_t dst = ring0 + ASX_AT((stage * 2 + half) * Ti::BYTES, (2 * AT_STAGES - 1) * Ti::BYTES + 1, 130) + hl * 16;
#pragma unroll
            for (int i = 0; i < (Ti::BYTES / 16 + 15) / 16; ++i)
                if (i * 16 + 16 <= Ti::BYTES / 16 || i * 16 + hl < Ti::BYTES / 16)
                    cp_async16(dst + ASX_AT(i * 256 + hl * 16, Ti::BYTES - 15, 131) - hl * 16, src + i * 256);
        }
        if (--to_issue > 0) {
            ahead.step(a, p);
            look();
            if (ahead.u == 0) {                     // the next item's queries: into L1 meanwhile
                const int row = ahead.row0 + r;
                if (row < p.rows) asm volatile("prefetch.global.L1 [%0];" ::"l"(query_row<DT, D>(a, ahead.lane0, ahead.head, row) + cc * (D / 4)));
            }
        }
    };
    look();
    issue(0);
    cp_commit();

    using E = typename Io<DT>::type;
    uint32_t qf[PARTS][NT][KS][2];
    float o[NT][KS][4], m[NT][2], mu[NT][2], l[NT][2], k2[NT][2];
    int lim[NT][2], lim_min = 0;
    int seg_u0 = 0, stage = 0;
    bool fresh = true;
#pragma unroll 1
    for (; left > 0; --left) {
        if (fresh) {                                // ---- a new item: its query rows ----
            fresh = false;
            seg_u0 = cu.u;
            const int head = cu.head, row0 = cu.row0, lane0 = cu.lane0;
            const float kg = c.k_scale ? c.k_scale[head] : 1.f;
            const float to_log2 = a.scale * kg * 1.44269504088896f;
            lim_min = 0x7FFFFFFF;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int row = row0 + n * 8 + r;
                float top = 0.f, xq[D / 4];
#pragma unroll
                for (int e = 0; e < D / 4; ++e) xq[e] = 0.f;
                if (row < p.rows) {
                    const E* src = query_row<DT, D>(a, lane0, head, row) + cc * (D / 4);
                    const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
#pragma unroll
                    for (int e = 0; e < D / 4; e += 16) Io<DT>::read16(src + e, vec, *reinterpret_cast<float(*)[16]>(&xq[e]));
                }
#pragma unroll
                for (int e = 0; e < D / 4; ++e) top = fmaxf(top, fabsf(xq[e]));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                // the row's largest magnitude is brought into [1, 2)
                int ex = (int)(__float_as_uint(top) >> 23) - 127;
                ex = ex > 126 ? 126 : ex < -126 ? -126 : ex;
                const float down = __uint_as_float((uint32_t)(127 - ex) << 23), up = __uint_as_float((uint32_t)(127 + ex) << 23);
#pragma unroll
                for (int j = 0; j < KS; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float f0 = xq[4 * j + 2 * h] * down, f1 = xq[4 * j + 2 * h + 1] * down;
                        qf[0][n][j][h] = pack_f16(f0, f1);
                        if (F32) {
                            const float2 hi = unpack_f16(qf[0][n][j][h]);
                            qf[PARTS - 1][n][j][h] = pack_f16(f0 - hi.x, f1 - hi.y);
                        }
                    }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int rw = row0 + n * 8 + 2 * cc + h;
                    k2[n][h] = __shfl_sync(0xFFFFFFFFu, up, 4 * (2 * cc + h)) * to_log2;
                    lim[n][h] = rw < p.rows ? min(row_limit(a, lane0, rw), cu.hi) : 0;
                    if (rw < p.rows) lim_min = min(lim_min, lim[n][h]);
                    m[n][h] = -INFINITY; mu[n][h] = 0.f; l[n][h] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
            }
            lim_min = __reduce_min_sync(0xFFFFFFFFu, lim_min);
        }
        cp_wait<0>();
        __syncwarp();
        if (to_issue > 0) issue(stage ^ 1);
        cp_commit();
        const int pos = cu.lo + (SOLO ? cu.u : cu.u * AT_W + w) * 32;
        if (pos < cu.hi) {
            const uint32_t st = ring0 + ASX_AT(stage, AT_STAGES, 132) * 2 * Ti::BYTES;
            const bool two = pos + 16 < cu.hi;              // (the second tile may lie behind the last token: nothing was copied)
            // ---- S^T = K q^T ----
            const int t0 = 4 * (r >> 1) + (r & 1);      // the thread's tokens of a tile: t0 and t0 + 2
            float s[2][NT][4];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t sb = st + b * Ti::BYTES;
                uint32_t kw[2][D / 32], ks[2][D / 64];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int t = t0 + 2 * i;
                    if (D == 128) {
                        const uint4 v = lds<uint4>(sb + Ti::K + ASX_AT(t * (D / 2) + cc * 16, 8 * D - 15, 133));
                        kw[i][0] = v.x; kw[i][1] = v.y; kw[i][D / 32 - 2] = v.z; kw[i][D / 32 - 1] = v.w;
                        const uint32_t s2 = e4m3_f16x2(lds<unsigned short>(sb + Ti::KS + ASX_AT(t * Ti::NB + 2 * cc, D - 1, 134)));
                        ks[i][0] = __byte_perm(s2, s2, 0x1010);
                        ks[i][D / 64 - 1] = __byte_perm(s2, s2, 0x3232);
                    } else {
                        const uint2 v = lds<uint2>(sb + Ti::K + ASX_AT(t * (D / 2) + cc * 8, 8 * D - 7, 135));
                        kw[i][0] = v.x; kw[i][1] = v.y;
                        const uint32_t s2 = e4m3_f16x2(lds<unsigned char>(sb + Ti::KS + ASX_AT(t * Ti::NB + cc, D, 136)));
                        ks[i][0] = __byte_perm(s2, s2, 0x1010);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][n][e] = 0.f;
                float rest[4] = {0.f, 0.f, 0.f, 0.f};       // (32-bit queries: the sum over their second halves)
#pragma unroll
                for (int j = 0; j < KS; j += 2) {           // a word of each token is two steps of 16 dimensions
                    float part[4] = {0.f, 0.f, 0.f, 0.f};   // (32-bit queries: two steps' sum)
                    uint32_t f[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) codes_f16x2(kw[i][j / 2], f[i]);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) f[i][e] = mul_f16(f[i][e], ks[i][j / 4]);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma_f16(F32 ? part : s[b][n], f[0][2 * h], f[1][2 * h], f[0][2 * h + 1], f[1][2 * h + 1], qf[0][n][j + h][0], qf[0][n][j + h][1]);
                            if (F32) mma_f16(rest, f[0][2 * h], f[1][2 * h], f[0][2 * h + 1], f[1][2 * h + 1], qf[PARTS - 1][n][j + h][0], qf[PARTS - 1][n][j + h][1]);
                        }
                    if (F32) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][0][e] += part[e];
                    }
                }
                if (F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][0][e] += rest[e];
                }
            }
            // ---- weights ----
            bool rise = false;
            const bool cut = pos + 32 > lim_min;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {           // tokens t0, t0 + 2 of the first tile, then of the second
                        float& x = s[e >> 1][n][2 * (e & 1) + h];
                        x *= k2[n][h];
                        if (cut && pos + 16 * (e >> 1) + t0 + 2 * (e & 1) >= lim[n][h]) x = -INFINITY;
                        top = fmaxf(top, x);
                    }
                    rise |= top > m[n][h] + AT_RISE<DT>;
                }
            if (__any_sync(0xFFFFFFFFu, rise)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float top = fmaxf(fmaxf(s[0][n][h], s[0][n][2 + h]), fmaxf(s[1][n][h], s[1][n][2 + h]));
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                        top = fmaxf(top - AT_BELOW<DT>, m[n][h]);
                        const float f = top == -INFINITY ? 1.f : ex2(m[n][h] - top);
                        m[n][h] = top;
                        mu[n][h] = top == -INFINITY ? 0.f : top;
                        l[n][h] *= f;
#pragma unroll
                        for (int i = 0; i < KS; ++i) { o[n][i][h] *= f; o[n][i][2 + h] *= f; }
                    }
            }
            uint32_t pf[2][PARTS][NT][2];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float pr[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) pr[e] = ex2(s[b][n][e] - mu[n][e & 1]);
                    l[n][0] += pr[0] + pr[2];
                    l[n][1] += pr[1] + pr[3];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float w0 = pr[2 * i] * AT_UP<DT>, w1 = pr[2 * i + 1] * AT_UP<DT>;
                        const uint32_t hi = pack_f16(w0, w1);
                        pf[b][0][n][i] = transpose8x8(hi);
                        if (F32) {
                            const float2 h2 = unpack_f16(hi);
                            pf[b][PARTS - 1][n][i] = transpose8x8(pack_f16(w0 - h2.x, w1 - h2.y));
                        }
                    }
                }
            // ---- O^T += V^T P^T ----
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (b == 1 && !two) break;
                const uint32_t sb = st + b * Ti::BYTES;
                uint32_t vw[4][D / 64];             // tokens 4 cc .. 4 cc + 3, the thread's D / 8 dimensions
                const uint32_t vb = sb + Ti::V + ASX_AT((D == 128 ? r : r >> 1) * 128 + cc * 32, 8 * D - 31, 137);
                const bool odd = r & 1;
                {
                    // (odd r reads its two halves in the other order: no two threads of a phase meet in a bank)
                    const bool swap = D == 128 && odd;
                    const uint4 x0v = lds<uint4>(vb + (swap ? 16 : 0)), x1v = lds<uint4>(vb + (swap ? 0 : 16));
                    const uint4 v0 = swap ? x1v : x0v, v1 = swap ? x0v : x1v;
                    if (D == 128) {
                        vw[0][0] = v0.x; vw[0][D / 64 - 1] = v0.y; vw[1][0] = v0.z; vw[1][D / 64 - 1] = v0.w;
                        vw[2][0] = v1.x; vw[2][D / 64 - 1] = v1.y; vw[3][0] = v1.z; vw[3][D / 64 - 1] = v1.w;
                    } else {
                        vw[0][0] = odd ? v0.y : v0.x; vw[1][0] = odd ? v0.w : v0.z;
                        vw[2][0] = odd ? v1.y : v1.x; vw[3][0] = odd ? v1.w : v1.z;
                    }
                }
                uint32_t vs4 = lds<uint32_t>(sb + Ti::VS + ASX_AT((D == 128 ? r : r >> 1) * 16 + cc * 4, D - 3, 138));
                if (pos + 32 > cu.hi) {             // tokens behind the last one: whatever the page holds there counts as zero
                    const int have = cu.hi - pos - 16 * b - 4 * cc;
                    vs4 &= have >= 4 ? 0xFFFFFFFFu : have <= 0 ? 0u : (1u << (8 * have)) - 1;
                }
                const uint32_t vs[2] = {e4m3_f16x2(vs4 & 0xFFFFu), e4m3_f16x2(vs4 >> 16)};
#pragma unroll
                for (int i4 = 0; i4 < D / 64; ++i4) {
                    uint32_t even[2], oddw[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t x = vw[2 * h][i4], y = vw[2 * h + 1][i4];
                        even[h] = (x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u);
                        oddw[h] = ((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u);
                    }
                    uint32_t f[4][4];
                    codes_f16x2(even[0], f[0]);
                    codes_f16x2(oddw[0], f[1]);
                    codes_f16x2(even[1], f[2]);
                    codes_f16x2(oddw[1], f[3]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t f0 = mul_f16(f[0][i], vs[0]), f1 = mul_f16(f[1][i], vs[0]), f2 = mul_f16(f[2][i], vs[1]), f3 = mul_f16(f[3][i], vs[1]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if constexpr (F32) {
                                float part[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_f16(part, f0, f1, f2, f3, pf[b][PARTS - 1][n][0], pf[b][PARTS - 1][n][1]);
                                mma_f16(part, f0, f1, f2, f3, pf[b][0][n][0], pf[b][0][n][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[n][4 * i4 + i][e] += part[e];
                            } else {
                                mma_f16(o[n][4 * i4 + i], f0, f1, f2, f3, pf[b][0][n][0], pf[b][0][n][1]);
                            }
                        }
                    }
                }
            }
        }
        __syncwarp();
        stage ^= 1;

        // ---- the end of an item, or of the run (the four warps' states become one) ----
        const bool item_ends = cu.u + 1 == cu.nu;
        if (item_ends || left == 1) {
            const int head = cu.head, mine = SOLO ? blockIdx.x * AT_W + w : blockIdx.x;
            const bool whole = item_ends && seg_u0 == 0;
            const size_t item = ASX_AT((size_t)cu.entry * c.heads + cu.head, (long long)p.n * p.row_tiles * c.heads, 139);
            if ((SOLO ? lane : tid) == 0) {
                if (seg_u0 == 0) p.first_run[item] = mine;
                if (item_ends) p.last_run[item] = mine;
            }
            float* part = nullptr;
            if (!whole) part = p.part_run + (size_t)ASX_AT(2 * mine + (seg_u0 == 0), 2 * p.runs, 140) * state_floats<D>(8 * NT);
            else if (p.part_item) part = p.part_item + item * state_floats<D>(8 * NT);
            const float vg = c.v_scale ? c.v_scale[head] : 1.f;
            if constexpr (SOLO) {
                // a thread has D / 8 neighbouring dimensions of the rows 2 cc and 2 cc + 1
                constexpr int PER = D / 8;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float L = l[n][h];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, d);
                        const int rw = n * 8 + 2 * cc + h, row = cu.row0 + rw;
                        if (part) {
                            float* at = part + ASX_AT(rw * D + r * PER, 8 * NT * D - PER + 1, 141);
#pragma unroll
                            for (int i = 0; i < KS; i += 2) *reinterpret_cast<float4*>(at + 2 * i) = make_float4(o[n][i][h], o[n][i][2 + h], o[n][i + 1][h], o[n][i + 1][2 + h]);
                            if (r == 0) { part[8 * NT * D + rw] = m[n][h]; part[8 * NT * (D + 1) + rw] = L; }
                        } else if (row < p.rows) {
                            const float inv = L == 0.f ? 0.f : vg / L * AT_DOWN<DT>;
                            const size_t orow = out_row(a, cu.lane0, head, row);
                            E* at = static_cast<E*>(a.out) + orow * D + r * PER;
                            if constexpr (F32) {
#pragma unroll
                                for (int i = 0; i < KS; i += 2)
                                    *reinterpret_cast<float4*>(at + 2 * i) = make_float4(o[n][i][h] * inv, o[n][i][2 + h] * inv, o[n][i + 1][h] * inv, o[n][i + 1][2 + h] * inv);
                            } else {
#pragma unroll
                                for (int i = 0; i < KS; i += 4) {
                                    uint32_t x[4];
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const __nv_bfloat162 b2 = __floats2bfloat162_rn(o[n][i + e][h] * inv, o[n][i + e][2 + h] * inv);
                                        x[e] = *reinterpret_cast<const uint32_t*>(&b2);
                                    }
                                    *reinterpret_cast<uint4*>(at + 2 * i) = make_uint4(x[0], x[1], x[2], x[3]);
                                }
                            }
                            if (a.lse && r == 0) a.lse[orow] = L == 0.f ? -INFINITY : 0.693147180559945f * (m[n][h] + log2f(L));
                        }
                    }
            } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float sum = l[n][h];
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
                    if (r == 0) { sm.join_m[w][2 * cc + h] = m[n][h]; sm.join_l[w][2 * cc + h] = sum; }
#pragma unroll
                    for (int i = 0; i < KS; ++i)
                        *reinterpret_cast<float2*>(&sm.join[w][2 * cc + h][ASX_AT(r * (D / 8 + 2) + 2 * i, D + 19, 142)]) = make_float2(o[n][i][h], o[n][i][2 + h]);
                }
                __syncthreads();
                constexpr int PER = D / 16;         // dimensions of a thread; 16 threads a row
                const int rw = tid >> 4, d0 = (tid & 15) * PER;
                float f[AT_W], M = -INFINITY, L = 0.f, acc[PER];
#pragma unroll
                for (int i = 0; i < AT_W; ++i) M = fmaxf(M, sm.join_m[i][rw]);
#pragma unroll
                for (int i = 0; i < AT_W; ++i) {
                    f[i] = sm.join_m[i][rw] == -INFINITY ? 0.f : ex2(sm.join_m[i][rw] - M);
                    L += f[i] * sm.join_l[i][rw];
                }
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    acc[e] = 0.f;
#pragma unroll
                    for (int i = 0; i < AT_W; ++i) acc[e] += f[i] * sm.join[i][ASX_AT(rw, 8, 143)][ASX_AT((d0 / (D / 8)) * (D / 8 + 2) + d0 % (D / 8) + e, D + 20, 144)];
                }
                const int row = cu.row0 + n * 8 + rw;
                if (part) {
                    float* at = part + ASX_AT((n * 8 + rw) * D + d0, 8 * NT * D - PER + 1, 145);
#pragma unroll
                    for (int e = 0; e < PER; e += 4) *reinterpret_cast<float4*>(at + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
                    if (d0 == 0) { part[8 * NT * D + n * 8 + rw] = M; part[8 * NT * (D + 1) + n * 8 + rw] = L; }
                } else if (row < p.rows) {
                    const float inv = L == 0.f ? 0.f : vg / L * AT_DOWN<DT>;
                    const size_t orow = out_row(a, cu.lane0, head, row);
                    E* at = static_cast<E*>(a.out) + orow * D + d0;
#pragma unroll
                    for (int e = 0; e < PER; e += 2) {
                        if constexpr (F32) *reinterpret_cast<float2*>(at + e) = make_float2(acc[e] * inv, acc[e + 1] * inv);
                        else *reinterpret_cast<__nv_bfloat162*>(at + e) = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
                    }
                    if (a.lse && d0 == 0) a.lse[orow] = L == 0.f ? -INFINITY : 0.693147180559945f * (M + log2f(L));
                }
                __syncthreads();
            }
            }
            fresh = true;
        }
        cu.step(a, p);
    }
}

// Joins the states of row rw of an item into (M, L, acc): dimensions d0 .. d0 + PER - 1.  The item was shared by runs
// c0 .. c1: the first kept its state in its second slot (that item was its last), the others in their first; one
// that a run saw whole has a state of its own.  Two states are read at a time (12 x 30001 tokens in 32 bits 98.2 -> 97.1 us).
template <int D, int PER>
__device__ __forceinline__ void join_states(const PassArgs& p, size_t item, int c0, int c1, int rw, int d0, float& M, float& L, float (&acc)[PER]) {
    if (c0 < 0 || c1 >= p.runs) return;                 // (a pass whose waits ran out may not have noted its runs)
#pragma unroll 2
    for (int k = c0; k <= c1; ++k) {
        const float* s = c0 == c1 ? p.part_item + item * state_floats<D>(p.tile_rows) : p.part_run + (size_t)ASX_AT(2 * k + (k == c0), 2 * p.runs, 146) * state_floats<D>(p.tile_rows);
        const float m2 = s[p.tile_rows * D + rw], l2 = s[p.tile_rows * (D + 1) + rw];
        float x[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) x[e] = s[ASX_AT(rw * D + d0 + e, p.tile_rows * D, 147)];
        const float top = fmaxf(M, m2);
        const float f = M == -INFINITY ? 0.f : ex2(M - top), f2 = m2 == -INFINITY ? 0.f : ex2(m2 - top);
        L = L * f + l2 * f2;
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[e] = acc[e] * f + x[e] * f2;
        M = top;
    }
}
// the same for what the pass over shared beginnings has left for a row of a lane
template <int D, int PER>
__device__ __forceinline__ void join_shared(const AttendArgs& a, const PassArgs& pre, int lane, int row, int rows, int head, int d0, float& M, float& L, float (&acc)[PER]) {
    const int gr = pre.by_N.div(lane);
    if (pre.begin[gr] == 0) return;
    const int prow = (lane - gr * pre.N) * rows + row, pt = pre.by_tile_rows.div(prow);
    const size_t item = ASX_AT(((size_t)gr * pre.row_tiles + pt) * a.c.heads + head, (long long)pre.n * pre.row_tiles * a.c.heads, 148);
    join_states<D>(pre, item, pre.first_run[item], pre.last_run[item], prow - pt * pre.tile_rows, d0, M, L, acc);
}

// One CTA per item of the lanes' own pass and 32 of its rows, a warp to a row: joins the states of rows that were split
// over CTAs or passes, in a fixed order, and writes rows that saw nothing.  Latency: 7 us for 1024 items of 4 rows.  8 or 16 rows
// a CTA cost the chunk of 2 x 2048 tokens more CTAs that leave at once than they save (465 -> 471 and 467 us).
constexpr int JOIN_ROWS = 32;
template <int DT, int D>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ PassArgs own, const __grid_constant__ PassArgs pre) {
    constexpr int PER = D / 32;
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned items = (unsigned)own.n * own.row_tiles * c.heads;       // (the host holds it below 2^31)
    const int first = blockIdx.y * JOIN_ROWS + (threadIdx.x >> 5);
#pragma unroll 1
    for (unsigned i = blockIdx.x; i < items; i += gridDim.x) {
        const int entry = c.by_heads.div(i), head = (int)i - entry * c.heads, ln = own.by_row_tiles.div(entry);
        const bool none = entry_units(a, own, entry) == 0;
        const int c0 = none ? 0 : own.first_run[i], c1 = none ? -1 : own.last_run[i];
        if (!none && c0 == c1 && !own.part_item) continue;                  // the pass has written the output itself
        const int row0 = (entry - ln * own.row_tiles) * own.tile_rows;
        const int end = min(min(own.tile_rows, own.rows - row0), (int)(blockIdx.y + 1) * JOIN_ROWS);
#pragma unroll 1
        for (int rw = first; rw < end; rw += 4) {
            const int row = row0 + rw;
            float M = -INFINITY, L = 0.f, acc[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) acc[e] = 0.f;
            if (pre.begin) join_shared<D>(a, pre, ln, row, own.rows, head, lane * PER, M, L, acc);
            join_states<D>(own, i, c0, c1, rw, lane * PER, M, L, acc);
            const float inv = L == 0.f ? 0.f : (c.v_scale ? c.v_scale[head] : 1.f) / L * AT_DOWN<DT>;
            const size_t orow = out_row(a, ln, head, row);
            typename Io<DT>::type* out = static_cast<typename Io<DT>::type*>(a.out) + orow * D + lane * PER;
#pragma unroll
            for (int e = 0; e < PER; ++e) out[e] = acc[e] * inv;
            if (a.lse && lane == 0) a.lse[orow] = L == 0.f ? -INFINITY : 0.693147180559945f * (M + log2f(L));
        }
    }
}

// One CTA per group: the shared beginning that can be used (0 where the caller's does not fit).
__global__ void __launch_bounds__(128) attend_shared_kernel(const CacheArgs c, int N, const int* shared, int* begin) {
    const int gr = blockIdx.x, s = shared[gr];
    bool ok = s > 0 && (s & ((1 << c.page_shift) - 1)) == 0;
    for (int j = threadIdx.x; j < N; j += 128) ok &= s <= lane_len(c, gr * N + j);
    ok = __syncthreads_and(ok);
    if (threadIdx.x == 0) begin[gr] = ok ? s : 0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Lanes whose length is out of range.
__global__ void __launch_bounds__(256) attend_status_kernel(const CacheArgs c) {
    for (int j = blockIdx.x * 256 + threadIdx.x; j < c.lanes; j += gridDim.x * 256) {
        bool bad;
        lane_len(c, j, &bad);
        c.lane_status[j] = bad ? AS_ERR_INVALID_ARG : AS_OK;
    }
}

}  // namespace asx
