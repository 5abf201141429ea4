// Attention weights of cached tokens, summed over the rows that look at them.
//
// For a token t of a lane and key head: w_t = sum over query rows r of 2^(s_rt - z_r), scores s and the rows' log-sums z in units of
// log 2.  The log-sums are known, so there is no running maximum.  Here, for few rows, a token's sum belongs to one warp and nothing is
// joined; the kernel for many rows adds up what groups of threads and CTAs have of it.
#pragma once
#include "as_attend.cuh"

namespace asx {

struct WeighArgs {
    AttendArgs a;                           // c.len: lengths that can be used (0 for a lane that is left alone)
    PassArgs p;                             // one entry a lane; begin[lane]: its first tile that has a token to weigh
    const float* lse;
    const int* first;                       // [lanes] first position to weigh
    float* weight;
    long long weight_ld;
    bool add;
};

// Adds what a token has got to its weight, or sets it.
__device__ __forceinline__ void put_weight(const WeighArgs& wa, int lane, int head, int pos, int from, int len, float x) {
    if (pos < from || pos >= len) return;
    float* at = wa.weight + ((size_t)ASX_AT(lane, wa.a.c.lanes, 301) * wa.a.c.heads + ASX_AT(head, wa.a.c.heads, 302)) * wa.weight_ld + ASX_AT(pos, wa.weight_ld, 303);
    *at = wa.add && pos < len - wa.a.c.T ? *at + x : x;
}

constexpr int WG_W = 4, WG_NT = 32 * WG_W;  // warps of a CTA; a unit of work is 2 tiles of 16 tokens for one of them
constexpr int WG_STAGES = 3;                // pairs of tiles (their keys) that a warp has in flight or in use

template <int D> struct WeighSmem {
    char ring[WG_W][WG_STAGES][2 * 9 * D];  // of each tile: key codes, key scales
    RunSmem run;
};

// Up to 48 rows, or 32-bit ones.  A warp has a run of its own: tokens of all lanes and heads are dealt out to the warps in equal contiguous
// runs of pairs of tiles, and as sums stay with their tokens nothing is joined.  Scores are formed as in attention, S^T = K q^T (tokens x
// rows), so that a token's sum is over neighbouring threads' columns: two shuffles; rows beyond 8 NT (MANY) are taken 8 NT at a time on the same keys.
// Bound by issue slots: about 240 instructions for a tile of 16 tokens at head dimension 128, widening the keys mostly (59 % of the slots, ALU
// pipe 40 %, DRAM 37 %, 3.8 warps a scheduler).  64 lanes of up to 8192 tokens, 32 heads on 8: 70 us (3.2 TB/s, 49 % of a copy's rate); a page's id is
// fetched a unit ahead, the old weight while the scores are formed (84 us without both).
template <int DT, int D, int NT, bool MANY>
__global__ void __launch_bounds__(WG_NT) weigh_mma_kernel(const __grid_constant__ WeighArgs wa) {
    using Ti = Tile4<D>;
    constexpr int PARTS = DT == AS_F32 ? 2 : 1;
    extern __shared__ __align__(16) char wg_smem[];
    WeighSmem<D>& sm = *reinterpret_cast<WeighSmem<D>*>(wg_smem);
    const AttendArgs& a = wa.a;
    const PassArgs& p = wa.p;
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, r = lane >> 2, cc = lane & 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Cursor<true> cu, ahead;
    int left = find_run<WG_NT, WG_W, true>(a, p, sm.run, cu), to_issue = left;
    if (left == 0) return;
    ahead = cu;

    // ---- copies: half a warp brings in the keys of one of its two tiles; the page id is fetched a unit before ----
    const int half = lane >> 4, hl = lane & 15;
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(&sm.ring[w][0][0]);
    const int page_mask = (1 << c.page_shift) - 1, tiles_per_page = 1 << (c.page_shift - 4);
    int page = 0;
    auto look = [&]() {
        const int pos = ahead.lo + (ahead.u * 2 + half) * 16;
        if (pos < ahead.hi) page = c.table[(size_t)ASX_AT(ahead.lane0, c.lanes, 304) * c.max_pages + ASX_AT(ahead.hole.real(pos) >> c.page_shift, c.max_pages, 305)];
    };
    auto issue = [&](int stage) {
        if (to_issue > 0) {
            const int pos = ahead.lo + (ahead.u * 2 + half) * 16;
            if (pos < ahead.hi) {
                if (page < 0 || page >= c.n_pages) {
                    if (hl == 0) flag_lane(c.lane_status, ahead.lane0, AS_ERR_INVALID_ARG);
                    page = 0;
                }
                const char* src = c.pages + (((size_t)page * c.heads + ASX_AT(ahead.head, c.heads, 306)) * tiles_per_page + ((ahead.hole.real(pos) & page_mask) >> 4)) * Ti::BYTES + hl * 16;
                const uint32_t dst = ring0 + ASX_AT((stage * 2 + half) * 9 * D, (2 * WG_STAGES - 1) * 9 * D + 1, 307) + hl * 16;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) cp_async16(dst + i * 256, src + Ti::K + i * 256);
                if (hl < D / 16) cp_async16(dst + 8 * D, src + Ti::KS);
            }
            if (--to_issue > 0) {
                ahead.step(a, p);
                look();
            }
        }
        cp_commit();
    };
    look();
#pragma unroll
    for (int i = 0; i < WG_STAGES - 1; ++i) issue(i);

    uint32_t qf[PARTS][NT][D / 16][2];
    float k2[NT][2], z[NT][2];
    int lim[NT][2], low[NT][2], lim_min = 0, low_max = 0;
    const int row_tiles = MANY ? (p.rows + 8 * NT - 1) / (8 * NT) : 1;
    const int t0 = 4 * (r >> 1) + (r & 1);          // the thread's tokens of a tile: t0 and t0 + 2
    const int mine = 16 * (cc >> 1) + t0 + 2 * (cc & 1);    // of the unit's tokens the one whose sum it writes
    int stage = 0, from = 0, len = 0;
    float* weight = nullptr;
    bool fresh = true;
#pragma unroll 1
    for (; left > 0; --left) {
        cp_wait<WG_STAGES - 2>();
        __syncwarp();
        issue(stage == 0 ? WG_STAGES - 1 : stage - 1);
        const int pos = cu.lo + cu.u * 32;
        if (fresh) {
            from = wa.first[cu.lane0];
            len = c.len[cu.lane0];
            weight = wa.weight + ((size_t)ASX_AT(cu.lane0, c.lanes, 301) * c.heads + ASX_AT(cu.head, c.heads, 302)) * wa.weight_ld;
        }
        // the thread's own token: its weight is on its way while the scores are formed
        const int place = pos + mine, at = cu.hole.real(place);
        const bool put = place < cu.hi && at >= from && at < len;
        float old = 0.f;
        if (put && wa.add && at < len - c.T) old = weight[ASX_AT(at, wa.weight_ld, 303)];
        float sum[4] = {0.f, 0.f, 0.f, 0.f};        // tokens t0, t0 + 2 of the first tile, then of the second
#pragma unroll 1
        for (int rt = 0; rt < row_tiles; ++rt) {
            if (fresh || MANY) {                    // ---- these rows' queries ----
                fresh = false;
                const float to_log2 = a.scale * (c.k_scale ? c.k_scale[cu.head] : 1.f) * 1.44269504088896f;
                lim_min = 0x7FFFFFFF;
                low_max = 0;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float of[2];                    // the log-sums of the thread's two columns
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int rw = (rt * NT + n) * 8 + 2 * cc + h;
                        of[h] = rw < p.rows ? wa.lse[out_row(a, cu.lane0, cu.head, rw)] : -INFINITY;
                    }
                    // (a row that sees nothing is not read: whatever it holds, its scores are 0)
                    const int row = (rt * NT + n) * 8 + r, from_lane = (lane & ~3) | (r >> 1);
                    const float even = __shfl_sync(0xFFFFFFFFu, of[0], from_lane), odd = __shfl_sync(0xFFFFFFFFu, of[1], from_lane);
                    const float up = row_queries<DT, D>((r & 1 ? odd : even) == -INFINITY ? nullptr : query_row<DT, D>(a, cu.lane0, cu.head, row) + cc * (D / 4),
                                                        [&](int part, int j, int h) -> uint32_t& { return qf[part][n][j][h]; });
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int rw = (rt * NT + n) * 8 + 2 * cc + h;
                        const float lse = of[h];
                        const int rl = lse == -INFINITY ? 0 : row_limit(a, cu.lane0, rw);
                        k2[n][h] = __shfl_sync(0xFFFFFFFFu, up, 4 * (2 * cc + h)) * to_log2;
                        z[n][h] = lse * 1.44269504088896f;
                        lim[n][h] = lse == -INFINITY ? -1 : min(rl - cu.hole.skip, cu.hi);
                        low[n][h] = max(rl - p.window, 0) - cu.hole.skip;
                        if (lse != -INFINITY) {
                            lim_min = min(lim_min, lim[n][h]);
                            low_max = max(low_max, low[n][h]);
                        } else {                    // no row, or one that sees nothing: 2^(score x 0 - inf), unless a row that sees ends the tile
                            k2[n][h] = 0.f;
                            z[n][h] = INFINITY;
                        }
                    }
                }
                lim_min = __reduce_min_sync(0xFFFFFFFFu, lim_min);
                low_max = __reduce_max_sync(0xFFFFFFFFu, low_max);
            }
            const uint32_t st = ring0 + ASX_AT(stage, WG_STAGES, 308) * 2 * 9 * D;
            const bool cut = pos + 32 > lim_min || (pos < low_max && pos + 32 > p.sinks);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float s[NT][4];
                tile_scores<DT, D, NT>(st + b * 9 * D, st + b * 9 * D + 8 * D, t0, cc, [&](int part, int n, int j, int h) { return qf[part < PARTS ? part : 0][n][j][h]; }, s);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {   // (token t0 + 2 (e / 2), row e mod 2)
                        float x = ex2(s[n][e] * k2[n][e & 1] - z[n][e & 1]);
                        if (cut) {
                            const int at = pos + 16 * b + t0 + 2 * (e >> 1);
                            x = at < lim[n][e & 1] && (at >= low[n][e & 1] || at < p.sinks) ? x : 0.f;
                        }
                        sum[2 * b + (e >> 1)] += x;
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], 1);
            sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], 2);
        }
        if (put) weight[at] = old + (cc == 0 ? sum[0] : cc == 1 ? sum[1] : cc == 2 ? sum[2] : sum[3]);
        __syncwarp();
        if (++stage == WG_STAGES) stage = 0;
        if (cu.u + 1 == cu.nu) fresh = true;
        cu.step(a, p);
    }
    cp_wait<0>();
}

}  // namespace asx
