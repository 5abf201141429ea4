// Attention weights of cached tokens for many query rows (a chunk of a prompt, the last tokens of one): products on the tensor
// cores with accumulators in TMEM.
#pragma once
#include "as_attend_tc.cuh"
#include "as_weigh.cuh"

namespace asx {

constexpr int WT_ROWS = 128;                // query rows of a tile
constexpr int WT_STAGES = 4;                // row tiles in shared memory, and score tiles in TMEM
constexpr int WT_CONSTS = 8;                // row tiles whose factors and log-sums are in shared memory: those are needed until a tile is summed
// Threads: a warp that issues products, one that brings in query tiles (two are not used), four that fill in keys, groups of four that sum.
constexpr int WT_FILL = 4, WT_GROUPS = 3, WT_NT = 32 * (4 * WT_GROUPS + 8);
constexpr int WT_MAX_RUNS = 160;

// A row tile as it lies in scratch and in shared memory: 128 rows of f16, swizzled as tc_at() has it, then for each pair of rows
// (factor of both, minus log-sum of both): a score s adds 2^(s factor - log-sum).
template <int D> constexpr int WT_MAT = WT_ROWS * D * 2;
template <int D> constexpr int WT_TILE = WT_MAT<D> + WT_ROWS * 8;

struct WeighTcArgs {
    WeighArgs w;
    char* tiles;                            // [lanes][heads][row_tiles] of WT_TILE
    int row_tiles;
    const int* steps;                       // [lanes] pairs of a token tile and a row tile that it needs, of one head
    float* part;                            // [2 * runs][128] sums of token tiles that a run saw in part
    int4* info;                             // [runs] (lane, head, token tile, bits: 1 its first token tile was begun by another run, 2 that one ends here, 4 the
                                            // run has come to its end)
    int runs;
};

// Rows [lo, hi) look at position t; rows are ordered by query token.
__device__ __forceinline__ int rows_from(const WeighArgs& w, int len, int t) { return min(w.a.c.T, max(0, t - (len - w.a.c.T))) * (int)w.a.by_g.d; }
__device__ __forceinline__ int rows_to(const WeighArgs& w, int len, int t) {
    const long long tok = (long long)t + w.p.window - (len - w.a.c.T);      // (query tokens below it)
    return (t < w.p.sinks || tok > w.a.c.T ? w.a.c.T : max(0, (int)tok)) * (int)w.a.by_g.d;
}

// A lane's places [lo, hi), counted without the hole.
struct WeighLane {
    int lo, hi, len;
    Hole<true> hole;
    __device__ __forceinline__ WeighLane(const WeighArgs& w, int b) {
        token_range<true>(w.a, w.p, b, b, lo, hi, hole);
        len = lane_len(w.a.c, b);
    }
    __device__ __forceinline__ int tiles() const { return (hi - lo + TC_KV - 1) / TC_KV; }
    // first row tile of a token tile and how many there are
    __device__ __forceinline__ int2 row_span(const WeighArgs& w, int tile) const {
        const int v0 = lo + tile * TC_KV, v1 = min(v0 + TC_KV, hi) - 1;
        const int from = rows_from(w, len, hole.real(v0));
        const int to = v0 < w.p.sinks ? w.p.rows : rows_to(w, len, hole.real(v1));
        const int a = from / WT_ROWS, b = (to + WT_ROWS - 1) / WT_ROWS;
        return make_int2(a, max(0, b - a));
    }
};

// One CTA per row tile of a lane and key head: rows as f16, scaled by a power of two each (exact down to 2^-17 of the row's largest element,
// below that within 2^-25 of it), as the products take them.  Done once here and not by every CTA that meets the tile: a
// tile of rows meets up to 64 of tokens.  HBM and L2: 17 us for 2 x 2048 x 32 heads of 128.
template <int D>
__global__ void __launch_bounds__(256) weigh_rows_kernel(const __grid_constant__ WeighTcArgs t) {
    constexpr int PER = D / 8, AT_ONCE = 256 / PER;     // threads to a row, 8 elements each
    const WeighArgs& w = t.w;
    const AttendArgs& a = w.a;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int items = a.c.lanes * a.c.heads * t.row_tiles;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int rt = item % t.row_tiles, lh = item / t.row_tiles, lane = a.c.by_heads.div(lh), head = lh - lane * a.c.heads;
        char* to = t.tiles + (size_t)item * WT_TILE<D>;
        float* consts = reinterpret_cast<float*>(to + WT_MAT<D>);
        const float to_log2 = a.scale * (a.c.k_scale ? a.c.k_scale[head] : 1.f) * 1.44269504088896f;
        const int j = threadIdx.x % PER;
#pragma unroll
        for (int i = 0; i < WT_ROWS / AT_ONCE; ++i) {
            const int r = i * AT_ONCE + threadIdx.x / PER, row = rt * WT_ROWS + r;
            float lse = -INFINITY;
            if (row < w.p.rows) lse = w.lse[out_row(a, lane, head, row)];
            uint32_t x[4] = {0, 0, 0, 0};
            if (lse != -INFINITY) {         // (a row that sees nothing, or is none, is all zeros and adds 2^-inf)
                const uint16_t* from = reinterpret_cast<const uint16_t*>(query_row<AS_BF16, D>(a, lane, head, row)) + 8 * j;
                if ((reinterpret_cast<uintptr_t>(from) & 15) == 0) {
                    const uint4 q = *reinterpret_cast<const uint4*>(from);
                    x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = from[2 * e] | (uint32_t)from[2 * e + 1] << 16;
                }
            }
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max(top, max(x[e] & 0x7FFFu, x[e] >> 16 & 0x7FFFu));
#pragma unroll
            for (int o = PER / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            int ex = (int)(top >> 7) - 127;
            ex = ex > 126 ? 126 : ex < -126 ? -126 : ex;
            const float down = __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = pack_f16(__uint_as_float(x[e] << 16) * down, __uint_as_float(x[e] & 0xFFFF0000u) * down);
            *reinterpret_cast<uint4*>(to + ASX_AT((j / 8) * (WT_ROWS * 128) + tc_at(r, j % 8), WT_MAT<D> - 15, 361)) = make_uint4(x[0], x[1], x[2], x[3]);
            if (j == 0) {
                consts[(r >> 1) * 4 + (r & 1)] = __uint_as_float((uint32_t)(127 + ex) << 23) * to_log2;
                consts[(r >> 1) * 4 + 2 + (r & 1)] = -lse * 1.44269504088896f;
                if (lse == -INFINITY) consts[(r >> 1) * 4 + 2 + (r & 1)] = -INFINITY;
            }
        }
    }
}

// A wait for loads from TMEM that what they bring in depends on.
__device__ __forceinline__ void wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                   "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) : : "memory");
}
struct WeighTcSmem {
    unsigned long long q_full[WT_STAGES], q_empty[WT_STAGES], c_full[WT_CONSTS], c_empty[WT_CONSTS], s_full[WT_STAGES], s_empty[WT_STAGES], k_full[2], k_empty[2], sum_full[2], sum_empty[2], fin;
    uint32_t tmem;
    int failed;
    int start[5];                           // lane, head, token tile, step within it; steps of the run
    int4 info;                              // of the run, for the join
    int warp_sum[WT_NT / 32];
    float sum[2][WT_GROUPS - 1][TC_KV];
};
template <int D> constexpr size_t weigh_tc_smem() { return 1024 + (size_t)2 * TC_KV * D * 2 + (size_t)WT_STAGES * WT_MAT<D> + (size_t)WT_CONSTS * WT_ROWS * 8 + (size_t)TC_KV * (D / 2) + sizeof(WeighTcSmem); }

// Where a run stands: (lane, head, token tile), the row tiles of that and how many of them are behind.
struct WeighCursor {
    int lane, head, tile, tiles, at, n, first;  // first: the first of the row tiles
    WeighLane l;
    __device__ __forceinline__ WeighCursor(const WeighTcArgs& t, const int* start) : lane(start[0]), head(start[1]), tile(start[2]), at(start[3]), l(t.w, start[0]) {
        tiles = l.tiles();
        span(t);
    }
    __device__ __forceinline__ void span(const WeighTcArgs& t) {
        const int2 s = l.row_span(t.w, tile);
        first = s.x;
        n = s.y;
    }
    // the next token tile that any row looks at
    __device__ __noinline__ void next(const WeighTcArgs& t) {
        at = 0;
        do {
            if (++tile >= tiles) {
                tile = 0;
                if (++head >= t.w.a.c.heads) {
                    head = 0;
                    do { ++lane; } while (lane < t.w.a.c.lanes && t.steps[lane] == 0);
                    if (lane >= t.w.a.c.lanes) return;
                    l = WeighLane(t.w, lane);
                    tiles = l.tiles();
                }
            }
            span(t);
        } while (n == 0);
    }
};

// A token of a tile of 128 is a thread, S = K Q^T has a row for each token and a column for each query row: a thread adds up
// 2^(s - z) over the columns that look at its token, row tile after row tile.  Groups of 128 threads take the row tiles of a
// token tile in turn.  Steps (a token tile with a row tile) are dealt out to the CTAs in equal runs; a token tile that falls to
// several leaves partial sums that the join kernel adds in the runs' order.
// Tokens as rows: a thread's sum stays in a register over all row tiles, where rows as rows would have to be summed across
// threads.  A query's factor and log-sum come with its tile; -inf takes a row out, so that only tiles on the diagonal or a window's edge are
// masked.  Bound by the special-function unit: an exponential for each pair, 736 M of them for 2 x 2048 rows x 32 heads over up to 8192 tokens (its
// pipe 72 % busy over the kernel, tensor pipe 36 %): 250 us, 280 with the kernels around it (672 TFLOP/s).  Two groups that sum: 316 us in all, three
// 284; four do not fit the registers.  Part of the exponentials as polynomials gained nothing once three groups summed.
template <int D>
__global__ void __launch_bounds__(WT_NT, 1) weigh_tc_kernel(const __grid_constant__ WeighTcArgs t) {
    using Ti = Tile4<D>;
    constexpr int MAT = TC_KV * D * 2, BLK = TC_KV * 128, KSTEPS = D / 16;
    extern __shared__ char raw[];
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(raw) + 1023) & ~1023u;
    const uint32_t k_s = base, q_s = k_s + 2 * MAT, c_s = q_s + WT_STAGES * WT_MAT<D>, raw_s = c_s + WT_CONSTS * WT_ROWS * 8;
    WeighTcSmem& sm = *reinterpret_cast<WeighTcSmem*>(raw + (raw_s + TC_KV * (D / 2) - (uint32_t)__cvta_generic_to_shared(raw)));
    auto bar = [](const unsigned long long& b) { return (uint32_t)__cvta_generic_to_shared(&b); };
    const WeighArgs& wa = t.w;
    const CacheArgs& c = wa.a.c;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int i = 0; i < WT_STAGES; ++i) {
            tc_bar_init(bar(sm.q_full[i]), 1); tc_bar_init(bar(sm.q_empty[i]), 1);
            tc_bar_init(bar(sm.s_full[i]), 1); tc_bar_init(bar(sm.s_empty[i]), 4);
        }
        for (int i = 0; i < WT_CONSTS; ++i) { tc_bar_init(bar(sm.c_full[i]), 1); tc_bar_init(bar(sm.c_empty[i]), 4); }
        for (int i = 0; i < 2; ++i) {
            tc_bar_init(bar(sm.k_full[i]), WT_FILL); tc_bar_init(bar(sm.k_empty[i]), 1);
            tc_bar_init(bar(sm.sum_full[i]), 4 * (WT_GROUPS - 1)); tc_bar_init(bar(sm.sum_empty[i]), 4);
        }
        tc_bar_init(bar(sm.fin), 1);
        sm.failed = 0;
        sm.start[4] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // ---- the run: lanes' steps are added up, the run's first step is looked for in its lane ----
    {
        const int per = (c.lanes + WT_NT - 1) / WT_NT, j0 = min(tid * per, c.lanes), j1 = min(j0 + per, c.lanes);
        int mine = 0;
        for (int j = j0; j < j1; ++j) mine += t.steps[j];
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) sm.warp_sum[w] = incl;
        __syncthreads();
        int before = incl - mine, total = 0;
        for (int i = 0; i < WT_NT / 32; ++i) {
            before += i < w ? sm.warp_sum[i] : 0;
            total += sm.warp_sum[i];
        }
        const unsigned U = (unsigned)total * c.heads, G = min((unsigned)t.runs, U), k = blockIdx.x;
        if (k >= G) return;
        if (tid == 0) sm.info = make_int4(0, 0, 0, 0);
        const unsigned q = U / G, r = U - q * G;
        const unsigned from = q * k + r * k / G, n = q * (k + 1) + r * (k + 1) / G - from;
        unsigned at = (unsigned)before * c.heads;
        for (int j = j0; j < j1; ++j) {
            const unsigned all = (unsigned)t.steps[j] * c.heads;
            if (from >= at && from < at + all) {
                sm.start[0] = j;
                sm.start[1] = (int)((from - at) / t.steps[j]);
                sm.start[3] = (int)((from - at) % t.steps[j]);
                sm.start[4] = (int)n;
            }
            at += all;
        }
        __syncthreads();
        if (w == 0) {                       // the token tile, 32 at a time
            const WeighLane l(wa, sm.start[0]);
            int left = sm.start[3], found = -1;
            for (int i0 = 0; i0 < l.tiles() && found < 0; i0 += 32) {
                const int mine2 = i0 + lane < l.tiles() ? l.row_span(wa, i0 + lane).y : 0;
                int sum = mine2;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                    if (lane >= o) sum += v;
                }
                const unsigned hit = __ballot_sync(0xFFFFFFFFu, sum > left);
                if (hit) {
                    const int at32 = __ffs(hit) - 1;
                    found = i0 + at32;
                    left -= __shfl_sync(0xFFFFFFFFu, sum - mine2, at32);
                } else {
                    left -= __shfl_sync(0xFFFFFFFFu, sum, 31);
                }
            }
            if (lane == 0) { sm.start[2] = found; sm.start[3] = left; }
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(&sm.tmem)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;              // (all 512 columns: 0)
    const int run = sm.start[4];
    const long long limit = wa.p.wait_cycles;
    volatile int* failed = &sm.failed;
    bool ok = true;
    auto wait_warp = [&](const unsigned long long& b, uint32_t parity) { return __all_sync(0xFFFFFFFFu, tc_wait(bar(b), parity, limit, failed)); };
    int x = 0;                                  // steps behind

    if (w >= 8) {
        // ------------------------------------------------ sums ------------------------------------------------
        const int s = (w - 8) >> 2, r = tid & 127;
        const uint32_t mine = (uint32_t)(w & 3) << 21;              // the warp's 32 lanes of TMEM
        WeighCursor cu(t, sm.start);
#pragma unroll 1
        for (int unit = 0; x < run && ok; ++unit) {
            const int tiles = min(cu.n - cu.at, run - x);
            const int place = cu.l.lo + cu.tile * TC_KV + r, pos = cu.l.hole.real(place);
            const int from = rows_from(wa, cu.l.len, pos), to = place < cu.l.hi ? rows_to(wa, cu.l.len, pos) : 0;
            float sum = 0.f;
#pragma unroll 1
            for (int j = (s + WT_GROUPS - x % WT_GROUPS) % WT_GROUPS; j < tiles; j += WT_GROUPS) {          // (the groups take a run's steps in turn)
                const int step = x + j, b = step % WT_STAGES, cb = step % WT_CONSTS;
                ok = wait_warp(sm.c_full[cb], (uint32_t)(step / WT_CONSTS) & 1) && wait_warp(sm.s_full[b], (uint32_t)(step / WT_STAGES) & 1);
                if (!ok) break;
                tc_fence_after();
                const int row0 = (cu.first + cu.at + j) * WT_ROWS;
                const uint32_t consts = c_s + ASX_AT(cb, WT_CONSTS, 362) * (WT_ROWS * 8);
                const int lo = from - row0, hi = to - row0;
                const bool cut = __any_sync(0xFFFFFFFFu, lo > 0 || hi < WT_ROWS);
                uint64_t part[2] = {0, 0};
                // 16 columns while the next 16 come in
                auto columns = [&](uint32_t (&v)[16], int col) {
                    const uint32_t at = consts + col * 8;
                    float y[16];
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const uint4 kz = lds<uint4>(at + e * 8);
                        const float2 x = unpair(fma2(pair(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), pair(__uint_as_float(kz.x), __uint_as_float(kz.y)),
                                                     pair(__uint_as_float(kz.z), __uint_as_float(kz.w))));
                        y[e] = ex2(x.x);
                        y[e + 1] = ex2(x.y);
                    }
                    if (cut) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = col + e >= lo && col + e < hi ? y[e] : 0.f;
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 2) part[e / 2 & 1] = add2(part[e / 2 & 1], pair(y[e], y[e + 1]));
                };
                uint32_t va[16], vb[16];
                const uint32_t scores = 128 * b + mine;
                tc_ld16(scores, va);
#pragma unroll 1
                for (int col = 0; col < WT_ROWS; col += 32) {
                    wait16(va);
                    tc_ld16(scores + ASX_AT(col + 16, 113, 363), vb);
                    columns(va, col);
                    wait16(vb);
                    if (col + 32 < WT_ROWS) tc_ld16(scores + col + 32, va);
                    columns(vb, col + 16);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { tc_bar_arrive(bar(sm.s_empty[b])); tc_bar_arrive(bar(sm.c_empty[cb])); }
                const float2 both = unpair(add2(part[0], part[1]));
                sum += both.x + both.y;         // (a tile's sum first, then the tiles')
            }
            if (!ok) break;
            // ---- the end of a token tile or of the run: the groups' sums become one ----
            const int p = unit & 1;
            const uint32_t again = (uint32_t)(unit >> 1) & 1;
            if (s > 0) {
                if (unit >= 2) ok = wait_warp(sm.sum_empty[p], again ^ 1);
                if (!ok) break;
                sm.sum[p][ASX_AT(s - 1, WT_GROUPS - 1, 373)][r] = sum;
                __syncwarp();
                if (lane == 0) tc_bar_arrive(bar(sm.sum_full[p]));
            } else {
                ok = wait_warp(sm.sum_full[p], again);
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < WT_GROUPS - 1; ++i) sum += sm.sum[p][i][r];
                __syncwarp();
                if (lane == 0) tc_bar_arrive(bar(sm.sum_empty[p]));
                const bool begun = cu.at > 0, ends = cu.at + tiles == cu.n;
                if (begun || !ends) t.part[(size_t)ASX_AT(2 * blockIdx.x + (begun ? 0 : 1), 2 * WT_MAX_RUNS, 364) * TC_KV + r] = sum;
                else if (place < cu.l.hi) put_weight(wa, cu.lane, cu.head, pos, wa.first[cu.lane], cu.l.len, sum);
                if (unit == 0 && r == 0) sm.info = make_int4(cu.lane, cu.head, cu.tile, (begun ? 1 : 0) | (ends ? 2 : 0) | 4);
            }
            x += tiles;
            if (x < run) cu.next(t);
        }
    } else if (w >= 4) {
        // ------------------------------------------------ keys ------------------------------------------------
        const int r = tid & 127, tk = r & 15;
        const int page_mask = (1 << c.page_shift) - 1, tiles_per_page = 1 << (c.page_shift - 4);
        WeighCursor cu(t, sm.start);
        const uint32_t own = raw_s + r * 16;
        uint4 code[D / 32];
        uint2 scale = make_uint2(0, 0);
        // the token's codes and scales a token tile before they are widened, its page's id one before that
        WeighCursor ahead = cu;
        int looked = 0, page = 0, next_lane = 0;
        bool real = false;
        const char* place0 = c.pages;           // the token's place within page 0 of its head
        auto look = [&]() {
            real = false;
            if (looked >= run) return;
            const int place = ahead.l.lo + ahead.tile * TC_KV + r, pos = ahead.l.hole.real(place);
            if (place < ahead.l.hi) {
                page = c.table[(size_t)ASX_AT(ahead.lane, c.lanes, 366) * c.max_pages + ASX_AT(pos >> c.page_shift, c.max_pages, 367)];
                place0 = c.pages + ((size_t)ASX_AT(ahead.head, c.heads, 368) * tiles_per_page + ((pos & page_mask) >> 4)) * Ti::BYTES;
                next_lane = ahead.lane;
                real = true;
            }
            looked += min(ahead.n - ahead.at, run - looked);
            if (looked < run) ahead.next(t);
        };
        auto load = [&]() {
            if (real && (page < 0 || page >= c.n_pages)) {
                flag_lane(c.lane_status, next_lane, AS_ERR_INVALID_ARG);
                page = 0;
            }
            const char* src = real ? place0 + (size_t)page * c.heads * tiles_per_page * Ti::BYTES : c.pages;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) code[i] = __ldg(reinterpret_cast<const uint4*>(src + Ti::k_code(tk, 2 * i)));
            if constexpr (D == 128) scale = __ldg(reinterpret_cast<const uint2*>(src + Ti::k_scale(tk, 0)));
            else scale.x = __ldg(reinterpret_cast<const uint32_t*>(src + Ti::k_scale(tk, 0)));
            look();
        };
        auto widen = [](uint32_t codes, uint32_t scale2) {
            uint32_t f[4];
            codes_f16x2(codes, f);
            return make_uint4(mul_f16(f[0], scale2), mul_f16(f[1], scale2), mul_f16(f[2], scale2), mul_f16(f[3], scale2));
        };
        auto put = [](uint32_t at, const uint4& v) { asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); };
        look();
        load();
#pragma unroll 1
        for (int unit = 0; x < run && ok; ++unit) {
            const int b = unit & 1;
            if (unit >= 2) ok = wait_warp(sm.k_empty[b], (uint32_t)((unit >> 1) & 1) ^ 1);
            if (!ok) break;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) put(raw_s + ASX_AT(own - raw_s + i * (TC_KV * 16), TC_KV * (D / 2) - 15, 369), code[i]);
            const uint32_t sc_lo = scale.x, sc_hi = scale.y;
            x += min(cu.n - cu.at, run - x);
            if (x < run) {
                cu.next(t);
                load();
            }
#pragma unroll 1
            for (int i = 0; i < D / 32; ++i) {
                const uint4 q = lds<uint4>(raw_s + ASX_AT(own - raw_s + i * (TC_KV * 16), TC_KV * (D / 2) - 15, 370));
                const uint32_t two = e4m3_f16x2(((D == 128 && i >= 2 ? sc_hi : sc_lo) >> (16 * (i & 1))) & 0xFFFFu);
                const uint32_t sa = __byte_perm(two, two, 0x1010), sb = __byte_perm(two, two, 0x3232);
                const uint32_t at = k_s + ASX_AT(b * MAT + (i >> 1) * BLK + r * 128, 2 * MAT - 127, 371);
                const int cx = (4 * (i & 1)) ^ (r & 7);
                put(at + ((cx ^ 0) << 4), widen(q.x, sa));
                put(at + ((cx ^ 1) << 4), widen(q.y, sa));
                put(at + ((cx ^ 2) << 4), widen(q.z, sb));
                put(at + ((cx ^ 3) << 4), widen(q.w, sb));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tc_bar_arrive(bar(sm.k_full[b]));
        }
    } else if (w == 1) {
        // ------------------------------------------------ query tiles ------------------------------------------------
        if (tc_elect()) {
            WeighCursor cu(t, sm.start);
#pragma unroll 1
            while (x < run && ok) {
                const int tiles = min(cu.n - cu.at, run - x);
                const char* src = t.tiles + (((size_t)cu.lane * c.heads + cu.head) * t.row_tiles + cu.first + cu.at) * WT_TILE<D>;
#pragma unroll 1
                for (int j = 0; j < tiles && ok; ++j, ++x, src += WT_TILE<D>) {
                    const int b = x % WT_STAGES, cb = x % WT_CONSTS;
                    if (x >= WT_CONSTS) ok = tc_wait(bar(sm.c_empty[cb]), ((uint32_t)(x / WT_CONSTS) & 1) ^ 1, limit, failed);
                    if (ok && x >= WT_STAGES) ok = tc_wait(bar(sm.q_empty[b]), ((uint32_t)(x / WT_STAGES) & 1) ^ 1, limit, failed);
                    if (!ok) break;
                    auto copy = [&](uint32_t to, const char* from, uint32_t bytes, uint32_t full) {
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full), "r"(bytes) : "memory");
                        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                     ::"r"(to), "l"(from), "r"(bytes), "r"(full) : "memory");
                    };
                    copy(q_s + ASX_AT(b, WT_STAGES, 372) * WT_MAT<D>, src, WT_MAT<D>, bar(sm.q_full[b]));
                    copy(c_s + ASX_AT(cb, WT_CONSTS, 374) * (WT_ROWS * 8), src + WT_MAT<D>, WT_ROWS * 8, bar(sm.c_full[cb]));
                }
                if (ok && x < run) cu.next(t);
            }
            // copies in flight end before the CTA does
            auto landed = [&](uint32_t full, uint32_t parity) {
                const long long start = clock64();
#pragma unroll 1
                while (!tc_try(full, parity) && clock64() - start < 2000000000LL) {}
            };
            for (int i = max(0, x - WT_STAGES); i < x; ++i) landed(bar(sm.q_full[i % WT_STAGES]), (uint32_t)(i / WT_STAGES) & 1);
            for (int i = max(0, x - WT_CONSTS); i < x; ++i) landed(bar(sm.c_full[i % WT_CONSTS]), (uint32_t)(i / WT_CONSTS) & 1);
        }
    } else if (w == 0) {
        // ------------------------------------------------ issuing ------------------------------------------------
        if (tc_elect()) {
            constexpr uint32_t ID = tc_idesc(128, WT_ROWS, false);
            WeighCursor cu(t, sm.start);
#pragma unroll 1
            for (int unit = 0; x < run && ok; ++unit) {
                const int tiles = min(cu.n - cu.at, run - x), kb = unit & 1;
                ok = tc_wait(bar(sm.k_full[kb]), (uint32_t)(unit >> 1) & 1, limit, failed);
                const uint64_t k_d = tc_desc(k_s + kb * MAT, 0);
#pragma unroll 1
                for (int j = 0; j < tiles && ok; ++j, ++x) {
                    const int b = x % WT_STAGES;
                    const uint32_t use = (uint32_t)(x / WT_STAGES) & 1;
                    ok = tc_wait(bar(sm.q_full[b]), use, limit, failed);
                    if (ok && x >= WT_STAGES) ok = tc_wait(bar(sm.s_empty[b]), use ^ 1, limit, failed);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t q_d = tc_desc(q_s + b * WT_MAT<D>, 0);
#pragma unroll
                    for (int k = 0; k < KSTEPS; ++k) {
                        const uint32_t at = (k / 4) * (BLK >> 4) + (k % 4) * 2;
                        tc_mma_ss(128 * b, k_d + at, q_d + at, ID, k > 0);
                    }
                    tc_commit(bar(sm.s_full[b]));
                    tc_commit(bar(sm.q_empty[b]));
                    if (j + 1 == tiles) tc_commit(bar(sm.k_empty[kb]));
                }
                if (ok && x < run) cu.next(t);
            }
            // whatever is still in flight ends before TMEM is freed
            tc_commit(bar(sm.fin));
            const long long start = clock64();
#pragma unroll 1
            while (!tc_try(bar(sm.fin), 0) && clock64() - start < 2000000000LL) {}
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // (of a run in which a wait has run out, none of the sums in scratch are joined: some may never have been written)
    if (tid == 0) t.info[ASX_AT(blockIdx.x, WT_MAX_RUNS, 365)] = sm.failed ? make_int4(0, 0, 0, 0) : sm.info;
    if (sm.failed && tid == 0) {
#pragma unroll 1
        for (int j = 0; j < c.lanes; ++j) flag_lane(c.lane_status, j, AS_ERR_TIMEOUT);
    }
    if (w == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// One CTA per run that ends a token tile which others began: their sums in order, so that nothing depends on timing.  Latency, 5 us.
static __global__ void __launch_bounds__(TC_KV) weigh_join_kernel(const __grid_constant__ WeighTcArgs t) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int k = blockIdx.x, r = threadIdx.x;
    unsigned steps = 0;                         // (all the lanes')
    for (int j = r; j < t.w.a.c.lanes; j += TC_KV) steps += t.steps[j];
    __shared__ unsigned all;
    if (r == 0) all = 0;
    __syncthreads();
    atomicAdd(&all, steps);
    __syncthreads();
    if (k >= (int)min((unsigned)t.runs, all * t.w.a.c.heads)) return;
    const int4 i = t.info[k];
    if (i.w != 7) return;                       // (a tile that runs on is joined where it ends)
    int c0 = k - 1;
    while (c0 > 0 && t.info[c0].w == 5) --c0;   // (a run inside one token tile)
    if (!(t.info[c0].w & 4)) return;            // (a wait has run out there: the tile's weights stay as they are)
    float sum = t.part[(size_t)(2 * c0 + 1) * TC_KV + r];
    for (int j = c0 + 1; j <= k; ++j) sum += t.part[(size_t)(2 * j) * TC_KV + r];
    const WeighLane l(t.w, i.x);
    const int place = l.lo + i.z * TC_KV + r;
    if (place < l.hi) put_weight(t.w, i.x, i.y, l.hole.real(place), t.w.first[i.x], l.len, sum);
}

}  // namespace asx
