// Eviction: which tokens of a lane and key head stay, and where they go.
#include "as_cache4_host.cuh"

namespace asx {

ASX_BOUNDS_READER(bounds_evict)

constexpr int EV_NT = 512;
constexpr int EV_LIST = 1024;               // places to fill, and tokens to go there, that are matched at a time

struct EvictArgs {
    CacheArgs c;
    const float* weight;
    float* out;
    long long weight_ld;
    const int *keep, *first, *ref;
    int recent;
};

struct EvictSmem {
    int hist[256];
    int hole[EV_LIST + EV_NT], mover[EV_LIST + EV_NT];
    int warp_a[EV_NT / 32], warp_b[EV_NT / 32];
    int digit, above;
};

// a weight's place in the order: larger keys for larger weights, one key for both zeros, 0 for a NaN
__device__ __forceinline__ uint32_t weight_key(float x) {
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Exclusive sums over the CTA's threads of two small numbers, and their totals.
__device__ __forceinline__ void scan_two(EvictSmem& sm, int a, int b, int& before_a, int& before_b, int& total_a, int& total_b) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int v = a | b << 16;                    // (each total is at most EV_NT)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                        // (the last call's readers are done)
    if (lane == 31) sm.warp_a[w] = v;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < EV_NT / 32; ++i) {
        const int u = sm.warp_a[i];
        before += i < w ? u : 0;
        total += u;
    }
    before += v;
    before_a = (before & 0xFFFF) - a;
    before_b = (before >> 16) - b;
    total_a = total & 0xFFFF;
    total_b = total >> 16;
}

// A token of a head is moved by D / 8 threads, thread j of them: 16 bytes of key codes (j < D / 32), 8 bytes of value codes and
// their scale (block j - D / 32, of D / 16), or the key scales (the one behind those).
template <int D> struct TokenPiece {
    uint4 q;
    uint32_t s;
    float w;
};
template <int D>
__device__ __forceinline__ char* token_tile(const EvictArgs& e, int lane, int head, int pos) {
    const CacheArgs& c = e.c;
    const int mask = (1 << c.page_shift) - 1;
    const int page = c.table[(size_t)ASX_AT(lane, c.lanes, 321) * c.max_pages + ASX_AT(pos >> c.page_shift, c.max_pages, 322)];
    return c.pages + (((size_t)ASX_AT(page, c.n_pages, 323) * c.heads + ASX_AT(head, c.heads, 324)) * (mask + 1 >> 4) + ((pos & mask) >> 4)) * Tile4<D>::BYTES;
}
template <int D>
__device__ __forceinline__ void take_token(const char* tile, int t, int j, TokenPiece<D>& x) {
    using Ti = Tile4<D>;
    constexpr int KP = D / 32, NB = D / 16;
    if (j < KP) {
        x.q = *reinterpret_cast<const uint4*>(tile + Ti::k_code(t, 2 * j));
    } else if (j < KP + NB) {
        const uint2 v = *reinterpret_cast<const uint2*>(tile + Ti::v_code(t, j - KP));
        x.q.x = v.x; x.q.y = v.y;
        x.s = *reinterpret_cast<const unsigned char*>(tile + Ti::v_scale(t, j - KP));
    } else if (j == KP + NB) {
        if constexpr (D == 128) {
            const uint2 v = *reinterpret_cast<const uint2*>(tile + Ti::k_scale(t, 0));
            x.q.x = v.x; x.q.y = v.y;
        } else {
            x.q.x = *reinterpret_cast<const uint32_t*>(tile + Ti::k_scale(t, 0));
        }
    }
}
template <int D>
__device__ __forceinline__ void put_token(char* tile, int t, int j, const TokenPiece<D>& x) {
    using Ti = Tile4<D>;
    constexpr int KP = D / 32, NB = D / 16;
    if (j < KP) {
        *reinterpret_cast<uint4*>(tile + Ti::k_code(t, 2 * j)) = x.q;
    } else if (j < KP + NB) {
        *reinterpret_cast<uint2*>(tile + Ti::v_code(t, j - KP)) = make_uint2(x.q.x, x.q.y);
        tile[Ti::v_scale(t, j - KP)] = (char)x.s;
    } else if (j == KP + NB) {
        if constexpr (D == 128) *reinterpret_cast<uint2*>(tile + Ti::k_scale(t, 0)) = make_uint2(x.q.x, x.q.y);
        else *reinterpret_cast<uint32_t*>(tile + Ti::k_scale(t, 0)) = x.q.x;
    }
}

// One CTA per lane and key head.  The weight that decides is found by a radix select on ordered keys (8 bits a pass); then the
// middle is walked twice side by side, by the places that come free below the new end and by the tokens that stay from behind it, a list
// of each at a time; then the recent tokens move down in their order, a batch being read before it is written.
template <int D>
__global__ void __launch_bounds__(EV_NT) evict_kernel(const __grid_constant__ EvictArgs e) {
    __shared__ EvictSmem sm;
    const CacheArgs& c = e.c;
    const int tid = threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int item = blockIdx.x; item < c.lanes * c.heads; item += gridDim.x) {
        const int lane = c.by_heads.div(item), head = item - lane * c.heads;
        const int len = c.len[lane], keep = e.keep[lane], first = e.first ? e.first[lane] : 0, recent = e.recent;
        const float* w = e.weight + (size_t)item * e.weight_ld;
        float* out = e.out + (size_t)item * e.weight_ld;
        bool bad = len < 0 || len > ((long long)c.max_pages << c.page_shift) || len > e.weight_ld || keep < 0 || first < 0;
        const bool cut = !bad && len > keep;
        if (cut) bad = (long long)first + recent > keep;
        if (cut && !bad) {
            // every page that is read or written
            const int* row = c.table + (size_t)lane * c.max_pages;
            bool odd = false;
            for (int m = (first >> c.page_shift) + tid; m <= (len - 1) >> c.page_shift; m += EV_NT) {
                const int g = row[ASX_AT(m, c.max_pages, 325)];
                const bool in = g >= 0 && g < c.n_pages;
                odd |= !in || (e.ref && m << c.page_shift < keep && e.ref[in ? g : 0] > 1);
            }
            bad = __syncthreads_or(odd);
        }
        if (bad && c.lane_status && head == 0 && tid == 0) c.lane_status[lane] = AS_ERR_INVALID_ARG;
        // places [first, end) and behind them the recent tokens; `shift`: how far those move
        const int end = cut && !bad ? keep - recent : 0, shift = len - keep;
        if (out != w) {
            const bool go = cut && !bad;
            for (long long t = tid; t < e.weight_ld; t += EV_NT)
                out[t] = !go || t < end || t >= len ? w[t] : t < keep ? w[t + shift] : 0.f;
        }
        if (bad || !cut) continue;
        const int last = len - recent, want = end - first;      // of the middle [first, last) `want` tokens stay

        // ---- the key that decides, and how many of those equal to it stay ----
        uint32_t prefix = 0, mask = 0;
        int need = want;
        if (want > 0) {
            for (int shift8 = 24; shift8 >= 0; shift8 -= 8) {
                for (int i = tid; i < 256; i += EV_NT) sm.hist[i] = 0;
                __syncthreads();
                for (int t = first + tid; t < last; t += EV_NT) {
                    const uint32_t k = weight_key(w[t]);
                    if ((k & mask) == prefix) atomicAdd(&sm.hist[(k >> shift8) & 255], 1);
                }
                __syncthreads();
                if (tid < 32) {
                    int n[8], mine = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) { n[i] = sm.hist[255 - (8 * tid + i)]; mine += n[i]; }
                    int incl = mine;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                        if (tid >= o) incl += u;
                    }
                    int at = incl - mine;
                    if (at < need && need <= incl) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (at < need && need <= at + n[i]) { sm.digit = 255 - (8 * tid + i); sm.above = at; }
                            at += n[i];
                        }
                    }
                }
                __syncthreads();
                prefix |= (uint32_t)sm.digit << shift8;
                mask |= 0xFFu << shift8;
                need -= sm.above;
                __syncthreads();
            }
        } else {
            prefix = 0xFFFFFFFFu;           // (no key is as large)
            need = 0;
        }

        // ---- kept tokens from behind the new end, to the places of those given up in front of it ----
        constexpr int PER = D / 8, GROUPS = EV_NT / PER, U = 4;
        const int j = tid % PER, grp = tid / PER;
        int ph = first, pm = end, nh = 0, nm = 0, tie_h = 0;
        // equal keys in front of `end`: the places' walk counts them again as it goes, the tokens' walk starts behind them
        int tie_m = 0;
        {
            int mine = 0;
            for (int t = first + tid; t < end; t += EV_NT) mine += weight_key(w[t]) == prefix;
            mine = __reduce_add_sync(0xFFFFFFFFu, mine);
            if ((tid & 31) == 0) sm.warp_b[tid >> 5] = mine;
            __syncthreads();
            for (int i = 0; i < EV_NT / 32; ++i) tie_m += sm.warp_b[i];
        }
        while (true) {
            while (nh < EV_LIST && ph < end) {
                const int t = ph + tid;
                const uint32_t k = t < end ? weight_key(w[t]) : 0u;
                int tb, hb, ties, holes;
                const bool tie = t < end && k == prefix;
                scan_two(sm, tie, 0, tb, hb, ties, holes);
                const bool hole = t < end && !(k > prefix || (tie && tie_h + tb < need));
                int b0, b1, t1;
                scan_two(sm, hole, 0, hb, b0, holes, t1);
                (void)b1;
                if (hole) sm.hole[ASX_AT(nh + hb, EV_LIST + EV_NT, 326)] = t;
                nh += holes;
                tie_h += ties;
                ph += EV_NT;
            }
            while (nm < EV_LIST && pm < last) {
                const int t = pm + tid;
                const uint32_t k = t < last ? weight_key(w[t]) : 0u;
                int tb, b0, ties, t1;
                const bool tie = t < last && k == prefix;
                scan_two(sm, tie, 0, tb, b0, ties, t1);
                const bool stays = t < last && (k > prefix || (tie && tie_m + tb < need));
                int mb, movers;
                scan_two(sm, stays, 0, mb, b0, movers, t1);
                if (stays) sm.mover[ASX_AT(nm + mb, EV_LIST + EV_NT, 327)] = t;
                nm += movers;
                tie_m += ties;
                pm += EV_NT;
            }
            __syncthreads();
            const int n = min(nh, nm);      // (in all there are as many of the ones as of the others)
            if (n == 0) break;
            for (int i0 = 0; i0 < n; i0 += GROUPS * U) {
                TokenPiece<D> x[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * GROUPS + grp;
                    if (i < n) {
                        const int src = sm.mover[i];
                        take_token<D>(token_tile<D>(e, lane, head, src), src & 15, j, x[u]);
                        if (j == PER - 1) x[u].w = w[src];
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * GROUPS + grp;
                    if (i < n) {
                        const int dst = sm.hole[i];
                        put_token<D>(token_tile<D>(e, lane, head, dst), dst & 15, j, x[u]);
                        if (j == PER - 1) out[dst] = x[u].w;
                    }
                }
            }
            __syncthreads();
            // what is left of the longer list comes first in the next round
            int a[(EV_LIST + EV_NT) / EV_NT], b[(EV_LIST + EV_NT) / EV_NT];
#pragma unroll
            for (int i = 0; i < (EV_LIST + EV_NT) / EV_NT; ++i) {
                const int at = n + i * EV_NT + tid;
                a[i] = at < nh ? sm.hole[at] : 0;
                b[i] = at < nm ? sm.mover[at] : 0;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < (EV_LIST + EV_NT) / EV_NT; ++i) {
                const int at = n + i * EV_NT + tid;
                if (at < nh) sm.hole[at - n] = a[i];
                if (at < nm) sm.mover[at - n] = b[i];
            }
            nh -= n;
            nm -= n;
            __syncthreads();
        }

        // ---- the recent tokens: places [end, keep) from `shift` further behind, in batches from the front ----
        for (int d0 = end; d0 < keep; d0 += GROUPS * U) {
            TokenPiece<D> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int dst = d0 + u * GROUPS + grp, src = dst + shift;
                if (dst < keep) {
                    take_token<D>(token_tile<D>(e, lane, head, src), src & 15, j, x[u]);
                    if (out == w && j == PER - 1) x[u].w = w[src];
                }
            }
            __syncthreads();                // (later batches' tokens lie behind this one's places)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int dst = d0 + u * GROUPS + grp;
                if (dst < keep) {
                    put_token<D>(token_tile<D>(e, lane, head, dst), dst & 15, j, x[u]);
                    if (out == w && j == PER - 1) out[dst] = x[u].w;
                }
            }
        }
        __syncthreads();
        if (out == w)
            for (int t = keep + tid; t < len; t += EV_NT) out[t] = 0.f;
        __syncthreads();
    }
}

}  // namespace asx

using namespace asx;

extern "C" {

int as_cache4_evict(const as_cache4* cache, const float* d_weight, long long weight_ld, int lanes, const int32_t* d_table, int max_pages,
                    const int32_t* d_len, const int32_t* d_keep, const int32_t* d_first, int recent, const int32_t* d_ref, float* d_weight_out,
                    int32_t* d_lane_status, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(AS_F32, lanes, 1, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    if (recent < 0) return set_err(AS_ERR_INVALID_ARG, "recent = %d must be >= 0", recent);
    if (weight_ld < 1) return set_err(AS_ERR_INVALID_ARG, "weight_ld = %lld must be >= 1", weight_ld);
    if ((long long)lanes * cache->heads > 0x7FFFFFFFLL) return set_err(AS_ERR_UNSUPPORTED, "lanes * heads must be below 2^31");
    if (lanes == 0) return AS_OK;
    if (!d_keep || !d_weight || !d_weight_out) return set_err(AS_ERR_INVALID_ARG, "d_keep, d_weight or d_weight_out is NULL");
    if ((reinterpret_cast<uintptr_t>(d_weight) | reinterpret_cast<uintptr_t>(d_weight_out)) & 3) return set_err(AS_ERR_INVALID_ARG, "d_weight or d_weight_out is not element-aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = clear_status(d_lane_status, lanes, st)) != AS_OK) return rc;
    EvictArgs e;
    e.c = cache_args(cache, lanes, 1, d_table, max_pages, d_len, d_lane_status);
    e.weight = d_weight; e.out = d_weight_out; e.weight_ld = weight_ld;
    e.keep = d_keep; e.first = d_first; e.ref = d_ref; e.recent = recent;
    const long long items = (long long)lanes * cache->heads;
    const unsigned grid = (unsigned)(items < 64 * di->sms ? items : 64 * di->sms);
    const cudaError_t err = cache->head_dim == 64 ? launch_after(evict_kernel<64>, grid, EV_NT, 0, st, e) : launch_after(evict_kernel<128>, grid, EV_NT, 0, st, e);
    return err == cudaSuccess ? AS_OK : cuda_fail(err, "evict kernel launch");
}

}  // extern "C"
