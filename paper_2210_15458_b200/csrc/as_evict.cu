// Eviction: which tokens of a lane and key head stay, and where they go.
#include "as_cache4_host.cuh"

#include <type_traits>

namespace asx {

ASX_BOUNDS_READER(bounds_evict)

template <int NT> constexpr int EV_PER = NT == 256 ? 4 : 8;     // positions that a thread looks at between two sums over the CTA
constexpr int EV_MAX_CTAS = 8;
template <int NT> constexpr int EV_LIST = NT == 256 ? 1024 : 2048;      // places to fill, and tokens to go there, that are matched at a time
constexpr int EV_BINS = 2048;

struct EvictArgs {
    CacheArgs c;
    const float* weight;
    float* out;
    long long weight_ld;
    const int *keep, *first, *ref;
    int recent;
};

// Shared memory: this, the two lists, then the middle's keys where there is room for them.
template <int NT> struct EvictSmem {
    static constexpr int ROOM = EV_LIST<NT> + NT * EV_PER<NT>;
    int hist[EV_BINS];
    int hole[ROOM], mover[ROOM];
    int warp_sum[NT / 32];
    int digit, above;
};

// a weight's place in the order: larger keys for larger weights, one key for both zeros, 0 for a NaN
__device__ __forceinline__ uint32_t weight_key(float x) {
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Exclusive sum over the CTA's threads, in thread order, and the total.
template <int NT>
__device__ __forceinline__ int sum_before(EvictSmem<NT>& sm, int mine, int& total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int v = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                        // (the last call's readers are done)
    if (lane == 31) sm.warp_sum[w] = v;
    __syncthreads();
    int s = lane < NT / 32 ? sm.warp_sum[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += u;
    }
    total = __shfl_sync(0xFFFFFFFFu, s, 31);
    const int before = __shfl_sync(0xFFFFFFFFu, s, w > 0 ? w - 1 : 0);
    return v - mine + (w > 0 ? before : 0);
}

// Sixteen tokens of a head are moved by half a warp, a thread to a token: in a tile, the codes of 16 values of neighbouring tokens lie side by
// side, and so do the scales (half a warp to a token: 512 recent tokens of 64 x 8 heads 68 us in place of 18).  Keys' codes are 64 or 32 bytes
// of a token: several threads to each.  The first half of the copy moves those, the second everything else; `between` separates loads from stores.
__device__ __forceinline__ long long token_tile(const EvictArgs& e, int lane, int head, int pos) {
    const CacheArgs& c = e.c;
    const int mask = (1 << c.page_shift) - 1;
    const int page = c.table[(size_t)ASX_AT(lane, c.lanes, 321) * c.max_pages + ASX_AT(pos >> c.page_shift, c.max_pages, 322)];
    return ((long long)ASX_AT(page, c.n_pages, 323) * c.heads + ASX_AT(head, c.heads, 324)) * (mask + 1 >> 4) + ((pos & mask) >> 4);
}
// A tile on its way into L2: a token's bytes lie in a dozen places of it, which HBM gives singly at a third of its rate.
template <int D>
__device__ __forceinline__ void fetch_tile(const EvictArgs& e, int lane, int head, int pos) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(e.c.pages + token_tile(e, lane, head, pos) * Tile4<D>::BYTES), "r"(Tile4<D>::BYTES) : "memory");
}
template <int D, class F>
__device__ __forceinline__ void move_tokens(const EvictArgs& e, int lane, int head, bool have, int src, int dst, const float* w, float* out, bool weights, F&& between) {
    using Ti = Tile4<D>;
    constexpr int KP = D / 32, NB = D / 16;             // 16-byte pieces of a token's key codes, blocks
    const int l = threadIdx.x & 15;
    char* const pages = e.c.pages;
    const long long from = have ? token_tile(e, lane, head, src) : -1, to = have ? token_tile(e, lane, head, dst) : -1;
    // f(i, tile, place in it, piece): the half warp's tokens, n threads to each
    auto spread = [&](auto n, long long tile, int pos, auto&& f) {
        constexpr int N = decltype(n)::value;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int who = i * (16 / N) + l / N;
            const long long at = __shfl_sync(0xFFFFFFFFu, tile, who, 16);
            const int t = __shfl_sync(0xFFFFFFFFu, pos, who, 16) & 15;
            if (at >= 0) f(i, pages + at * Ti::BYTES, t, l % N);
        }
    };
    using Keys = std::integral_constant<int, KP>;
    {
        uint4 q[KP];
        spread(Keys{}, from, src, [&](int i, char* at, int t, int k) { q[i] = *reinterpret_cast<const uint4*>(at + Ti::k_code(t, 2 * k)); });
        between();
        spread(Keys{}, to, dst, [&](int i, char* at, int t, int k) { *reinterpret_cast<uint4*>(at + Ti::k_code(t, 2 * k)) = q[i]; });
    }
    uint2 v[NB], ks = make_uint2(0, 0);
    unsigned char vs[NB];
    float mine = 0.f;
    if (have) {
        const char* at = pages + from * Ti::BYTES;
        const int t = src & 15;
#pragma unroll
        for (int b = 0; b < NB; ++b) v[b] = *reinterpret_cast<const uint2*>(at + Ti::v_code(t, b));
#pragma unroll
        for (int b = 0; b < NB; ++b) vs[b] = *reinterpret_cast<const unsigned char*>(at + Ti::v_scale(t, b));
        if constexpr (D == 128) ks = *reinterpret_cast<const uint2*>(at + Ti::k_scale(t, 0));
        else ks.x = *reinterpret_cast<const uint32_t*>(at + Ti::k_scale(t, 0));
        if (weights) mine = w[src];
    }
    between();
    if (have) {
        char* at = pages + to * Ti::BYTES;
        const int t = dst & 15;
#pragma unroll
        for (int b = 0; b < NB; ++b) *reinterpret_cast<uint2*>(at + Ti::v_code(t, b)) = v[b];
#pragma unroll
        for (int b = 0; b < NB; ++b) at[Ti::v_scale(t, b)] = (char)vs[b];
        if constexpr (D == 128) *reinterpret_cast<uint2*>(at + Ti::k_scale(t, 0)) = ks;
        else *reinterpret_cast<uint32_t*>(at + Ti::k_scale(t, 0)) = ks.x;
        if (weights) out[dst] = mine;
    }
}

// One CTA per lane and key head.  The middle's weights become ordered keys in shared memory (or are read again where there is no
// room); the key that decides is found by a radix select, 11 + 11 + 10 bits; then the middle is walked twice side by side, by the places
// that come free below the new end and by the tokens that stay from behind it, a list of each at a time; then the recent tokens move down in
// their order, a batch being read before it is written.
// Few lanes and heads: a cluster of CTAs to one, each of which selects for itself and moves its share of the tokens.
// Only what changes its place is read and written, and the recent tokens alone keep their order: a token that stays in front of the new
// end does not move.  Bound by latency: 64 x 8 heads, 2112 tokens to 2048 with 512 recent ones 50 us (1.8 TB/s of what has to move; issue slots 38 %, DRAM
// 23 %), selection a third of it; 8 x 8 heads, up to 30000 to 4096, 111 us: selection 40, then 3700 tokens from all over the cache to
// each head, whose tiles are brought into L2 whole (without that 204 us).
template <int D, int NT, bool CLUSTER>
__global__ void __launch_bounds__(NT, NT == 256 ? 4 : 1) evict_kernel(const __grid_constant__ EvictArgs e, int room, int ctas) {
    extern __shared__ __align__(16) char ev_smem[];
    EvictSmem<NT>& sm = *reinterpret_cast<EvictSmem<NT>*>(ev_smem);
    uint32_t* const keys = reinterpret_cast<uint32_t*>(ev_smem + sizeof(EvictSmem<NT>));
    constexpr int PER = EV_PER<NT>, LOADS = 8;
    const CacheArgs& c = e.c;
    const int tid = threadIdx.x, rank = CLUSTER ? (int)(blockIdx.x % ctas) : 0;
    auto meet = [] {
        if constexpr (CLUSTER) {
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        } else {
            __syncthreads();
        }
    };
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int item = CLUSTER ? blockIdx.x / ctas : blockIdx.x; item < c.lanes * c.heads; item += CLUSTER ? gridDim.x / ctas : gridDim.x) {
        const int lane = c.by_heads.div(item), head = item - lane * c.heads;
        const int len = c.len[lane], keep = e.keep[lane], first = e.first ? e.first[lane] : 0, recent = e.recent;
        const float* w = e.weight + (size_t)item * e.weight_ld;
        float* out = e.out + (size_t)item * e.weight_ld;
        bool bad = len < 0 || len > ((long long)c.max_pages << c.page_shift) || len > e.weight_ld || keep < 0 || first < 0;
        const bool cut = !bad && len > keep;
        if (cut) bad = (long long)first + recent > keep;
        const int last = len - recent, want = keep - recent - first;       // of the middle [first, last) `want` tokens stay
        bool go = cut && !bad;
        const bool cached = go && last - first <= room;
        if (go) {
            // every page that is read or written
            const int* row = c.table + (size_t)lane * c.max_pages;
            bool odd = false;
            for (int m = (first >> c.page_shift) + tid; m <= (len - 1) >> c.page_shift; m += NT) {
                const int g = row[ASX_AT(m, c.max_pages, 325)];
                const bool in = g >= 0 && g < c.n_pages;
                odd |= !in || (e.ref && m << c.page_shift < keep && e.ref[in ? g : 0] > 1);
            }
            for (int i = tid; i < EV_BINS; i += NT) sm.hist[i] = 0;
            go = !__syncthreads_or(odd);
            if (go)
                for (int t = (last & ~15) + 16 * (rank * NT + tid); t < len; t += 16 * ctas * NT) fetch_tile<D>(e, lane, head, t);
            if (cached && go) {
                // (the first of the three passes counts while it is at it)
#pragma unroll 1
                for (int t0 = first + tid; t0 < last; t0 += NT * LOADS) {
                    float x[LOADS];
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) x[i] = t0 + i * NT < last ? w[t0 + i * NT] : 0.f;
#pragma unroll
                    for (int i = 0; i < LOADS; ++i)
                        if (t0 + i * NT < last) {
                            const uint32_t k = weight_key(x[i]);
                            keys[ASX_AT(t0 + i * NT - first, room, 328)] = k;
                            atomicAdd(&sm.hist[k >> 21], 1);
                        }
                }
            }
        }
        if (!go && (cut || bad) && c.lane_status && head == 0 && rank == 0 && tid == 0) c.lane_status[lane] = AS_ERR_INVALID_ARG;
        // places [first, end) and behind them the recent tokens; `shift`: how far those move
        const int end = keep - recent, shift = len - keep;
        if (out != w) {
#pragma unroll 1
            for (long long t0 = rank * NT + tid; t0 < e.weight_ld; t0 += (long long)ctas * NT * LOADS) {
                float x[LOADS];
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const long long t = t0 + (long long)i * ctas * NT;
                    x[i] = t >= e.weight_ld ? 0.f : !go || t < end || t >= len ? w[t] : t < keep ? w[t + shift] : 0.f;
                }
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const long long t = t0 + (long long)i * ctas * NT;
                    if (t < e.weight_ld) out[t] = x[i];
                }
            }
        }
        if (!go) {
            __syncthreads();
            continue;
        }
        meet();                             // (in place, nothing is written before all have read; else places are filled after they were copied)
        const int share = cached ? ctas : 1, mine_of = rank;
        if (rank < share) {
        auto key = [&](int t) { return cached ? keys[ASX_AT(t - first, room, 329)] : weight_key(w[t]); };

        // ---- the key that decides, and how many of those equal to it stay ----
        uint32_t prefix = 0xFFFFFFFFu;      // (no key is as large)
        int need = want;
        if (want > 0) {
            uint32_t mask = 0;
            prefix = 0;
#pragma unroll 1
            for (int pass = 0; pass < 3; ++pass) {
                const int at = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : EV_BINS;
                if (pass > 0) {
                    for (int i = tid; i < EV_BINS; i += NT) sm.hist[i] = 0;
                    __syncthreads();
                }
                if (pass > 0 || !cached)
#pragma unroll 4
                    for (int t = first + tid; t < last; t += NT) {
                        const uint32_t k = key(t);
                        if ((k & mask) == prefix) atomicAdd(&sm.hist[ASX_AT((k >> at) & (bins - 1), EV_BINS, 330)], 1);
                    }
                __syncthreads();
                constexpr int BP = EV_BINS / NT;        // bins of a thread, the largest first
                int n[BP], mine = 0, total;
#pragma unroll
                for (int i = 0; i < BP; ++i) { n[i] = sm.hist[EV_BINS - 1 - (tid * BP + i)]; mine += n[i]; }
                int above = sum_before<NT>(sm, mine, total);
#pragma unroll
                for (int i = 0; i < BP; ++i) {
                    if (above < need && need <= above + n[i]) { sm.digit = EV_BINS - 1 - (tid * BP + i); sm.above = above; }
                    above += n[i];
                }
                __syncthreads();
                prefix |= (uint32_t)sm.digit << at;
                mask |= (uint32_t)(bins - 1) << at;
                need -= sm.above;
                __syncthreads();
            }
        }

        // ---- kept tokens from behind the new end, to the places of those given up in front of it ----
        constexpr int STEP = NT * PER, ROOM = EvictSmem<NT>::ROOM;
        int ph = first, pm = end, nh = 0, nm = 0, tie_h = 0, tie_m = 0;
        {   // equal keys in front of `end`
            int mine = 0, total;
            for (int t = first + tid; t < end; t += NT) mine += key(t) == prefix;
            sum_before<NT>(sm, mine, total);
            tie_m = total;
        }
        // A thread looks at PER neighbours; larger keys and equal ones are counted in halves of a word.
        auto look = [&](int t0, int to, int ties, int& bigger, int& equal, int (&rank)[PER], unsigned& stays) {
            uint32_t k[PER];
            int mine = 0, total;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                k[i] = t0 + i < to ? key(t0 + i) : 0u;
                if (t0 + i < to) mine += k[i] > prefix ? 1 : k[i] == prefix ? 1 << 16 : 0;
            }
            const int before = sum_before<NT>(sm, mine, total);
            bigger = total & 0xFFFF;
            equal = total >> 16;
            int b = before & 0xFFFF, q = ties + (before >> 16);
            stays = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                // (of those before it: the larger ones, and of the equal ones the first `need`)
                rank[i] = b + min(q, need) - min(ties, need);
                if (t0 + i >= to) continue;
                if (k[i] > prefix) { stays |= 1u << i; ++b; }
                else if (k[i] == prefix) { if (q < need) stays |= 1u << i; ++q; }
            }
        };
        while (true) {
            while (nh < EV_LIST<NT> && ph < end) {
                const int t0 = ph + tid * PER;
                int bigger, equal, rank[PER];
                unsigned stays;
                look(t0, end, tie_h, bigger, equal, rank, stays);
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (t0 + i < end && !(stays >> i & 1)) sm.hole[ASX_AT(nh + tid * PER + i - rank[i], ROOM, 326)] = t0 + i;
                nh += min(STEP, end - ph) - (bigger + min(tie_h + equal, need) - min(tie_h, need));
                tie_h += equal;
                ph += STEP;
            }
            while (nm < EV_LIST<NT> && pm < last) {
                const int t0 = pm + tid * PER;
                int bigger, equal, rank[PER];
                unsigned stays;
                look(t0, last, tie_m, bigger, equal, rank, stays);
                if (stays && (t0 >> 4) % share == mine_of) fetch_tile<D>(e, lane, head, t0);
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (stays >> i & 1) sm.mover[ASX_AT(nm + rank[i], ROOM, 327)] = t0 + i;
                nm += bigger + min(tie_m + equal, need) - min(tie_m, need);
                tie_m += equal;
                pm += STEP;
            }
            __syncthreads();
            const int n = min(nh, nm);      // (in all there are as many of the ones as of the others)
            if (n == 0) break;
            for (int i0 = 0; i0 < n; i0 += share * NT) {
                const int i = i0 + ((tid >> 4) * share + rank) * 16 + (tid & 15);       // (sixteen to a CTA in turn)
                move_tokens<D>(e, lane, head, i < n, i < n ? sm.mover[i] : 0, i < n ? sm.hole[i] : 0, w, out, true, [] {});
            }
            __syncthreads();
            // what is left of the longer list comes first in the next round
            constexpr int MOST = ROOM / NT;
            int a[MOST], b[MOST];
#pragma unroll
            for (int i = 0; i < MOST; ++i) {
                const int at = n + i * NT + tid;
                a[i] = at < nh ? sm.hole[at] : 0;
                b[i] = at < nm ? sm.mover[at] : 0;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MOST; ++i) {
                const int at = n + i * NT + tid;
                if (at < nh) sm.hole[at - n] = a[i];
                if (at < nm) sm.mover[at - n] = b[i];
            }
            nh -= n;
            nm -= n;
            __syncthreads();
        }

        }
        meet();                             // (tokens that stayed from behind the new end have been read)

        // ---- the recent tokens: places [end, keep) from `shift` further behind, in batches from the front; where the two do not overlap
        // their order does not matter ----
        const bool apart = shift >= recent;
        if (rank == 0 || apart)
            for (int d0 = (end & ~15) + (apart ? rank * NT : 0); d0 < keep; d0 += apart ? ctas * NT : NT) {
                const int dst = d0 + tid;
                const bool have = dst >= end && dst < keep;
                move_tokens<D>(e, lane, head, have, have ? dst + shift : 0, have ? dst : 0, w, out, out == w, [&] { if (!apart) __syncthreads(); });
            }
        meet();
        if (out == w)
            for (int t = keep + rank * NT + tid; t < len; t += ctas * NT) out[t] = 0.f;
        __syncthreads();
    }
}

template <int D, int NT, bool CLUSTER>
static cudaError_t launch_evict_nt(const EvictArgs& e, size_t most, int ctas, int sms, cudaStream_t st) {
    static bool attr_set[64] = {false};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = evict_kernel<D, NT, CLUSTER>;
    if (!attr_set[dev]) {
        const cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_OPTIN_MAX);
        if (err != cudaSuccess) return err;
        attr_set[dev] = true;
    }
    const long long tokens = (long long)e.c.max_pages << e.c.page_shift, have = (long long)(most - sizeof(EvictSmem<NT>)) / 4;
    long long room = e.weight_ld < tokens ? e.weight_ld : tokens;
    if (room > have) room = have;
    const long long items = (long long)e.c.lanes * e.c.heads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((items < 64 * sms ? items : 64 * sms) * ctas));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = sizeof(EvictSmem<NT>) + 4 * (size_t)room;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)ctas, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = CLUSTER ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, e, (int)room, ctas);
}
template <int D>
static cudaError_t launch_evict(const EvictArgs& e, int sms, cudaStream_t st) {
    // Many lanes and heads: small CTAs, four on an SM, if the keys find room there; few, or long ones: the largest there are, each with an SM's
    // shared memory, several to one as long as they all run side by side.  Small / large, us: 2112 tokens, 8 heads, 32 lanes 29 / 51, 64 lanes 46 / 101, 16
    // lanes 27 / 27; up to 30000 tokens, 40 lanes 555 / 374, 8 lanes 288 / 113 (one to each 153).
    const long long items = (long long)e.c.lanes * e.c.heads, tokens = (long long)e.c.max_pages << e.c.page_shift;
    constexpr size_t SMALL = 56 * 1024;
    const bool fits = (e.weight_ld < tokens ? e.weight_ld : tokens) <= (long long)(SMALL - sizeof(EvictSmem<256>)) / 4;
    if (fits && items > sms) return launch_evict_nt<D, 256, false>(e, SMALL, 1, sms, st);
    int ctas = 1;
    while (ctas < EV_MAX_CTAS && 2 * ctas * items <= sms) ctas *= 2;
    return ctas == 1 ? launch_evict_nt<D, 1024, false>(e, SMEM_OPTIN_MAX, 1, sms, st) : launch_evict_nt<D, 1024, true>(e, SMEM_OPTIN_MAX, ctas, sms, st);
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
    const cudaError_t err = cache->head_dim == 64 ? launch_evict<64>(e, di->sms, st) : launch_evict<128>(e, di->sms, st);
    return err == cudaSuccess ? AS_OK : cuda_fail(err, "evict kernel launch");
}

}  // extern "C"
