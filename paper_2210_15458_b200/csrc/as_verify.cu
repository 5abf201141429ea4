// The step over drafted tokens: which of them are accepted, and the token behind them.
#include "../../include/arith_sampling.h"
#include "as_generic.cuh"
#include "as_host.h"

namespace asx {

ASX_BOUNDS_READER(bounds_verify)

// What a row's distribution needs besides the row: p_j = exp((l_j - lmax) / temp) / Z over the kept tokens, those whose key is
// above T or equal to it and at an index up to `tie`.
struct RowCut {
    double lmax, Z;
    uint32_t T;
    int tie, status, pad;
};

struct VerifyArgs {
    const char *target, *draft;
    long long target_ld, draft_ld;          // bytes
    int lanes, K, V;
    const int *drafted, *n;
    const double *u, *codes;
    double inv_tau, top_p;
    int top_k;
    int *tokens, *accepted;
    double* codes_out;
    int* lane_status;
    RowCut* cuts;                           // [lanes][2 K + 1]: the target's rows, then the draft's
    int *stop, *arrived;                    // [lanes] K + 1 - place of the first refusal known so far, [lanes][K] rows of a place that are done; 0 at first
};

__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int lane) {
    const int n = a.n ? a.n[lane] : a.K;
    return n < 0 || n > a.K ? -1 : n;
}
__device__ __forceinline__ const char* target_row(const VerifyArgs& a, int lane, int i) { return a.target + ((long long)lane * (a.K + 1) + i) * a.target_ld; }
__device__ __forceinline__ const char* draft_row(const VerifyArgs& a, int lane, int i) { return a.draft + ((long long)lane * a.K + i) * a.draft_ld; }
__device__ __forceinline__ RowCut* cut_of(const VerifyArgs& a, int lane, int i, bool of_draft) {
    return a.cuts + ASX_AT((long long)lane * (2 * a.K + 1) + (of_draft ? a.K + 1 + i : i), (long long)a.lanes * (2 * a.K + 1), 341);
}

template <int DT>
struct RowMass {
    using Tr = Traits<DT>;
    const char* row;
    bool vec;
    RowCut c;
    __device__ RowMass(const char* r, const RowCut* cut) : row(r), vec((reinterpret_cast<uintptr_t>(r) & 15) == 0) {
        // (another CTA may just have written it: past L1)
        c.lmax = __ldcg(&cut->lmax); c.Z = __ldcg(&cut->Z);
        c.T = __ldcg(&cut->T); c.tie = __ldcg(&cut->tie); c.status = __ldcg(&cut->status);
    }
    __device__ __forceinline__ double operator()(uint32_t key, int j, double inv_tau, const double* tbl) const {
        return key > c.T || (key == c.T && j <= c.tie) ? exp_nonpos(((double)Tr::value_f(key) - c.lmax) * inv_tau, tbl) : 0.0;
    }
};

// What becomes of the lane's drafted token i, both rows' cuts known: 0 accepted, 1 refused, else an error.
template <int DT>
__device__ __noinline__ int decide(const VerifyArgs& a, int lane, int i, const double* tbl) {
    const int x = a.drafted[(size_t)lane * a.K + i];
    const double u = a.u[(size_t)lane * a.K + i];
    const RowMass<DT> p(target_row(a, lane, i), cut_of(a, lane, i, false));
    if (x < 0 || x >= a.V) return AS_ERR_INVALID_ARG;
    if (!(u >= 0.0 && u < 1.0) || p.c.status != ST_OK) return AS_ERR_NUMERIC;
    const double px = p(Traits<DT>::load_key(p.row, x), x, a.inv_tau, tbl) / p.c.Z;
    double qx = 1.0;
    if (a.draft) {
        const RowMass<DT> q(draft_row(a, lane, i), cut_of(a, lane, i, true));
        if (q.c.status != ST_OK) return AS_ERR_NUMERIC;
        qx = q(Traits<DT>::load_key(q.row, x), x, a.inv_tau, tbl) / q.c.Z;
    }
    return u * qx < px ? 0 : 1;
}

// A CTA to a row: its kept tokens and their mass, by the general routine of the step.  Rows come in the order of their places; whoever
// finishes a place's last row looks what becomes of its token, and rows behind a refusal that is known by the time they start are left out.
// (Which those are depends on timing, what comes out does not: nobody looks at them.)
// Bound by the general routine's instructions, some 92 us for a row of 50257 alone, hardly by bytes (issue slots 61 %, DRAM 7 %): 96 x 5 x 50257 in 32
// bits with a nucleus of 0.95: 276 us, 296 with all rows read, and the next kernel 37 (wide nuclei, of logits of spread 2: 627 us in all).
template <int DT, int VF_NT>
__global__ void __launch_bounds__(VF_NT) verify_rows_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ GenericSmem<VF_NT> sm;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // rows in the order of the places, the target's and the draft's of a place side by side
    const int per = a.draft ? 2 : 1, block = blockIdx.x / a.lanes, lane = blockIdx.x - block * a.lanes;
    const int i = block / per;
    const bool of_draft = block % per;
    const int n = drafts_of(a, lane);
    if (i > n - (of_draft ? 1 : 0) || a.K + 1 - i < __ldcg(a.stop + lane)) return;
    const char* row = of_draft ? draft_row(a, lane, i) : target_row(a, lane, i);
    GenericLane<DT, VF_NT> g(sm, row, a.V, (reinterpret_cast<uintptr_t>(row) & 15) == 0);
    g.inv_tau = a.inv_tau;
    fill_exp_table(sm.exp_tbl, threadIdx.x);
    Pred p;
    int n_kept;
    RowCut c;
    c.status = g.prepare(a.top_k, a.top_p, p, n_kept);
    if (c.status == ST_OK) {
        // the index of the last of the equal keys that are kept
        c.tie = p.eq_mode == 1 ? 0x7FFFFFFF : -1;
        if (p.eq_mode == 2) {
            if (threadIdx.x == 0) sm.b_i[0] = -1;
            __syncthreads();
            for (int ci = threadIdx.x; ci < g.nchunks; ci += VF_NT)
                if (sm.chunk_eq[ci] < p.need && p.need <= sm.chunk_eq[ci + 1]) sm.b_i[0] = ci;
            __syncthreads();
            const int ci = sm.b_i[0];
            if (ci >= 0 && threadIdx.x < 32) {
                int run = sm.chunk_eq[ci];
                for (int r = 0; r < g.R; ++r) {
                    uint32_t k[Traits<DT>::E];
                    int base;
                    g.chunk_keys(ci, r, k, base);
                    int rank = g.lane_rank0(k, p, run);
#pragma unroll
                    for (int e = 0; e < Traits<DT>::E; ++e)
                        if (k[e] == p.T && ++rank == p.need) sm.b_i[1] = base + e;
                }
            }
            __syncthreads();
            c.tie = sm.b_i[1];
        }
        c.lmax = g.lmax;
        c.Z = sm.chunk_sum[g.nchunks];
        c.T = p.T;
    }
    if (threadIdx.x == 0) {
        *cut_of(a, lane, i, of_draft) = c;
        if (i < n) {
            __threadfence();
            if (!a.draft || atomicAdd(&a.arrived[(size_t)lane * a.K + i], 1) == 1) {
                __threadfence();
                if (decide<DT>(a, lane, i, sm.exp_tbl) != 0) atomicMax(&a.stop[lane], a.K + 1 - i);
            }
        }
    }
}

// One CTA per lane: how many of its tokens are accepted, and the token behind them by its code, over masses
// max(p - q Zp / Zq, 0) in units of 1 / Zp: sums of chunks in index order, the chunk that holds the code, the token in it.
template <int DT, int VF_NT>
__global__ void __launch_bounds__(VF_NT) verify_finish_kernel(const __grid_constant__ VerifyArgs a) {
    using Tr = Traits<DT>;
    constexpr int E = Tr::E, NW = VF_NT / 32;
    __shared__ GenericSmem<VF_NT> sm;
    __shared__ int s_at, s_status;
    __shared__ bool s_refused;
    const int tid = threadIdx.x, lane32 = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    fill_exp_table(sm.exp_tbl, tid);
    __syncthreads();
    for (int lane = blockIdx.x; lane < a.lanes; lane += gridDim.x) {
        const int n = drafts_of(a, lane);
        const double c_in = a.codes[lane];
        if (warp == 0) {
            // a lane of the warp to a place: 0 accepted, 1 refused, else an error
            int at = max(n, 0), status = n < 0 ? AS_ERR_INVALID_ARG : AS_OK;
            bool refused = false;
            for (int i0 = 0; i0 < n; i0 += 32) {
                const int i = i0 + lane32;
                int what = 0;
                // (rows behind a refusal may have been left out)
                if (i < n && a.K + 1 - i >= a.stop[lane]) what = decide<DT>(a, lane, i, sm.exp_tbl);
                const unsigned stop = __ballot_sync(FULL, what != 0);
                if (stop) {
                    const int l = __ffs(stop) - 1;
                    at = i0 + l;
                    what = __shfl_sync(FULL, what, l);
                    refused = what == 1;
                    if (!refused) status = what;
                    break;
                }
            }
            if (status == AS_OK && (!(c_in >= 0.0 && c_in <= 1.0) || cut_of(a, lane, at, false)->status != ST_OK)) status = AS_ERR_NUMERIC;
            if (lane32 == 0) { s_at = at; s_refused = refused; s_status = status; }
        }
        __syncthreads();
        const int at = s_at;
        const bool refused = s_refused;
        int* out = a.tokens + (size_t)lane * (a.K + 1);
        int token = -1;
        double code = c_in;
        if (s_status == AS_OK) {
            const RowMass<DT> p(target_row(a, lane, at), cut_of(a, lane, at, false));
            const bool two = refused && a.draft;
            const RowMass<DT> q(two ? draft_row(a, lane, at) : p.row, two ? cut_of(a, lane, at, true) : cut_of(a, lane, at, false));
            double ratio = two ? p.c.Z / q.c.Z : 0.0;
            int drop = refused && !a.draft ? a.drafted[(size_t)lane * a.K + at] : -1;
            GenericLane<DT, VF_NT> g(sm, p.row, a.V, p.vec);
            auto masses = [&](int ci, int r, double (&ev)[E], int& base) {
                const int vi = (ci * g.R + r) * 32 + lane32;
                base = vi * E;
                uint32_t k[E];
                g.chunk_keys(ci, r, k, base);
#pragma unroll
                for (int e = 0; e < E; ++e) ev[e] = base + e == drop ? 0.0 : p(k[e], base + e, a.inv_tau, sm.exp_tbl);
                if (ratio > 0.0 && vi < g.nvec) {
                    load_vec_keys<DT>(q.row, a.V, vi, q.vec, k);
#pragma unroll
                    for (int e = 0; e < E; ++e) ev[e] = fmax(fma(-ratio, q(k[e], base + e, a.inv_tau, sm.exp_tbl), ev[e]), 0.0);
                }
            };
            double Z = 0.0;
#pragma unroll 1
            for (int turn = 0; turn < 2; ++turn) {
                g.clear_has();
                for (int ci = warp; ci < g.nchunks; ci += NW) {
                    double local = 0.0;
                    for (int r = 0; r < g.R; ++r) {
                        double ev[E];
                        int base;
                        masses(ci, r, ev, base);
#pragma unroll
                        for (int e = 0; e < E; ++e) local += ev[e];
                    }
                    local = warp_sum_d(local);
                    if (lane32 == 0) g.put_chunk(ci, local);
                }
                __syncthreads();
                g.scan_exclusive(sm.chunk_sum, g.nchunks);
                Z = sm.chunk_sum[g.nchunks];
                if (Z > 0.0) break;
                __syncthreads();
                ratio = 0.0;                // p and q are alike in 64 bits: nothing is left of p - q
                drop = -1;
            }
            const double t = (c_in == 1.0 ? ASX_ONE_BELOW : c_in) * Z;
            if (tid == 0) { sm.b_i[0] = INT_MAX; sm.b_i[1] = -1; }
            __syncthreads();
            for (int ci = tid; ci < g.nchunks; ci += VF_NT)
                if (g.has_mass(ci)) {
                    atomicMax(&sm.b_i[1], ci);
                    if (t < sm.chunk_sum[ci + 1]) atomicMin(&sm.b_i[0], ci);
                }
            __syncthreads();
            const bool force_last = sm.b_i[0] == INT_MAX;
            const int ci = force_last ? sm.b_i[1] : sm.b_i[0];
            if (warp == 0) {
                double run = sm.chunk_sum[ASX_AT(ci, MAXCH + 1, 342)];
                int pick = -1, last = -1;
                double pick_S = 0.0, pick_e = 1.0, last_S = 0.0, last_e = 1.0;
                bool found = false;
                for (int r = 0; r < g.R && !found; ++r) {
                    double ev[E], local = 0.0;
                    int base;
                    masses(ci, r, ev, base);
#pragma unroll
                    for (int e = 0; e < E; ++e) local += ev[e];
                    const double incl = warp_incl_scan_d(local, lane32);
                    double S = __shfl_up_sync(FULL, incl, 1);
                    S = run + (lane32 == 0 ? 0.0 : S);
                    int mine = -1;
                    double mine_S = 0.0, mine_e = 1.0;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (ev[e] > 0.0) {
                            if (mine < 0 && t < S + ev[e]) { mine = base + e; mine_S = S; mine_e = ev[e]; }
                            last = base + e; last_S = S; last_e = ev[e];
                            S += ev[e];
                        }
                    const unsigned bal = __ballot_sync(FULL, !force_last && local > 0.0 && t < run + incl);
                    if (bal) {
                        const int l = __ffs(bal) - 1;
                        if (mine < 0) { mine = last; mine_S = last_S; mine_e = last_e; }
                        pick = __shfl_sync(FULL, mine, l);
                        pick_S = __shfl_sync(FULL, mine_S, l);
                        pick_e = __shfl_sync(FULL, mine_e, l);
                        found = true;
                    }
                    run += __shfl_sync(FULL, incl, 31);
                }
                if (!found) {               // rounding at the top end: the last token of the chunk
                    const unsigned best = warp_max_u((unsigned)(last + 1));
                    const int l = __ffs(__ballot_sync(FULL, (unsigned)(last + 1) == best)) - 1;
                    pick = __shfl_sync(FULL, last, l);
                    pick_S = __shfl_sync(FULL, last_S, l);
                    pick_e = __shfl_sync(FULL, last_e, l);
                }
                token = pick;
                code = (t - pick_S) / pick_e;
                if (!(code >= 0.0)) code = 0.0;
                if (code > ASX_ONE_BELOW) code = ASX_ONE_BELOW;
            }
        }
        const bool ok = s_status == AS_OK;
        for (int i = tid; i <= a.K; i += VF_NT)
            if (!ok || i != at) out[i] = ok && i < at ? a.drafted[(size_t)lane * a.K + i] : -1;
        if (tid == 0) {
            if (ok) out[at] = token;
            a.accepted[lane] = ok ? at : 0;
            a.codes_out[lane] = code;
            if (a.lane_status) a.lane_status[lane] = s_status;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Without a cut: a cluster of CTAs to a lane (one CTA where the lanes are many), from the first row to the last token.
//
// A decision needs u q(x) < p(x), that is the rows' sums, and those only as exactly as it takes: rows are read once, in 32 bits, with a
// running maximum, and where the two sides are then within VN_NEAR of each other the pair is read again in 64 bits.  Rows behind
// the first refusal are not read.  The last row pair is read once in 64 bits: with w near Zp / Zq from the sums in 32, every token but
// those within VN_NEAR of e_p = w e_q is known to have p > q or not, and
//   sum of max(p - q, 0) over a chunk = A / Zp - B / Zq,   A, B the masses of its tokens with p > q;
// the few others are listed and added once Zp and Zq are known.
// Bound by instructions: 1024 x 4 x 128256 in bf16 takes 600 to 643 us where its bytes take 199 (issue slots 60 %, special-function unit 39 %, 64-bit pipe
// 25 %), about half of it the rows in 32 bits, half the last pair in 64; all of it in 64 bits took 1013 us, exponentials by the step's routine
// 3254.  4 x 3 x 32000: 24 us, the kernel 20 of them; row sums a fifth of it, decisions, chunk sums and the pick by single warps most of the rest.
// ---------------------------------------------------------------------------
constexpr int VN_NT = 256, VN_NW = VN_NT / 32;
constexpr int VN_CHUNKS = 128;              // of a CTA
constexpr int VN_LIST = 256;
constexpr int VN_BATCH = 4;                 // places, at most, whose rows are read before the decisions are taken
constexpr int VN_MAX_CTAS = 8;
constexpr int VN_U = 4, VN_STAGES = 3;      // granules of a thread at a time, steps that it has in flight or in use
// Of a sum in 32 bits: terms are off by 2^-22 (the exponential) and 2^-23 of their exponent, at most 130 before they vanish (2^-16 in all); 32 of
// them are added up before 64 bits take over (2^-19).  Where a thread's running maximum goes up its sum is scaled by a factor that is off by
// 2^-22, at most 256 times, once for each step of a row of 2^20 tokens in 32 bits (2^-14).  Sums are then joined up to 16 times (5 in a
// warp, 8 warps, 3 in a cluster), by such factors too (2^-18).  The factors' exponents are off by 1.5 x 2^-23 of themselves, and a sum that
// counts has not more than 60 of those in all (2^-17).  That makes 2^-13.3, and 2^-12.3 for the ratio of two sums; a row that falls, or hardly rises, has
// 2^-15.  Maxima beyond VN_FAR in units of log 2 (nothing that a model says) are left to 64 bits altogether.
constexpr double VN_NEAR = 1.0 / 4096;
constexpr int VN_NEAR_BITS = 12;
constexpr float VN_FAR = 1e6f;

struct RowSum { double s; float m; int bad; };
struct PairSum { double zp, zq; int listed, pad; };

constexpr int VN_RING = VN_STAGES * VN_U * VN_NT * 16;
constexpr int VN_SMEM = VN_RING + 16384;
struct VerifySmem {
    RowSum warp[2 * VN_BATCH][VN_NW];
    RowSum mine[2 * VN_BATCH];              // of the CTA's part of each row
    RowSum row[2 * VN_BATCH];
    PairSum part, warp_pair[VN_NW];
    double a[VN_CHUNKS + 1], b[VN_CHUNKS + 1];
    double sub[VN_NW];                      // (of the chosen chunk)
    double list_p[VN_LIST], list_q[VN_LIST];
    int list_j[VN_LIST], order[VN_LIST];
    int listed;
    double exp_tbl[256];                    // 2^(j / 256)
    double rest;                            // mass of max(p - q, 0) in the CTA's chunks
    int at, status, chunk, force_last;
};

static_assert(sizeof(VerifySmem) <= VN_SMEM - VN_RING, "shared memory of verify_lane_kernel");

__device__ __forceinline__ void cluster_sync(int ctas) {
    if (ctas == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}
// an object of another CTA of the cluster at the place that it has in this one
template <class V>
__device__ __forceinline__ V peer(const V& mine, int rank, int ctas) {
    if (ctas == 1) return mine;
    V got;
    uint32_t at, *to = reinterpret_cast<uint32_t*>(&got);
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&mine)), "r"(rank));
#pragma unroll
    for (int i = 0; i < (int)sizeof(V) / 4; ++i) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(to[i]) : "r"(at + 4 * i));
    return got;
}

// The CTAs' values of a cluster, one to a thread of each warp (0 behind the last): what is done with them is the same everywhere.
__device__ __forceinline__ double of_cluster(const double& mine, int ctas) { return (int)(threadIdx.x & 31) < ctas ? peer(mine, threadIdx.x & 31, ctas) : 0.0; }
__device__ __forceinline__ double cluster_total(const double& mine, int ctas) { return ctas == 1 ? mine : warp_sum_d(of_cluster(mine, ctas)); }

// A row as 16-byte granules from the boundary at or below its start: element e of granule g is token g E + e - off.
template <int DT>
struct Granules {
    static constexpr int E = Traits<DT>::E;
    const char* from;
    int off, n;
    __device__ __forceinline__ Granules(const char* row, int V) {
        const int low = (int)(reinterpret_cast<uintptr_t>(row) & 15);
        from = row - low;
        off = low / Traits<DT>::BYTES;
        n = (off + V + E - 1) / E;
    }
    __device__ __forceinline__ uint4 load(int g) const { return __ldg(reinterpret_cast<const uint4*>(from) + g); }
    // the same with -inf outside the row: only a row's first and last granules need it
    __device__ __forceinline__ void masked(int g, int V, uint4& q) const {
        if (g == 0 || (g + 1) * E - off > V) q = cut(q, g * E - off, V);
    }
    static __device__ __noinline__ uint4 cut(uint4 q, int j0, int V) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (j0 + e >= 0 && j0 + e < V) continue;
            if constexpr (DT == DT_F32) w[e] = 0xFF800000u;
            else w[e / 2] = (w[e / 2] & (e & 1 ? 0x0000FFFFu : 0xFFFF0000u)) | (e & 1 ? 0xFF800000u : 0x0000FF80u);
        }
        return q;
    }
};

__device__ __forceinline__ uint64_t two(float lo, float hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ float2 both(uint64_t x) {
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(x));
    return d;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

__device__ __forceinline__ RowSum join_sums(const RowSum& a, const RowSum& b, float c) {
    RowSum r;
    r.bad = a.bad | b.bad;
    r.m = fmaxf(a.m, b.m);
    r.s = (a.m == -INFINITY ? 0.0 : a.s * (double)ex2_approx((a.m - r.m) * c)) + (b.m == -INFINITY ? 0.0 : b.s * (double)ex2_approx((b.m - r.m) * c));
    return r;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The CTA's part of a row's maximum and sum, steps rank, rank + ctas, ... of VN_U VN_NT granules each; a warp's goes to out[warp].  A thread brings its
// granules into places of its own in shared memory, VN_STAGES - 1 steps ahead, so that nothing is waited for but its own copies.
template <int DT>
__device__ __forceinline__ void row_sum(const char* row, int V, float c, int rank, int ctas, uint32_t ring, RowSum* out) {
    constexpr int E = Traits<DT>::E;
    using P = Pass<DT>;
    const Granules<DT> g(row, V);
    const int step = ctas * VN_U * VN_NT, first = rank * VN_U * VN_NT + threadIdx.x;
    auto issue = [&](int g0, int stage) {
#pragma unroll
        for (int u = 0; u < VN_U; ++u)
            if (g0 + u * VN_NT < g.n) copy16(ring + (ASX_AT(stage, VN_STAGES, 347) * VN_U + u) * (VN_NT * 16), g.from + (size_t)(g0 + u * VN_NT) * 16);
        copies_close();
    };
#pragma unroll
    for (int i = 0; i < VN_STAGES - 1; ++i) issue(first + i * step, i);
    typename P::Acc acc = P::init();
    float m = -INFINITY, ref = 0.f;         // terms are 2^(x c - ref), ref = m c rounded; 0 where a finite number has masked all that the thread has seen
    double s = 0.0;
    const uint64_t cc = two(c, c);
    int stage = 0;
#pragma unroll 1
    for (int g0 = first; g0 < g.n; g0 += step) {
        copies_wait<VN_STAGES - 2>();
        issue(g0 + (VN_STAGES - 1) * step, stage == 0 ? VN_STAGES - 1 : stage - 1);
        uint4 q[VN_U];
#pragma unroll
        for (int u = 0; u < VN_U; ++u) {
            const int at = g0 + u * VN_NT;
            q[u] = DT == DT_F32 ? make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u) : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
            if (at < g.n) {
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q[u].x), "=r"(q[u].y), "=r"(q[u].z), "=r"(q[u].w)
                             : "r"(ring + (ASX_AT(stage, VN_STAGES, 348) * VN_U + u) * (VN_NT * 16)));
                g.masked(at, V, q[u]);
            }
        }
        if (++stage == VN_STAGES) stage = 0;
        typename P::Acc now = P::reduce(q[0]);
#pragma unroll
        for (int u = 1; u < VN_U; ++u) P::fold(now, q[u]);
        P::merge(acc, now);
        const float top = P::part_max(now);
        if (top > m) {
            const float to = fmaxf(top * c, -2.f * VN_FAR);
            s *= (double)ex2_approx(m == -INFINITY ? -INFINITY : ref - to);
            m = top;
            ref = to;
        }
        const uint64_t mm = two(-ref, -ref);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int u = 0; u < VN_U; ++u) {
            float x[E];
            P::floats(q[u], x);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 y = both(fma_two(two(x[e], x[e + 1]), cc, mm));
                sum[e / 2 & 1] = add_two(sum[e / 2 & 1], two(ex2_approx(y.x), ex2_approx(y.y)));
            }
        }
        const float2 t = both(add_two(sum[0], sum[1]));
        s += (double)(t.x + t.y);
    }
    copies_wait<0>();
    uint32_t k0, k1;
    P::keys(acc, k0, k1);
    RowSum r;
    r.bad = max(k0, k1) >= Traits<DT>::KEY_PINF || min(k0, k1) < Traits<DT>::KEY_NINF;      // +inf or a NaN
    r.m = m;
    // (What the rounding of ref has put on every term comes off; the product of two floats is exact in a double.  Not beyond VN_FAR, where that
    // may be any power of two: the sum vanishes beside the others', or the row's maximum lies out there too and no sum of it is used.)
    r.s = m == -INFINITY ? 0.0 : fabsf(ref) > VN_FAR ? s : s * (double)ex2_approx((float)((double)ref - (double)m * (double)c));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        RowSum other;
        other.s = __shfl_xor_sync(FULL, r.s, o);
        other.m = __shfl_xor_sync(FULL, r.m, o);
        other.bad = __shfl_xor_sync(FULL, r.bad, o);
        r = join_sums(r, other, c);
    }
    if ((threadIdx.x & 31) == 0) out[threadIdx.x >> 5] = r;
}

// Masses in 64 bits: 2^(t / 256), t = (x - m) 256 log2(e) / temp, = 2^n 2^(j / 256) exp(f ln2 / 256), |f| <= 1/2, the last factor by a polynomial of
// degree 4 (truncation 4e-17).  Logits far below m are raised to where their mass is 2^-1000: a token of VN_NONE or less counts as none,
// masked tokens among it.  Sums are over all tokens, those too; a chunk whose sum is above VN_SOME has a token that counts, as 2^20
// of those that do not come up to 2^-960.  t is one fused multiply-add: the rounding of m's product is the same for all of
// a row.  Maxima beyond VN_FAR are taken off the logits first (which is exact: differences that matter are multiples of a
// float's spacing there).
constexpr double VN_NONE = 0x1p-980, VN_SOME = 0x1p-955;
struct MassRow {
    float sub, low;
    double mc;
    __device__ __forceinline__ MassRow(float m, double c256) {
        const bool far = fabs((double)m * c256) > 256.0 * VN_FAR;
        sub = far ? m : 0.f;
        const double top = far ? 0.0 : m;
        mc = top * c256;
        low = fmaxf((float)(top - 256000.0 / c256), -3.4e38f);      // (above -inf)
    }
};
__device__ __forceinline__ double mass64(float x, const MassRow& r, double c256, const double* tbl) {
    x = fmaxf(x - r.sub, r.low);
    const double MAGIC = 6755399441055744.0;
    const double t = fma((double)x, c256, -r.mc);
    double k = t + MAGIC;
    const int i = __double2loint(k);
    k -= MAGIC;
    const double f = t - k;
    const double L = 0x1.62e42fefa39efp-9;               // ln2 / 256
    double p = fma(f, L * L * L * L / 24.0, L * L * L / 6.0);
    p = fma(p, f, L * L / 2.0);
    p = fma(p, f, L);
    p = fma(p, f, 1.0);
    const double v = tbl[i & 255] * p;
    return __hiloint2double(__double2hiint(v) + ((i >> 8) << 20), __double2loint(v));
}

// of one token of a row: 0 where it counts as none
__device__ __forceinline__ double token_mass(float l, const MassRow& r, double c256, const double* tbl) {
    const double e = mass64(l, r, c256, tbl);
    return e > VN_NONE ? e : 0.0;
}

// The last row pair of a lane (q.from null: p alone).
template <int DT>
struct LastPair {
    static constexpr int E = Traits<DT>::E;
    Granules<DT> p;
    const char* q;                          // the draft's row
    bool q_vec;                             // both rows lie alike on the granules
    MassRow mp, mq;
    double c256;
    int V, drop, R, per, c0, c1;            // R: sub-rows of 32 granules of a chunk; the CTA's chunks [c0, c1)
    const double* tbl;
    __device__ __forceinline__ LastPair(const VerifyArgs& a, const char* prow, const char* qrow, float mp_, float mq_, int drop_, double c256_, int rank, int ctas, const double* tbl_)
        : p(prow, a.V), q(qrow), mp(mp_, c256_), mq(mq_, c256_), c256(c256_), V(a.V), drop(drop_), tbl(tbl_) {
        q_vec = qrow && Granules<DT>(qrow, a.V).off == p.off;
        const int rows = (p.n + 31) / 32;
        R = (rows + ctas * (VN_CHUNKS / 2) - 1) / (ctas * (VN_CHUNKS / 2));
        const int chunks = (rows + R - 1) / R;
        per = (chunks + ctas - 1) / ctas;
        c0 = min(rank * per, chunks);
        c1 = min(c0 + per, chunks);
    }
    // A granule of the row and the draft's logits of the same tokens, -inf outside the row.
    struct Raw { uint4 p, q; };
    __device__ __forceinline__ Raw load(int g) const {
        Raw v;
        v.p = v.q = DT == DT_F32 ? make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u) : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
        if (g >= p.n) return v;
        v.p = p.load(g);
        if (!q) return v;
        if (q_vec) {
            v.q = __ldg(reinterpret_cast<const uint4*>(q - p.off * Traits<DT>::BYTES) + g);
        } else {
            uint32_t* w = reinterpret_cast<uint32_t*>(&v.q);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int j = g * E + e - p.off;
                if (j < 0 || j >= V) continue;
                if constexpr (DT == DT_F32) w[e] = reinterpret_cast<const uint32_t*>(q)[j];
                else w[e / 2] = (w[e / 2] & (e & 1 ? 0x0000FFFFu : 0xFFFF0000u)) | (uint32_t)reinterpret_cast<const uint16_t*>(q)[j] << (e & 1 ? 16 : 0);
            }
        }
        return v;
    }
    // f(e, mass of p, mass of q) for the tokens of a granule; without Q the draft's row is not looked at, and p's dropped token has no mass
    template <bool Q, class F>
    __device__ __forceinline__ void each(int g, Raw v, F&& f) const {
        if (g < p.n) {
            p.masked(g, V, v.p);
            if (Q && q_vec) p.masked(g, V, v.q);
        }
        float x[E], y[E];
        Pass<DT>::floats(v.p, x);
        if constexpr (Q) {
            Pass<DT>::floats(v.q, y);
#pragma unroll
            for (int e = 0; e < E; ++e) f(e, mass64(x[e], mp, c256, tbl), mass64(y[e], mq, c256, tbl));
        } else {
            const int gone = drop < 0 ? -1 : drop + p.off - g * E;
#pragma unroll
            for (int e = 0; e < E; ++e) f(e, mass64(e == gone ? -INFINITY : x[e], mp, c256, tbl), 0.0);
        }
    }
};

// Once over the CTA's chunks of the pair: their masses of tokens with p > q, the rows' sums, and the list if w is but near Zp / Zq.
template <int DT, bool Q>
__device__ __forceinline__ void pair_pass(VerifySmem& sm, const LastPair<DT>& l, double w, bool near) {
    constexpr int E = Traits<DT>::E;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) sm.listed = 0;
    __syncthreads();
    const unsigned listing = near ? (unsigned)VN_NEAR_BITS << 20 : 0x7FF00000u;
    double zp = 0.0, zq = 0.0;
    typename LastPair<DT>::Raw next = l.load(((l.c0 + warp) * l.R) * 32 + lane);
#pragma unroll 1
    for (int ci = l.c0 + warp; ci < l.c1; ci += VN_NW) {
        double A = 0.0, Bq = 0.0, cp = 0.0, cq = 0.0;
#pragma unroll 1
        for (int r = 0; r < l.R; ++r) {
            const int g = (ci * l.R + r) * 32 + lane;
            const typename LastPair<DT>::Raw now = next;
            next = l.load(r + 1 < l.R ? g + 32 : ((ci + VN_NW) * l.R) * 32 + lane);
            l.template each<Q>(g, now, [&](int e, double ep, double eq) {
                cp += ep;
                if constexpr (Q) {
                    cq += eq;
                    const double d = fma(-w, eq, ep);
                    const int hd = __double2hiint(d);
                    double yes = __hiloint2double(hd > 0 ? 0x3FF00000 : 0, 0);     // (a positive d that counts has a high word)
                    // |d| below 2^-VN_NEAR_BITS of ep, by exponents (2^-VN_NEAR_BITS to 2^(1 - VN_NEAR_BITS))
                    if ((unsigned)(hd & 0x7FFFFFFF) + listing <= (unsigned)__double2hiint(ep) && ep > VN_NONE) {
                        const int at = atomicAdd(&sm.listed, 1);
                        if (at < VN_LIST) { sm.list_p[at] = ep; sm.list_q[at] = eq; sm.list_j[at] = g * E + e; }
                        yes = 0.0;
                    }
                    A = fma(yes, ep, A);
                    Bq = fma(yes, eq, Bq);
                }
            });
        }
        if (!Q) A = cp;
        A = warp_sum_d(A);
        Bq = warp_sum_d(Bq);
        zp += cp;
        zq += cq;
        if (lane == 0) { sm.a[ASX_AT(ci - l.c0, VN_CHUNKS, 343)] = A; sm.b[ci - l.c0] = Bq; }
    }
    zp = warp_sum_d(zp);
    zq = warp_sum_d(zq);
    if (lane == 0) { sm.warp_pair[warp].zp = zp; sm.warp_pair[warp].zq = zq; }
    __syncthreads();
    if (threadIdx.x == 0) {
        PairSum t = {0.0, 0.0, sm.listed, 0};
        for (int i = 0; i < VN_NW; ++i) { t.zp += sm.warp_pair[i].zp; t.zq += sm.warp_pair[i].zq; }
        sm.part = t;
    }
}

template <int DT>
__global__ void __launch_bounds__(VN_NT, 3) verify_lane_kernel(const __grid_constant__ VerifyArgs a, int ctas, int batch) {
    constexpr int E = Traits<DT>::E;
    extern __shared__ __align__(16) char vn_smem[];
    VerifySmem& sm = *reinterpret_cast<VerifySmem*>(vn_smem + VN_RING);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(vn_smem) + threadIdx.x * 16;
    const int tid = threadIdx.x, lane32 = tid & 31, warp = tid >> 5;
    const int rank = ctas == 1 ? 0 : (int)(blockIdx.x % ctas);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // 2^(j / 256) = 2^((j / 4) / 64) 2^((j mod 4) / 256)
    sm.exp_tbl[tid] = ASX_T64[tid >> 2] * (tid & 2 ? 0x1.0163da9fb3335p+0 : 1.0) * (tid & 1 ? 0x1.00b1afa5abcbfp+0 : 1.0);
    __syncthreads();
    const double c256 = 256.0 * 1.4426950408889634 * a.inv_tau;
    const float c = (float)(1.4426950408889634 * a.inv_tau);
#pragma unroll 1
    for (int lane = blockIdx.x / ctas; lane < a.lanes; lane += gridDim.x / ctas) {
        const int n = drafts_of(a, lane);
        const double c_in = a.codes[lane];
        int at = max(n, 0), status = n < 0 ? AS_ERR_INVALID_ARG : !(c_in >= 0.0 && c_in <= 1.0) ? AS_ERR_NUMERIC : AS_OK;
        bool refused = false, exact = false;
        RowSum rp = {1.0, 0.f, 0}, rq = {1.0, 0.f, 0};
        // (a bad code ends the lane whatever its rows hold; but rows' errors and drafted tokens' come first where both are there)
        int i0 = 0;
        bool done = n < 0;
#pragma unroll 1
        while (!done) {
            const int count = min(batch, n + 1 - i0);
            // (what the decisions need, on its way while the rows are summed)
            int x = -1;
            double u = 0.0;
            float lp = 0.f, lq = 0.f;
            if (tid < count && i0 + tid < n) {
                x = a.drafted[(size_t)lane * a.K + i0 + tid];
                u = a.u[(size_t)lane * a.K + i0 + tid];
                if (x >= 0 && x < a.V) {
                    lp = Pass<DT>::load_f(target_row(a, lane, i0 + tid), x);
                    if (a.draft) lq = Pass<DT>::load_f(draft_row(a, lane, i0 + tid), x);
                }
            }
#pragma unroll 1
            for (int b = 0; b < count; ++b) {
                row_sum<DT>(target_row(a, lane, i0 + b), a.V, c, rank, ctas, ring, sm.warp[2 * b]);
                if (a.draft && i0 + b < n) row_sum<DT>(draft_row(a, lane, i0 + b), a.V, c, rank, ctas, ring, sm.warp[2 * b + 1]);
            }
            __syncthreads();
            if (tid < 2 * count && (tid % 2 == 0 || (a.draft && i0 + tid / 2 < n))) {
                RowSum r = sm.warp[tid][0];
                for (int i = 1; i < VN_NW; ++i) r = join_sums(r, sm.warp[tid][i], c);
                sm.mine[tid] = r;
            }
            cluster_sync(ctas);
            if (tid < 2 * VN_BATCH * VN_MAX_CTAS) {     // eight threads to a row, one to a CTA's part
                const int row = tid / VN_MAX_CTAS, k = tid % VN_MAX_CTAS;
                const bool there = row < 2 * count && (row % 2 == 0 || (a.draft && i0 + row / 2 < n));
                RowSum r = {0.0, -INFINITY, 0};
                if (there && k < ctas) r = peer(sm.mine[row], k, ctas);
#pragma unroll
                for (int o = 1; o < VN_MAX_CTAS; o <<= 1) {
                    RowSum other;
                    other.s = __shfl_xor_sync(FULL, r.s, o);
                    other.m = __shfl_xor_sync(FULL, r.m, o);
                    other.bad = __shfl_xor_sync(FULL, r.bad, o);
                    r = join_sums(r, other, c);
                }
                if (k == 0) sm.row[row] = there ? r : RowSum{1.0, 0.f, 0};
            }
            __syncthreads();
            if (warp == 0) {
                // a thread to a place
                int what = 0;
                RowSum p = {1.0, 0.f, 0}, q = {1.0, 0.f, 0};
                const int i = i0 + lane32;
                if (lane32 < count) {
                    p = sm.row[2 * lane32];
                    q = sm.row[2 * lane32 + 1];
                    // 0 accepted, 1 refused, 2 too near, 3 the last place; else an error
                    const bool p_bad = p.bad || p.m == -INFINITY, q_bad = q.bad || q.m == -INFINITY;
                    if (i == n) {
                        what = p_bad ? AS_ERR_NUMERIC : 3;
                    } else {
                        if (x < 0 || x >= a.V) {
                            what = AS_ERR_INVALID_ARG;
                        } else if (!(u >= 0.0 && u < 1.0) || p_bad || q_bad) {
                            what = AS_ERR_NUMERIC;
                        } else {
                            const double ep = token_mass(lp, MassRow(p.m, c256), c256, sm.exp_tbl);
                            const double eq = u * (a.draft ? token_mass(lq, MassRow(q.m, c256), c256, sm.exp_tbl) : 1.0);
                            // (a side that is 0 is so whatever the sums; a row too far out for sums in 32 bits has none)
                            const bool far = fabsf(p.m) * c > VN_FAR || (a.draft && fabsf(q.m) * c > VN_FAR);
                            const double px = ep / p.s, qx = eq / q.s;
                            what = ep == 0.0 ? 1 : eq == 0.0 ? 0 : far || fabs(qx - px) <= VN_NEAR * fmax(qx, px) ? 2 : qx < px ? 0 : 1;
                        }
                    }
                }
                const unsigned stop = __ballot_sync(FULL, what != 0);
                const int l = stop ? __ffs(stop) - 1 : 0;
                what = stop ? __shfl_sync(FULL, what, l) : 0;
                if (lane32 == 0) { sm.at = l; sm.status = what; }
            }
            __syncthreads();
            const int what = sm.status, l = sm.at;
            rp = sm.row[2 * l];
            rq = sm.row[2 * l + 1];
            if (what == 0) {
                i0 += count;
            } else if (what == 2) {         // once more in 64 bits
                const int i = i0 + l;
                const LastPair<DT> pair(a, target_row(a, lane, i), a.draft ? draft_row(a, lane, i) : nullptr, rp.m, rq.m, -1, c256, rank, ctas, sm.exp_tbl);
                cluster_sync(ctas);         // (the other CTAs have read this one's sums)
                if (a.draft) pair_pass<DT, true>(sm, pair, 0.0, false);
                else pair_pass<DT, false>(sm, pair, 0.0, false);
                cluster_sync(ctas);
                const double zp = cluster_total(sm.part.zp, ctas), zq = cluster_total(sm.part.zq, ctas);
                const int x = a.drafted[(size_t)lane * a.K + i];
                const double px = token_mass(Pass<DT>::load_f(target_row(a, lane, i), x), pair.mp, c256, sm.exp_tbl) / zp;
                const double qx = a.draft ? token_mass(Pass<DT>::load_f(draft_row(a, lane, i), x), pair.mq, c256, sm.exp_tbl) / zq : 1.0;
                if (a.u[(size_t)lane * a.K + i] * qx < px) {
                    i0 = i + 1;
                } else {
                    at = i;
                    refused = done = exact = true;
                    rp.s = zp;
                    rq.s = zq;
                }
            } else {
                at = i0 + l;
                refused = what == 1;
                if (what < 0) status = status == AS_ERR_INVALID_ARG ? status : what;
                done = true;
            }
            cluster_sync(ctas);             // (sums that others read are written anew)
        }

        int token = -1;
        double code = c_in;
        if (status == AS_OK) {
            const bool pairs = refused && a.draft;
            const int drop = refused && !a.draft ? a.drafted[(size_t)lane * a.K + at] : -1;
            LastPair<DT> l(a, target_row(a, lane, at), pairs ? draft_row(a, lane, at) : nullptr, rp.m, rq.m, drop, c256, rank, ctas, sm.exp_tbl);
            bool vague = false;
            double w = pairs ? rp.s / rq.s : 0.0, ratio = 0.0, total = 0.0;
            // (w from sums in 32 bits; a row too far out for those has one of 0)
            bool near = pairs && !exact;
            if (near && (fabsf(rp.m) * c > VN_FAR || fabsf(rq.m) * c > VN_FAR)) { w = 1.0; near = false; vague = true; }
            // Once; again with the exact w if the list ran over; once more with p alone where nothing is left of p - q.
#pragma unroll 1
            for (int turn = 0; turn < 3; ++turn) {
                if (l.q) pair_pass<DT, true>(sm, l, w, near);
                else pair_pass<DT, false>(sm, l, w, near);
                cluster_sync(ctas);
                const double zp = cluster_total(sm.part.zp, ctas), zq = cluster_total(sm.part.zq, ctas);
                const int most = ctas == 1 ? sm.part.listed : __reduce_max_sync(FULL, lane32 < ctas ? peer(sm.part.listed, lane32, ctas) : 0);
                ratio = l.q ? zp / zq : 0.0;
                if (most > VN_LIST || vague) {
                    cluster_sync(ctas);
                    w = ratio;
                    near = vague = false;
                    continue;
                }
                // ---- chunks' masses of max(p - q, 0) in units of 1 / Zp; listed tokens in the order of their indices ----
                const int chunks = l.c1 - l.c0, listed = near ? sm.listed : 0;
                // (a chunk that comes out above 0 has a token that does: of those in its sum one is above VN_NONE, and all of them have
                // p > q by w, which is Zp / Zq or so near to it that those listed apart are the only ones for which it matters)
                for (int i = tid; i < chunks; i += VN_NT) sm.a[i] = sm.a[i] > VN_SOME ? fmax(fma(-ratio, sm.b[i], sm.a[i]), 0.0) : 0.0;
                for (int i = tid; i < listed; i += VN_NT) {
                    int before = 0;
                    for (int k = 0; k < listed; ++k) before += sm.list_j[k] < sm.list_j[i];
                    sm.order[ASX_AT(before, VN_LIST, 344)] = i;
                }
                __syncthreads();
                const int width = 32 * l.R * E;
                for (int i = tid; i < listed; i += VN_NT) {
                    const int mine = sm.list_j[sm.order[i]] / width;
                    if (i > 0 && sm.list_j[sm.order[i - 1]] / width == mine) continue;
                    double more = 0.0;
                    for (int k = i; k < listed && sm.list_j[sm.order[k]] / width == mine; ++k)
                        more += fmax(fma(-ratio, sm.list_q[sm.order[k]], sm.list_p[sm.order[k]]), 0.0);
                    sm.a[ASX_AT(mine - l.c0, VN_CHUNKS, 345)] += more;
                }
                __syncthreads();
                if (warp == 0) {            // exclusive sums in place of b
                    double run = 0.0;
                    for (int i = 0; i < chunks; i += 32) {
                        const double v = i + lane32 < chunks ? sm.a[i + lane32] : 0.0;
                        const double incl = warp_incl_scan_d(v, lane32);
                        double before = __shfl_up_sync(FULL, incl, 1);
                        if (lane32 == 0) before = 0.0;
                        if (i + lane32 < chunks) sm.b[i + lane32] = run + before;
                        run += __shfl_sync(FULL, incl, 31);
                    }
                    if (lane32 == 0) sm.rest = run;
                }
                cluster_sync(ctas);
                total = cluster_total(sm.rest, ctas);
                if (total > VN_NONE) break;
                cluster_sync(ctas);
                l.q = nullptr;              // p and q are alike in 64 bits
                l.drop = -1;
                w = 0.0;
                near = false;
            }
            const double t = (c_in == 1.0 ? ASX_ONE_BELOW : c_in) * total;
            // ---- the CTA, the chunk, the sub-row and the token whose interval holds t ----
            int owner = 0;
            double own_base = 0.0;
            bool top = !(t < sm.rest);          // (one CTA) rounding at the top end: the last token
            if (ctas > 1) {
                const double r = of_cluster(sm.rest, ctas), upto = warp_incl_scan_d(r, lane32);
                double before = __shfl_up_sync(FULL, upto, 1);
                if (lane32 == 0) before = 0.0;
                const unsigned has = __ballot_sync(FULL, r > 0.0), hit = __ballot_sync(FULL, r > 0.0 && t < upto);
                top = hit == 0;
                owner = hit ? __ffs(hit) - 1 : 31 - __clz(has);
                own_base = __shfl_sync(FULL, before, owner);
            }
            if (owner == rank) {
                const int chunks = l.c1 - l.c0;
                if (warp == 0) {
                    int pick = -1, end = -1;
                    for (int i = 0; i < chunks && pick < 0; i += 32) {
                        const bool has = i + lane32 < chunks && sm.a[i + lane32] > 0.0;
                        const unsigned bal = __ballot_sync(FULL, has), hit = __ballot_sync(FULL, has && !top && t < own_base + (sm.b[has ? i + lane32 : 0] + sm.a[has ? i + lane32 : 0]));
                        if (bal) end = i + 31 - __clz(bal);
                        if (hit) pick = i + __ffs(hit) - 1;
                    }
                    if (lane32 == 0) { sm.chunk = max(pick < 0 ? end : pick, 0); sm.force_last = top || pick < 0; }
                }
                __syncthreads();
                const int ci = sm.chunk + l.c0;
                const bool force = sm.force_last;
                const double start = own_base + sm.b[ASX_AT(sm.chunk, VN_CHUNKS, 346)];
                auto rest = [&](int r, double (&ev)[E]) {
                    const int g = (ci * l.R + r) * 32 + lane32;
                    auto take = [&](int e, double ep, double eq) {
                        const double d = fma(-ratio, eq, ep);
                        ev[e] = ep > VN_NONE && d > 0.0 ? d : 0.0;
                    };
                    if (l.q) l.template each<true>(g, l.load(g), take);
                    else l.template each<false>(g, l.load(g), take);
                };
                // sub-rows' sums, VN_NW at a time
                double run = start;
                int sub = -1, sub_end = -1;
                double sub_start = 0.0, end_start = 0.0;
                for (int r0 = 0; r0 < l.R && sub < 0; r0 += VN_NW) {
                    double local = 0.0;
                    if (r0 + warp < l.R) {
                        double ev[E];
                        rest(r0 + warp, ev);
#pragma unroll
                        for (int e = 0; e < E; ++e) local += ev[e];
                    }
                    local = warp_sum_d(local);
                    if (lane32 == 0) sm.sub[warp] = local;
                    __syncthreads();
                    for (int i = 0; i < VN_NW && r0 + i < l.R; ++i) {
                        const double v = sm.sub[i];
                        if (v > 0.0) {
                            if (sub < 0 && !force && t < run + v) { sub = r0 + i; sub_start = run; }
                            sub_end = r0 + i;
                            end_start = run;
                        }
                        run += v;
                    }
                    __syncthreads();
                }
                const bool force_sub = sub < 0;
                if (force_sub) { sub = max(sub_end, 0); sub_start = end_start; }    // (whatever the sums say, nothing in front of the chunk is read)
                if (warp == 0) {
                    double ev[E], local = 0.0;
                    rest(sub, ev);
#pragma unroll
                    for (int e = 0; e < E; ++e) local += ev[e];
                    const double incl = warp_incl_scan_d(local, lane32);
                    double S = __shfl_up_sync(FULL, incl, 1);
                    S = sub_start + (lane32 == 0 ? 0.0 : S);
                    const int j0 = ((ci * l.R + sub) * 32 + lane32) * E - l.p.off;
                    int mine = -1, mine_last = -1;
                    double mine_S = 0.0, mine_e = 1.0, last_S = 0.0, last_e = 1.0;
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (ev[e] > 0.0) {
                            if (mine < 0 && t < S + ev[e]) { mine = j0 + e; mine_S = S; mine_e = ev[e]; }
                            mine_last = j0 + e; last_S = S; last_e = ev[e];
                            S += ev[e];
                        }
                    const unsigned has = __ballot_sync(FULL, local > 0.0), hit = __ballot_sync(FULL, !force_sub && local > 0.0 && t < sub_start + incl);
                    const int who = hit ? __ffs(hit) - 1 : 31 - __clz(has);
                    if (!hit || mine < 0) { mine = mine_last; mine_S = last_S; mine_e = last_e; }
                    token = __shfl_sync(FULL, mine, who);
                    mine_S = __shfl_sync(FULL, mine_S, who);
                    mine_e = __shfl_sync(FULL, mine_e, who);
                    code = (t - mine_S) / mine_e;
                    if (!(code >= 0.0)) code = 0.0;
                    if (code > ASX_ONE_BELOW) code = ASX_ONE_BELOW;
                }
            }
            if (owner == rank && tid == 0) {
                a.tokens[(size_t)lane * (a.K + 1) + at] = token;
                a.codes_out[lane] = code;
            }
        }
        if (rank == 0) {
            const bool good = status == AS_OK;
            int* out = a.tokens + (size_t)lane * (a.K + 1);
            for (int i = tid; i <= a.K; i += VN_NT)
                if (!good || i != at) out[i] = good && i < at ? a.drafted[(size_t)lane * a.K + i] : -1;
            if (tid == 0) {
                a.accepted[lane] = good ? at : 0;
                if (!good) a.codes_out[lane] = c_in;
                if (a.lane_status) a.lane_status[lane] = status;
            }
        }
        cluster_sync(ctas);
    }
}

template <int DT>
static cudaError_t launch_verify_lanes(const VerifyArgs& a, int sms, cudaStream_t st) {
    static bool attr_set[64] = {false};
    int dev = 0;
    cudaGetDevice(&dev);
    auto kern = verify_lane_kernel<DT>;
    if (!attr_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, VN_SMEM);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    // CTAs to a lane: one on each SM, or as many as find room side by side, three on an SM, if a row has a step for each
    // (bf16, 120 x 4 x 128256: 3 of them 127 us, 1 of them 184; 150 x 5 x 25391: 70 us with 2, 80 with 1; 150 x 4 x 4000: 32 us with 1, 37 with 2;
    // 4 x 3 x 8000: 25 us with 8, 28 with 1)
    const long long steps = ((long long)a.V * Traits<DT>::BYTES + VN_U * VN_NT * 16 - 1) / (VN_U * VN_NT * 16), room = 3LL * sms / a.lanes;
    long long wanted = sms / a.lanes;
    if (wanted < (steps < room ? steps : room)) wanted = steps < room ? steps : room;
    const int ctas = (int)(wanted < 1 ? 1 : wanted > VN_MAX_CTAS ? VN_MAX_CTAS : wanted);
    // Places whose rows are read before their decisions: a meeting costs about what a CTA's step does.  Rows of one step, four (30 x 5 x 32000: 36 us,
    // 37 with two, 40 with eight; 759 x 8 x 2010: 87 us, 91 with one); longer ones, two if a cluster has to meet (1 x 7 x 127484: 34 us, 53
    // with eight; 4 x 3 x 32000: 26 us, 30 with one), else one (500 x 8 x 50257 in 32 bits: 327 us, 333 with two).
    const int batch = steps <= ctas ? VN_BATCH : ctas > 1 ? 2 : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.lanes < 64 * sms ? a.lanes : 64 * sms) * ctas));
    cfg.blockDim = dim3(VN_NT);
    cfg.dynamicSmemBytes = VN_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)ctas, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a, ctas, batch);
}

template <int DT>
static cudaError_t launch_verify(const VerifyArgs& a, int sms, cudaStream_t st) {
    // (temperatures whose reciprocals come near a float's range, next to which -inf and the lowest float are no masks any more, take the general routine)
    const bool tame = a.inv_tau >= 1e-30 && a.inv_tau <= 1e30;
    if (tame && (a.top_k <= 0 || a.top_k >= a.V) && !(a.top_p > 0.0 && a.top_p < 1.0)) return launch_verify_lanes<DT>(a, sms, st);
    const unsigned rows = (unsigned)((long long)a.lanes * (a.draft ? 2 * a.K + 1 : a.K + 1));
    // A CTA of either kernel has 1024 threads where each finds an SM of its own and the row has 16 bytes for more than 512 of them, else 512.
    // us with 1024 / 512 threads in the one kernel, the other as it is, logits of spread 2.  Rows: 5 x 2 x 38634, both cuts, 127 / 162 in 32 bits and 114 / 136
    // in bf16, 20 x 3 x 50257 in bf16, nucleus, 179 / 194; more rows than SMs, nucleus: 41 x 3 x 2836 in 32 bits 89 / 55, 200 x 2 x 32000 in bf16 435 / 355,
    // 96 x 5 x 50257 in 32 bits 632 / 627; a short row, 1 x 5 x 742: 47 / 38.  Tokens: 96 x 5 x 50257 627 / 667, 20 x 3 x 50257 179 / 219, 140 x 2 x 32000
    // 271 / 295, 41 x 3 x 2836 55 / 57; more lanes than SMs, 200 x 2 x 32000: 351 / 355.
    const bool wide = (long long)a.V * Traits<DT>::BYTES > 512 * 16;
    cudaError_t e = cudaMemsetAsync(a.stop, 0, sizeof(int) * (size_t)a.lanes * (a.K + 1), st);
    if (e == cudaSuccess) e = wide && rows <= (unsigned)sms ? launch_after(verify_rows_kernel<DT, 1024>, rows, 1024, 0, st, a) : launch_after(verify_rows_kernel<DT, 512>, rows, 512, 0, st, a);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)(a.lanes < 64 * sms ? a.lanes : 64 * sms);
    return wide && a.lanes <= sms ? launch_after(verify_finish_kernel<DT, 1024>, grid, 1024, 0, st, a) : launch_after(verify_finish_kernel<DT, 512>, grid, 512, 0, st, a);
}

}  // namespace asx

using namespace asx;

extern "C" {

size_t as_step_verify_work_bytes(int dtype, int lanes, int K, int V) {
    if (lanes < 1 || K < 0 || V < 1 || V > AS_MAX_V || (dtype != AS_F32 && dtype != AS_BF16)) return 0;
    if ((long long)lanes * (2LL * K + 1) > 0x7FFFFFFFLL) return 0;
    return sizeof(RowCut) * (size_t)lanes * (2 * (size_t)K + 1) + sizeof(int) * (size_t)lanes * (K + 1);
}

int as_step_verify(const void* d_target, long long target_ld, const void* d_draft, long long draft_ld, int dtype, int lanes, int K, int V,
                   const int32_t* d_drafted, const int32_t* d_n, const double* d_u, const double* d_codes, double temp, int top_k,
                   double top_p, int32_t* d_tokens, int32_t* d_accepted, double* d_codes_out, int32_t* d_lane_status, void* d_work,
                   size_t work_bytes, void* stream) {
    if (lanes < 0) return set_err(AS_ERR_INVALID_ARG, "lanes = %d must be >= 0", lanes);
    if (K < 0) return set_err(AS_ERR_INVALID_ARG, "K = %d must be >= 0", K);
    int rc = check_scalars(dtype, V, target_ld, temp, top_p);
    if (rc != AS_OK) return rc;
    const bool drafter = d_draft && K > 0;
    if (drafter && draft_ld < V) return set_err(AS_ERR_INVALID_ARG, "draft_ld = %lld is smaller than V = %d", draft_ld, V);
    if ((long long)lanes * (2LL * K + 1) > 0x7FFFFFFFLL) return set_err(AS_ERR_UNSUPPORTED, "lanes * (2 K + 1) rows must be below 2^31");
    if (lanes == 0) return AS_OK;
    if ((rc = check_data(d_target, dtype)) != AS_OK) return rc;
    if (drafter && (rc = check_data(d_draft, dtype)) != AS_OK) return rc;
    if (!d_codes || !d_tokens || !d_accepted || !d_codes_out || (K > 0 && (!d_drafted || !d_u)))
        return set_err(AS_ERR_INVALID_ARG, "d_drafted, d_u, d_codes, d_tokens, d_accepted or d_codes_out is NULL");
    const size_t need = as_step_verify_work_bytes(dtype, lanes, K, V);
    if (!d_work || work_bytes < need) return set_err(AS_ERR_INVALID_ARG, "d_work of %zu bytes is needed", need);
    if (reinterpret_cast<uintptr_t>(d_work) & 255) return set_err(AS_ERR_INVALID_ARG, "d_work is not 256-byte aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    const int es = dtype == AS_F32 ? 4 : 2;
    VerifyArgs a;
    a.target = static_cast<const char*>(d_target); a.draft = drafter ? static_cast<const char*>(d_draft) : nullptr;
    a.target_ld = target_ld * es; a.draft_ld = draft_ld * es;
    a.lanes = lanes; a.K = K; a.V = V;
    a.drafted = d_drafted; a.n = d_n; a.u = d_u; a.codes = d_codes;
    a.inv_tau = temp < 1e-300 ? 1e300 : 1.0 / temp;         // (finite: it is multiplied by differences of 0)
    a.top_p = top_p; a.top_k = top_k;
    a.tokens = d_tokens; a.accepted = d_accepted; a.codes_out = d_codes_out; a.lane_status = d_lane_status;
    a.cuts = static_cast<RowCut*>(d_work);
    a.stop = reinterpret_cast<int*>(a.cuts + (size_t)lanes * (2 * (size_t)K + 1));
    a.arrived = a.stop + lanes;
    const cudaError_t e = dtype == AS_F32 ? launch_verify<AS_F32>(a, di->sms, (cudaStream_t)stream) : launch_verify<AS_BF16>(a, di->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "verify kernel launch");
}

}  // extern "C"
