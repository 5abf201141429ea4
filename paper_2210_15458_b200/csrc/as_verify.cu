// The step over drafted tokens: which of them are accepted, and the token behind them.
#include "../../include/arith_sampling.h"
#include "as_generic.cuh"
#include "as_host.h"

namespace asx {

ASX_BOUNDS_READER(bounds_verify)

constexpr int VF_NT = 512;

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

// A CTA to a row: its kept tokens and their mass, by the general routine of the step.
template <int DT>
__global__ void __launch_bounds__(VF_NT) verify_rows_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ GenericSmem<VF_NT> sm;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // rows in the order of the places, the target's and the draft's of a place side by side
    const int per = a.draft ? 2 : 1, block = blockIdx.x / a.lanes, lane = blockIdx.x - block * a.lanes;
    const int i = block / per;
    const bool of_draft = block % per;
    if (i > drafts_of(a, lane) - (of_draft ? 1 : 0)) return;
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
    if (threadIdx.x == 0) *cut_of(a, lane, i, of_draft) = c;
}

template <int DT>
struct RowMass {
    using Tr = Traits<DT>;
    const char* row;
    bool vec;
    RowCut c;
    __device__ RowMass(const char* r, const RowCut* cut) : row(r), vec((reinterpret_cast<uintptr_t>(r) & 15) == 0), c(*cut) {}
    __device__ __forceinline__ double operator()(uint32_t key, int j, double inv_tau, const double* tbl) const {
        return key > c.T || (key == c.T && j <= c.tie) ? exp_nonpos(((double)Tr::value_f(key) - c.lmax) * inv_tau, tbl) : 0.0;
    }
};

// One CTA per lane: how many of its tokens are accepted, and the token behind them by its code, over masses
// max(p - q Zp / Zq, 0) in units of 1 / Zp: sums of chunks in index order, the chunk that holds the code, the token in it.
template <int DT>
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
                if (i < n) {
                    const int x = a.drafted[(size_t)lane * a.K + i];
                    const double u = a.u[(size_t)lane * a.K + i];
                    const RowMass<DT> p(target_row(a, lane, i), cut_of(a, lane, i, false));
                    if (x < 0 || x >= a.V) {
                        what = AS_ERR_INVALID_ARG;
                    } else if (!(u >= 0.0 && u < 1.0) || p.c.status != ST_OK) {
                        what = AS_ERR_NUMERIC;
                    } else {
                        const double px = p(Tr::load_key(p.row, x), x, a.inv_tau, sm.exp_tbl) / p.c.Z;
                        double qx = 1.0;
                        if (a.draft) {
                            const RowMass<DT> q(draft_row(a, lane, i), cut_of(a, lane, i, true));
                            if (q.c.status != ST_OK) what = AS_ERR_NUMERIC;
                            else qx = q(Tr::load_key(q.row, x), x, a.inv_tau, sm.exp_tbl) / q.c.Z;
                        }
                        if (what == 0) what = u * qx < px ? 0 : 1;
                    }
                }
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

template <int DT>
static cudaError_t launch_verify(const VerifyArgs& a, int sms, cudaStream_t st) {
    const unsigned rows = (unsigned)((long long)a.lanes * (a.draft ? 2 * a.K + 1 : a.K + 1));
    cudaError_t e = launch_after(verify_rows_kernel<DT>, rows, VF_NT, 0, st, a);
    if (e != cudaSuccess) return e;
    return launch_after(verify_finish_kernel<DT>, (unsigned)(a.lanes < 64 * sms ? a.lanes : 64 * sms), VF_NT, 0, st, a);
}

}  // namespace asx

using namespace asx;

extern "C" {

size_t as_step_verify_work_bytes(int dtype, int lanes, int K, int V) {
    if (lanes < 1 || K < 0 || V < 1 || V > AS_MAX_V || (dtype != AS_F32 && dtype != AS_BF16)) return 0;
    if ((long long)lanes * (2LL * K + 1) > 0x7FFFFFFFLL) return 0;
    return sizeof(RowCut) * (size_t)lanes * (2 * (size_t)K + 1);
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
    a.inv_tau = 1.0 / temp; a.top_p = top_p; a.top_k = top_k;
    a.tokens = d_tokens; a.accepted = d_accepted; a.codes_out = d_codes_out; a.lane_status = d_lane_status;
    a.cuts = static_cast<RowCut*>(d_work);
    const cudaError_t e = dtype == AS_F32 ? launch_verify<AS_F32>(a, di->sms, (cudaStream_t)stream) : launch_verify<AS_BF16>(a, di->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "verify kernel launch");
}

}  // extern "C"
