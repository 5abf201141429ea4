// Logit edits: penalties for repeated tokens, bias and grammar mask in one pass over the rows.
#include "../../include/arith_sampling.h"
#include "as_bounds.cuh"
#include "as_host.h"

#include <cmath>
#include <cuda_bf16.h>

namespace asx {

ASX_BOUNDS_READER(bounds_edit)

constexpr int ED_NT = 256;
constexpr int ED_CHUNK = 8192;          // tokens of a row that one CTA edits

struct EditArgs {
    const char* in;
    char* out;
    long long ld, out_ld;               // elements
    const int* seq;
    long long seq_ld;
    const int* len;
    const int* prompt_len;
    float repetition, presence, frequency;
    const float* bias;
    long long bias_ld;
    const uint32_t* mask;
    long long mask_ld;
    int mask_rows;
    const int* mask_row;
    int* lane_status;
    int lanes, V, chunks;
    bool same_grid;                     // rows of d_logits and d_out start at the same place of their 16-byte granules
};

template <int DT> struct Elem;
template <> struct Elem<AS_F32> {
    static constexpr int BYTES = 4, E = 4;
    __device__ static float get(const char* p) { return *reinterpret_cast<const float*>(p); }
    __device__ static void put(char* p, float x) { *reinterpret_cast<float*>(p) = x; }
    __device__ static void unpack(const uint4& q, float (&x)[4]) {
        x[0] = __uint_as_float(q.x); x[1] = __uint_as_float(q.y); x[2] = __uint_as_float(q.z); x[3] = __uint_as_float(q.w);
    }
    __device__ static uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static uint4 all_masked() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
};
template <> struct Elem<AS_BF16> {
    static constexpr int BYTES = 2, E = 8;
    __device__ static float get(const char* p) { return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); }
    __device__ static void put(char* p, float x) { *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(x); }
    __device__ static void unpack(const uint4& q, float (&x)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ static uint4 pack(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static uint4 all_masked() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
};

// The penalties of a token that the history holds, n of its occurrences in the output.  Each
// operation is rounded by itself (no fused multiply-add), as the formula is stated.
__device__ __forceinline__ float penalise(float x, uint32_t n, const EditArgs& a) {
    x = x > 0.f ? __fdiv_rn(x, a.repetition) : __fmul_rn(x, a.repetition);
    if (n) x = __fsub_rn(x, __fadd_rn(__fmul_rn(a.frequency, (float)n), a.presence));
    return x;
}

// One CTA edits one chunk of one row.  It first counts the lane's history within the chunk in
// shared memory (a bit per seen token, a count per token), then passes over the chunk once; the
// vectors of the row's own 16-byte grid decide where a chunk starts, so that any row start is served
// by 16-byte accesses.
template <int DT>
__global__ void __launch_bounds__(ED_NT) edit_kernel(const EditArgs a) {
    using El = Elem<DT>;
    constexpr int E = El::E;
    constexpr int SLOTS = ED_CHUNK + E;                 // the elements in front of the first vector, then the chunk
    __shared__ __align__(16) uint32_t count[SLOTS];
    __shared__ __align__(16) uint32_t seen[SLOTS / 32 + 1];
    const int tid = threadIdx.x;
    const long long items = (long long)a.lanes * a.chunks;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int lane = (int)(it / a.chunks), k = (int)(it % a.chunks);
        const char* in = a.in + (size_t)lane * (size_t)a.ld * El::BYTES;
        char* out = a.out + (size_t)lane * (size_t)a.out_ld * El::BYTES;
        const bool inplace = a.in == a.out;
        int lead = (int)((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / El::BYTES;
        const int vb = k * ED_CHUNK + lead;             // first vector's first token
        const int t0 = k == 0 ? 0 : vb;                 // first token of the chunk
        const int t1 = min(a.V, vb + ED_CHUNK);
        const int base = vb - E;                        // token of slot 0
        const bool has_history = a.seq != nullptr;
        bool bad = false;
        if (has_history) {
            for (int i = tid; i < SLOTS / 4; i += ED_NT) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
            for (int i = tid; i < SLOTS / 32 + 1; i += ED_NT) seen[i] = 0;
            __syncthreads();
            int n = a.len[lane], p = a.prompt_len ? a.prompt_len[lane] : 0;
            if (n < 0 || n > a.seq_ld) { bad = true; n = n < 0 ? 0 : (int)a.seq_ld; }
            const int* seq = a.seq + (size_t)lane * (size_t)a.seq_ld;
            for (int i = tid; i < n; i += ED_NT) {
                const int t = seq[i];
                if (t < 0 || t >= a.V) { bad = true; continue; }
                if (t >= t0 && t < t1) {
                    const int s = ASX_AT(t - base, SLOTS, 1);
                    atomicOr(&seen[s >> 5], 1u << (s & 31));
                    if (i >= p) atomicAdd(&count[s], 1u);
                }
            }
        }
        const uint32_t* mask = nullptr;
        if (a.mask) {
            int r = a.mask_row ? a.mask_row[lane] : (a.mask_rows == 1 ? 0 : lane);
            if (r < -1 || r >= a.mask_rows) { bad = true; r = -1; }
            if (r >= 0) mask = a.mask + (size_t)r * (size_t)a.mask_ld;
        }
        const float* bias = a.bias ? a.bias + (size_t)lane * (size_t)a.bias_ld : nullptr;
        const bool any_bad = __syncthreads_or(bad);
        if (tid == 0 && k == 0 && a.lane_status) a.lane_status[lane] = any_bad ? AS_ERR_INVALID_ARG : AS_OK;

        auto edit_one = [&](int t) {
            const int s = ASX_AT(t - base, SLOTS, 2);
            float x = El::get(in + (size_t)t * El::BYTES);
            if (has_history && (seen[s >> 5] >> (s & 31) & 1)) x = penalise(x, count[s], a);
            if (bias) x = __fadd_rn(x, bias[t]);
            if (mask && !(mask[t >> 5] >> (t & 31) & 1)) x = -INFINITY;
            El::put(out + (size_t)t * El::BYTES, x);
        };
        if (!a.same_grid) {                             // the rows lie differently: element by element
            for (int t = t0 + tid; t < t1; t += ED_NT) edit_one(t);
        } else {
            const int nvec = t1 > vb ? (t1 - vb) / E : 0;
            if (k == 0 && tid < min(vb, t1)) edit_one(tid);                     // in front of the first vector
            if (tid < t1 - (vb + nvec * E) && vb + nvec * E + tid >= t0) edit_one(vb + nvec * E + tid);  // behind the last
            for (int v = tid; v < nvec; v += ED_NT) {
                const int t = vb + v * E;
                uint32_t allow = (1u << E) - 1;
                if (mask) {
                    const int sh = t & 31;
                    allow = mask[t >> 5] >> sh;
                    if (sh + E > 32) allow |= mask[(t >> 5) + 1] << (32 - sh);
                    allow &= (1u << E) - 1;
                }
                uint4* dst = reinterpret_cast<uint4*>(out + (size_t)t * El::BYTES);
                if (allow == 0) { *dst = El::all_masked(); continue; }
                const int s = ASX_AT(E + v * E, SLOTS, 3);
                const uint32_t hit = has_history ? (seen[s >> 5] >> (s & 31)) & ((1u << E) - 1) : 0;
                const bool same = hit == 0 && !bias && allow == (1u << E) - 1;
                if (same && inplace) continue;
                uint4 q = *reinterpret_cast<const uint4*>(in + (size_t)t * El::BYTES);
                if (!same) {
                    float x[E];
                    El::unpack(q, x);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (hit >> e & 1) x[e] = penalise(x[e], count[s + e], a);
                        if (bias) x[e] = __fadd_rn(x[e], bias[t + e]);
                        if (!(allow >> e & 1)) x[e] = -INFINITY;
                    }
                    q = El::pack(x);
                }
                *dst = q;
            }
        }
        __syncthreads();
    }
}

}  // namespace asx

using namespace asx;

extern "C" int as_logits_edit(const void* d_logits, int dtype, int lanes, int V, long long ld, const as_logit_edits* e,
                              void* d_out, long long out_ld, int32_t* d_lane_status, void* stream) {
    if (dtype != AS_F32 && dtype != AS_BF16) return set_err(AS_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (lanes < 0) return set_err(AS_ERR_INVALID_ARG, "lanes = %d must be >= 0", lanes);
    if (V < 1) return set_err(AS_ERR_INVALID_ARG, "V = %d must be >= 1", V);
    if (V > AS_MAX_V) return set_err(AS_ERR_UNSUPPORTED, "V = %d exceeds AS_MAX_V = %d", V, AS_MAX_V);
    if (ld < V || out_ld < V) return set_err(AS_ERR_INVALID_ARG, "ld = %lld or out_ld = %lld is smaller than V = %d", ld, out_ld, V);
    if (!e) return set_err(AS_ERR_INVALID_ARG, "edits is NULL");
    if (!(e->repetition > 0.f) || std::isinf(e->repetition)) return set_err(AS_ERR_INVALID_ARG, "repetition must be positive and finite");
    if (!std::isfinite(e->presence) || !std::isfinite(e->frequency)) return set_err(AS_ERR_INVALID_ARG, "presence and frequency must be finite");
    if (e->d_bias && e->bias_ld != 0 && e->bias_ld < V) return set_err(AS_ERR_INVALID_ARG, "bias_ld = %lld must be 0 or >= V = %d", e->bias_ld, V);
    if (e->d_mask && e->mask_ld < (V + 31) / 32) return set_err(AS_ERR_INVALID_ARG, "mask_ld = %lld is smaller than ceil(V / 32)", e->mask_ld);
    if (e->d_mask && e->mask_rows < 1) return set_err(AS_ERR_INVALID_ARG, "mask_rows = %d must be >= 1", e->mask_rows);
    if (e->d_mask && !e->d_mask_row && e->mask_rows != 1 && e->mask_rows < lanes)
        return set_err(AS_ERR_INVALID_ARG, "mask_rows = %d: one row, a row for each lane, or d_mask_row is needed", e->mask_rows);
    if (lanes == 0) return AS_OK;
    if (!d_logits || !d_out) return set_err(AS_ERR_INVALID_ARG, "d_logits or d_out is NULL");
    if (e->d_seq && (!e->d_len || e->seq_ld < 0)) return set_err(AS_ERR_INVALID_ARG, "d_seq needs d_len and seq_ld >= 0");
    const int es = dtype == AS_F32 ? 4 : 2;
    const uintptr_t in = reinterpret_cast<uintptr_t>(d_logits), out = reinterpret_cast<uintptr_t>(d_out);
    if (in % es || out % es) return set_err(AS_ERR_INVALID_ARG, "d_logits or d_out is not element-aligned");
    if (in == out && ld != out_ld) return set_err(AS_ERR_INVALID_ARG, "in place, out_ld = %lld must be ld = %lld", out_ld, ld);
    const DeviceInfo* di;
    int rc = device_info(&di);
    if (rc != AS_OK) return rc;
    EditArgs a;
    a.in = static_cast<const char*>(d_logits); a.out = static_cast<char*>(d_out);
    a.ld = ld; a.out_ld = out_ld;
    const bool penalties = e->repetition != 1.f || e->presence != 0.f || e->frequency != 0.f;
    a.seq = penalties || d_lane_status ? e->d_seq : nullptr;
    a.seq_ld = e->seq_ld; a.len = e->d_len; a.prompt_len = e->d_prompt_len;
    a.repetition = e->repetition; a.presence = e->presence; a.frequency = e->frequency;
    a.bias = e->d_bias; a.bias_ld = e->bias_ld;
    a.mask = e->d_mask; a.mask_ld = e->mask_ld; a.mask_rows = e->mask_rows; a.mask_row = e->d_mask_row;
    a.lane_status = d_lane_status; a.lanes = lanes; a.V = V;
    a.same_grid = ((in ^ out) & 15) == 0 && ((ld - out_ld) * es) % 16 == 0;
    a.chunks = (V + ED_CHUNK - 1) / ED_CHUNK;       // a row's last chunk starts at or below its last token
    const long long items = (long long)lanes * a.chunks;
    const unsigned grid = (unsigned)(items < (1 << 30) ? items : (1 << 30));
    if (dtype == AS_F32) edit_kernel<AS_F32><<<grid, ED_NT, 0, (cudaStream_t)stream>>>(a);
    else edit_kernel<AS_BF16><<<grid, ED_NT, 0, (cudaStream_t)stream>>>(a);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return cuda_fail(err, "logit edit kernel launch");
    return AS_OK;
}
