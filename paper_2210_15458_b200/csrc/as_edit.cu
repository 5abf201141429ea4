// Logit edits: penalties for repeated tokens, bias and grammar mask in one pass over the rows.
#include "../../include/arith_sampling.h"
#include "as_bounds.cuh"
#include "as_host.h"

#include <cmath>
#include <cuda_bf16.h>

namespace asx {

ASX_BOUNDS_READER(bounds_edit)

constexpr int ED_NT = 256;

struct EditArgs {
    const char* in;
    char* out;
    long long ld, out_ld;               // elements
    const int* seq;
    long long seq_ld;
    const int* len;
    const int* prompt_len;
    float repetition, inv_repetition, presence, frequency;
    const float* bias;
    long long bias_ld;
    const uint32_t* mask;
    long long mask_ld;
    int mask_rows;
    const int* mask_row;
    int* lane_status;
    int lanes, V, chunks;
    bool same_grid;                     // rows of d_logits and d_out start at the same place of their 16-byte granules
    bool seq_vec, bias_vec;             // histories / bias rows all start on 16-byte boundaries
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

// The penalties of a token that the history holds, n of its occurrences in the output.  Dividing by the repetition
// penalty is a product with its reciprocal (at most one unit in the last place apart): an IEEE division for each element
// was most of the kernel's code, which then no longer fit the instruction cache.
__device__ __forceinline__ float penalise(float x, uint32_t n, const EditArgs& a) {
    x = __fmul_rn(x, x > 0.f ? a.inv_repetition : a.repetition);
    return n ? __fsub_rn(x, __fadd_rn(__fmul_rn(a.frequency, (float)n), a.presence)) : x;
}

// One CTA edits one chunk of one row, VPT vectors of 16 bytes a thread; the vectors of the row's own 16-byte grid
// decide where a chunk starts, so that any row start is served by 16-byte accesses.  The thread's vectors are on
// their way (those that the mask leaves anything of) while the CTA counts the lane's history within the chunk in
// shared memory: a bit per seen token, a count per token.  Bound by HBM where histories are short: each element is read and written once; the
// history is read once per chunk, from L2 (a lane's 4096 tokens are an eighth of what its chunks of 8192 move).
// 1024 x 128256 in 32 bits: 249 us (1.06 GB; 206 us without bias and mask, 157 without a history: 6.7 TB/s); 256 x 50257 bf16: 20.6 us,
// 12.6 without a history (each of a row's chunks reads and filters all of it: issue slots 65 % busy, DRAM 10 %); 8 x 32000 bf16: 5.6 us
// on the device.
template <int DT, int VPT>
__global__ void __launch_bounds__(ED_NT) edit_kernel(const __grid_constant__ EditArgs a) {
    using El = Elem<DT>;
    constexpr int E = El::E, CHUNK = ED_NT * VPT * E;
    constexpr int SLOTS = CHUNK + E;                    // the elements in front of the first vector, then the chunk
    __shared__ __align__(16) uint32_t count[SLOTS];
    __shared__ __align__(16) uint32_t seen[SLOTS / 32 + 1];
    const int tid = threadIdx.x;
    const int lane = blockIdx.x / a.chunks, k = blockIdx.x - lane * a.chunks;
    const char* in = a.in + (size_t)lane * (size_t)a.ld * El::BYTES;
    char* out = a.out + (size_t)lane * (size_t)a.out_ld * El::BYTES;
    const bool inplace = a.in == a.out;
    const int lead = (int)((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / El::BYTES;
    const int vb = k * CHUNK + lead;                    // first vector's first token
    const int t0 = k == 0 ? 0 : vb;                     // first token of the chunk
    const int t1 = min(a.V, vb + CHUNK);
    const int base = vb - E;                            // token of slot 0
    const int nvec = a.same_grid && t1 > vb ? (t1 - vb) / E : 0;
    bool bad = false;
    const uint32_t* mask = nullptr;
    if (a.mask) {
        int r = a.mask_row ? a.mask_row[lane] : (a.mask_rows == 1 ? 0 : lane);
        if (r < -1 || r >= a.mask_rows) { bad = true; r = -1; }
        if (r >= 0) mask = a.mask + (size_t)r * (size_t)a.mask_ld;
    }
    auto allowed = [&](int t) {                         // bits of the E tokens from t on
        if (!mask) return (1u << E) - 1;
        const int sh = t & 31;
        uint32_t w = __ldg(mask + (t >> 5)) >> sh;
        if (sh + E > 32) w |= __ldg(mask + (t >> 5) + 1) << (32 - sh);
        return w & ((1u << E) - 1);
    };
    uint4 q[VPT];
    uint32_t allow[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) allow[i] = tid + i * ED_NT < nvec ? allowed(vb + (tid + i * ED_NT) * E) : 0u;
    if (!inplace) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (allow[i]) q[i] = __ldcs(reinterpret_cast<const uint4*>(in + (size_t)(vb + (tid + i * ED_NT) * E) * El::BYTES));
    }
    const bool has_history = a.seq != nullptr;
    if (has_history) {
#pragma unroll 1
        for (int i = tid; i < SLOTS / 4; i += ED_NT) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
#pragma unroll 1
        for (int i = tid; i < SLOTS / 32 + 1; i += ED_NT) seen[i] = 0;
        int n = a.len[lane], p = a.prompt_len ? a.prompt_len[lane] : 0;
        if (n < 0 || n > a.seq_ld) { bad = true; n = n < 0 ? 0 : (int)a.seq_ld; }
        const int* seq = a.seq + (size_t)lane * (size_t)a.seq_ld;
        __syncthreads();
        auto note = [&](int t, int i) {
            if (t < 0 || t >= a.V) { bad = true; return; }
            if (t >= t0 && t < t1) {
                const int s = ASX_AT(t - base, SLOTS, 1);
                atomicOr(&seen[s >> 5], 1u << (s & 31));
                if (i >= p) atomicAdd(&count[s], 1u);
            }
        };
        const int n4 = a.seq_vec ? n / 4 : 0;
#pragma unroll 1
        for (int i = tid; i < n4; i += ED_NT) {
            const int4 t4 = __ldg(reinterpret_cast<const int4*>(seq) + i);
            note(t4.x, 4 * i); note(t4.y, 4 * i + 1); note(t4.z, 4 * i + 2); note(t4.w, 4 * i + 3);
        }
#pragma unroll 1
        for (int i = 4 * n4 + tid; i < n; i += ED_NT) note(seq[i], i);
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
    if (!a.same_grid) {                                 // the rows lie differently: element by element
#pragma unroll 1
        for (int t = t0 + tid; t < t1; t += ED_NT) edit_one(t);
        return;
    }
    if (k == 0 && tid < min(vb, t1)) edit_one(tid);                                     // in front of the first vector
    if (tid < t1 - (vb + nvec * E) && vb + nvec * E + tid >= t0) edit_one(vb + nvec * E + tid);     // behind the last
    const bool bias_vec = a.bias_vec && lead % 4 == 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = tid + i * ED_NT, t = vb + v * E;
        if (v >= nvec) break;
        uint4* dst = reinterpret_cast<uint4*>(out + (size_t)t * El::BYTES);
        if (allow[i] == 0) { __stcs(dst, El::all_masked()); continue; }
        const int s = ASX_AT(E + v * E, SLOTS, 3);
        const uint32_t hit = has_history ? (seen[s >> 5] >> (s & 31)) & ((1u << E) - 1) : 0;
        const bool same = hit == 0 && !bias && allow[i] == (1u << E) - 1;
        if (inplace) {
            if (same) continue;
            q[i] = *reinterpret_cast<const uint4*>(in + (size_t)t * El::BYTES);
        }
        if (!same) {
            float x[E];
            El::unpack(q[i], x);
            if (hit) {
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const uint4 n = *reinterpret_cast<const uint4*>(&count[s + e]);
                    if (hit >> e & 1) x[e] = penalise(x[e], n.x, a);
                    if (hit >> e & 2) x[e + 1] = penalise(x[e + 1], n.y, a);
                    if (hit >> e & 4) x[e + 2] = penalise(x[e + 2], n.z, a);
                    if (hit >> e & 8) x[e + 3] = penalise(x[e + 3], n.w, a);
                }
            }
            if (bias) {
                if (bias_vec) {
#pragma unroll
                    for (int e = 0; e < E; e += 4) {
                        const float4 b4 = __ldg(reinterpret_cast<const float4*>(bias + t + e));
                        x[e] = __fadd_rn(x[e], b4.x); x[e + 1] = __fadd_rn(x[e + 1], b4.y);
                        x[e + 2] = __fadd_rn(x[e + 2], b4.z); x[e + 3] = __fadd_rn(x[e + 3], b4.w);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = __fadd_rn(x[e], __ldg(bias + t + e));
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (!(allow[i] >> e & 1)) x[e] = -INFINITY;
            q[i] = El::pack(x);
        }
        __stcs(dst, q[i]);
    }
}

template <int DT, int VPT>
static cudaError_t launch_edit(EditArgs& a, cudaStream_t st) {
    constexpr int CHUNK = ED_NT * VPT * Elem<DT>::E;
    a.chunks = (a.V + CHUNK - 1) / CHUNK;           // a row's last chunk starts at or below its last token
    edit_kernel<DT, VPT><<<(unsigned)((long long)a.lanes * a.chunks), ED_NT, 0, st>>>(a);
    return cudaGetLastError();
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
    if ((long long)lanes * ((V + 8191) / 8192) > 0x7FFFFFFFLL) return set_err(AS_ERR_UNSUPPORTED, "lanes = %d and V = %d make more than 2^31 chunks", lanes, V);
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
    a.repetition = e->repetition; a.inv_repetition = 1.f / e->repetition; a.presence = e->presence; a.frequency = e->frequency;
    a.bias = e->d_bias; a.bias_ld = e->bias_ld;
    a.mask = e->d_mask; a.mask_ld = e->mask_ld; a.mask_rows = e->mask_rows; a.mask_row = e->d_mask_row;
    a.lane_status = d_lane_status; a.lanes = lanes; a.V = V;
    a.same_grid = ((in ^ out) & 15) == 0 && ((ld - out_ld) * es) % 16 == 0;
    a.seq_vec = ((reinterpret_cast<uintptr_t>(e->d_seq) | (uintptr_t)(e->seq_ld * 4)) & 15) == 0;
    a.bias_vec = ((reinterpret_cast<uintptr_t>(e->d_bias) | (uintptr_t)(e->bias_ld * 4)) & 15) == 0;
    // Chunks of 8192 tokens, or of 2048 where those would not fill the SMs twice (50257 bf16, large / small chunks, us: 256 lanes
    // 22.4 / 27.0, 128 lanes 16.9 / 17.4; from 64 lanes down the host's call hides the difference)
    const cudaStream_t st = (cudaStream_t)stream;
    const bool large = (long long)lanes * ((V + 8191) / 8192) >= 2 * di->sms;
    if (in == out && !a.seq && !a.bias && !a.mask && !d_lane_status) return AS_OK;
    cudaError_t err;
    if (dtype == AS_F32) err = large ? launch_edit<AS_F32, 8>(a, st) : launch_edit<AS_F32, 2>(a, st);
    else err = large ? launch_edit<AS_BF16, 4>(a, st) : launch_edit<AS_BF16, 1>(a, st);
    if (err != cudaSuccess) return cuda_fail(err, "logit edit kernel launch");
    return AS_OK;
}
