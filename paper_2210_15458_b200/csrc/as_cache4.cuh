// The 4-bit cache: its layout, storing into it and reading it back.
#pragma once
#include "../../include/arith_sampling.h"
#include "as_bounds.cuh"
#include "as_host.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace asx {

// A tile: 16 tokens of one head (see as_cache4 in the header).
template <int D> struct Tile4 {
    static constexpr int NB = D / 16;               // blocks of 16 dimensions, one scale each
    static constexpr int K = 0, V = 8 * D, KS = 16 * D, VS = 17 * D, BYTES = 18 * D;
    __device__ static int k_code(int t, int b) { return K + t * (D / 2) + b * 8; }
    __device__ static int v_code(int t, int b) { return V + b * 128 + t * 8; }
    __device__ static int k_scale(int t, int b) { return KS + t * NB + b; }
    __device__ static int v_scale(int t, int b) { return VS + b * 16 + t; }
};

struct CacheArgs {
    char* pages;
    int n_pages, heads, page_shift;                 // page size = 1 << page_shift tokens
    const float *k_scale, *v_scale;
    const int* table;
    int max_pages;
    const int* len;
    int* lane_status;
    int lanes, T;
};

// e4m3 bits -> value
__device__ __forceinline__ float e4m3_value(uint32_t b) {
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((unsigned short)b));
    return __half2float(__ushort_as_half((unsigned short)h2));
}
// two values -> two e4m3 bytes (a in the low byte), nearest, saturating
__device__ __forceinline__ uint32_t to_e4m3(float a) {
    unsigned short d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(0.f), "f"(a));
    return d & 0xFFu;
}
// two values -> two codes in a byte (lo in the low half), nearest (half way: even), saturating
__device__ __forceinline__ uint32_t to_codes(float lo, float hi) {
    uint32_t d;
    asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tcvt.u32.u8 %0, b;\n\t}" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// a byte of two codes -> two f16 (the low half of the byte in the low half of the result)
__device__ __forceinline__ uint32_t codes_f16x2(uint32_t byte) {
    uint32_t d;
    asm("{\n\t.reg .b8 b;\n\tcvt.u8.u32 b, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(d) : "r"(byte));
    return d;
}

// the four bytes of a word at once (the conversion picks its byte itself: no shifts)
__device__ __forceinline__ void codes_f16x2(uint32_t word, uint32_t (&d)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}" : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "r"(word));
}

template <int DT> struct Io;
template <> struct Io<AS_F32> {
    using type = float;
    __device__ static void read16(const float* p, bool vec, float (&x)[16]) {
        if (vec) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 q = reinterpret_cast<const float4*>(p)[i];
                x[4 * i] = q.x; x[4 * i + 1] = q.y; x[4 * i + 2] = q.z; x[4 * i + 3] = q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = p[i];
        }
    }
    __device__ static void write16(float* p, const float (&x)[16]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
};
template <> struct Io<AS_BF16> {
    using type = __nv_bfloat16;
    __device__ static void read16(const __nv_bfloat16* p, bool vec, float (&x)[16]) {
        if (vec) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 q = reinterpret_cast<const uint4*>(p)[i];
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                    x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __bfloat162float(p[i]);
        }
    }
    __device__ static void write16(__nv_bfloat16* p, const float (&x)[16]) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
};

// Where position p of a lane's head lies: the tile's address, or null for a page id out of range.
template <int D>
__device__ __forceinline__ char* tile_of(const CacheArgs& c, int lane, int head, int p, bool& bad) {
    const int page = c.table[(size_t)lane * c.max_pages + (p >> c.page_shift)];
    if (page < 0 || page >= c.n_pages) { bad = true; return nullptr; }
    const int tiles = 1 << (c.page_shift - 4), tile = (p & ((1 << c.page_shift) - 1)) >> 4;
    return c.pages + (((size_t)page * c.heads + head) * tiles + tile) * Tile4<D>::BYTES;
}

__device__ __forceinline__ void flag_lane(int* lane_status, int lane, int code) {
    if (lane_status) atomicMin(&lane_status[lane], code);
}

// One thread stores one block of 16 dimensions of one token: it reads 16 elements, finds their
// largest magnitude, and writes 8 bytes of codes and a scale.  Blocks run fastest over the threads:
// a warp reads whole 32-byte sectors side by side.
constexpr int C4_NT = 256;

template <int DT, int D>
__global__ void __launch_bounds__(C4_NT)
append_kernel(const CacheArgs c, const typename Io<DT>::type* __restrict__ k, long long k_ld,
              const typename Io<DT>::type* __restrict__ v, long long v_ld, bool vec) {
    using Ti = Tile4<D>;
    // (lanes x T is at most 2^30, heads at most 128: pieces of a row are counted in 32 bits, rows in 32 bits)
    const unsigned per_row = 2 * c.heads * Ti::NB;
    const unsigned step = gridDim.x * C4_NT, first = blockIdx.x * C4_NT + threadIdx.x;
    const unsigned row_step = step / per_row, piece_step = step % per_row;
    unsigned row = first / per_row, piece = first % per_row;
    for (; row < (unsigned)c.lanes * c.T; row += row_step, piece += piece_step) {
        if (piece >= per_row) { piece -= per_row; if (++row >= (unsigned)c.lanes * c.T) break; }
        const int b = piece % Ti::NB, head = piece / Ti::NB % c.heads;
        const bool is_v = piece >= per_row / 2;
        const int lane = (int)(row / c.T), tok = (int)(row % c.T);
        const int len = c.len[lane];
        if (len < 0 || len > ((long long)c.max_pages << c.page_shift)) { flag_lane(c.lane_status, lane, AS_ERR_INVALID_ARG); continue; }
        const int p = len - c.T + tok;
        if (p < 0) continue;
        bool bad = false;
        char* tile = tile_of<D>(c, lane, head, p, bad);
        if (bad) { flag_lane(c.lane_status, lane, AS_ERR_INVALID_ARG); continue; }
        float x[16];
        Io<DT>::read16((is_v ? v + (long long)row * v_ld : k + (long long)row * k_ld) + head * D + b * 16, vec, x);
        const float* hs = is_v ? c.v_scale : c.k_scale;
        const float inv = hs ? __frcp_rn(hs[head]) : 1.f;
        float top = 0.f;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = __fmul_rn(x[e], inv);
            odd |= !(fabsf(x[e]) <= 3.402823466e38f);
            if (x[e] != x[e]) x[e] = 0.f;
            top = fmaxf(top, fabsf(x[e]));
        }
        if (odd) flag_lane(c.lane_status, lane, AS_ERR_NUMERIC);
        const uint32_t s8 = to_e4m3(__fmul_rn(top, 1.f / 6.f));
        const float s = e4m3_value(s8);
        const float rs = s > 0.f ? __frcp_rn(s) : 0.f;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            // (an infinite value with a zero factor cannot occur: its block's scale is the largest)
            w[e >> 3] |= to_codes(__fmul_rn(x[e], rs), __fmul_rn(x[e + 1], rs)) << (4 * (e & 7));
        }
        const int t = p & 15;
        *reinterpret_cast<uint2*>(tile + (is_v ? Ti::v_code(t, b) : Ti::k_code(t, b))) = make_uint2(w[0], w[1]);
        tile[is_v ? Ti::v_scale(t, b) : Ti::k_scale(t, b)] = (char)s8;
    }
}

template <int DT, int D>
__global__ void __launch_bounds__(C4_NT)
load_kernel(const CacheArgs c, typename Io<DT>::type* __restrict__ k, typename Io<DT>::type* __restrict__ v) {
    using Ti = Tile4<D>;
    const unsigned per_row = 2 * c.heads * Ti::NB;
    const unsigned step = gridDim.x * C4_NT, first = blockIdx.x * C4_NT + threadIdx.x;
    const unsigned row_step = step / per_row, piece_step = step % per_row;
    unsigned row = first / per_row, piece = first % per_row;
    for (; row < (unsigned)c.lanes * c.T; row += row_step, piece += piece_step) {
        if (piece >= per_row) { piece -= per_row; if (++row >= (unsigned)c.lanes * c.T) break; }
        const int b = piece % Ti::NB, head = piece / Ti::NB % c.heads;
        const bool is_v = piece >= per_row / 2;
        const int lane = (int)(row / c.T), tok = (int)(row % c.T);
        const int len = c.len[lane];
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
        bool bad = len < 0 || len > ((long long)c.max_pages << c.page_shift);
        const int p = len - c.T + tok;
        if (!bad && p >= 0) {
            const char* tile = tile_of<D>(c, lane, head, p, bad);
            if (!bad) {
                const int t = p & 15;
                const uint2 q = *reinterpret_cast<const uint2*>(tile + (is_v ? Ti::v_code(t, b) : Ti::k_code(t, b)));
                const float s = e4m3_value((uint8_t)tile[is_v ? Ti::v_scale(t, b) : Ti::k_scale(t, b)]);
                const float* hs = is_v ? c.v_scale : c.k_scale;
                const float g = hs ? hs[head] : 1.f;
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint32_t h2 = codes_f16x2((e < 8 ? q.x : q.y) >> (4 * (e & 7)));
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
                    x[e] = f.x * s * g;                 // code * scale is exact, one rounding
                    x[e + 1] = f.y * s * g;
                }
            }
        }
        if (bad) flag_lane(c.lane_status, lane, AS_ERR_INVALID_ARG);
        Io<DT>::write16((is_v ? v : k) + (size_t)row * c.heads * D + head * D + b * 16, x);
    }
}

}  // namespace asx
