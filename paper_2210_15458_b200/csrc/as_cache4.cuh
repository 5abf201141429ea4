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
    __device__ static int k_code(int t, int b) { return K + ASX_AT(t * (D / 2) + b * 8, 8 * D - 7, 101); }
    __device__ static int v_code(int t, int b) { return V + ASX_AT(b * 128 + t * 8, 8 * D - 7, 102); }
    __device__ static int k_scale(int t, int b) { return KS + ASX_AT(t * NB + b, D, 103); }
    __device__ static int v_scale(int t, int b) { return VS + ASX_AT(b * 16 + t, D, 104); }
};

// n / d for n < 2^31 by a multiplication (Granlund and Montgomery's round-up method)
struct Divisor {
    uint32_t d, mul, shift;
    __host__ void set(uint32_t by) {
        d = by;
        shift = 0;
        while ((1ull << shift) < by) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - by)) / by + 1);
    }
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
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
    Divisor by_T, by_heads;
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
// the eight codes of a word -> four pairs of f16 (the conversion picks its byte itself: no shifts)
__device__ __forceinline__ void codes_f16x2(uint32_t word, uint32_t (&d)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}" : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "r"(word));
}

template <int DT> struct Io;
template <> struct Io<AS_F32> {
    using type = float;
    struct raw16 { float4 q[4]; };                      // 16 elements as they are
    __device__ static raw16 load16(const float* p, bool vec) {
        raw16 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.q[i] = vec ? __ldcs(reinterpret_cast<const float4*>(p) + i) : make_float4(p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]);
        return r;
    }
    __device__ static void widen16(const raw16& r, float (&x)[16]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[4 * i] = r.q[i].x; x[4 * i + 1] = r.q[i].y; x[4 * i + 2] = r.q[i].z; x[4 * i + 3] = r.q[i].w; }
    }
    __device__ static void read16(const float* p, bool vec, float (&x)[16]) { widen16(load16(p, vec), x); }
    __device__ static void write16(float* p, const float (&x)[16]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
};
template <> struct Io<AS_BF16> {
    using type = __nv_bfloat16;
    struct raw16 { uint32_t w[8]; };
    __device__ static raw16 load16(const __nv_bfloat16* p, bool vec) {
        raw16 r;
        if (vec) {
            const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p)), b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
            r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w; r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
        } else {
            const uint16_t* e = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) r.w[i] = e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
        }
        return r;
    }
    __device__ static void widen16(const raw16& r, float (&x)[16]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[2 * i] = __uint_as_float(r.w[i] << 16); x[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u); }
    }
    __device__ static void read16(const __nv_bfloat16* p, bool vec, float (&x)[16]) { widen16(load16(p, vec), x); }
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

__device__ __forceinline__ void flag_lane(int* lane_status, int lane, int code) {
    if (lane_status) atomicMin(&lane_status[lane], code);
}

// Storing and reading back work on blocks: 16 dimensions of one token, which are 8 bytes of codes and a scale.
struct Block {
    int lane, len, tok, head, b;                    // tok: the token within the call
    bool is_v;
};
constexpr int C4_NT = 256;

// A thread to a block, blocks side by side in the caller's tensors side by side along the threads.  Tokens are rows (at most
// 2^30), a row has 2 x heads x D / 16 blocks.  (A group of threads to a tile of 16 positions, four of them at a time, moves whole
// sectors of the cache, but leaves threads without work where a call's tokens only touch a tile: 8 + 8 heads x 128, bf16, store +
// load, by tiles / by rows, us: 512 lanes x 16 tokens 52.8 / 34.3, 64 x 256 57.5 / 52.5, 16 x 1024 53.6 / 50.4, 8 x 4096 95.5 / 93.5; in 32
// bits 8 x 4096 149.5 / 136.6.)
template <int D, class F>
__device__ __forceinline__ void each_block(const CacheArgs& c, F&& f) {
    constexpr int NB = D / 16;
    const unsigned per_row = 2 * c.heads * NB, rows = (unsigned)c.lanes * c.T;
    const unsigned step = gridDim.x * C4_NT, first = blockIdx.x * C4_NT + threadIdx.x;
    const unsigned row_step = step / per_row, piece_step = step % per_row;
    unsigned row = first / per_row, piece = first % per_row;
#pragma unroll 1
    for (; row < rows; row += row_step, piece += piece_step) {
        if (piece >= per_row) { piece -= per_row; if (++row >= rows) break; }
        Block k;
        k.is_v = piece >= per_row / 2;
        const unsigned r = piece - (k.is_v ? per_row / 2 : 0);
        k.b = r % NB;
        k.head = r / NB;
        k.lane = c.by_T.div(row);
        k.tok = row - k.lane * c.T;
        k.len = c.len[k.lane];
        f(k);
    }
}

// The tile of a token: null for one in front of the first position or in no page.
template <int D>
__device__ __forceinline__ char* tile_of(const CacheArgs& c, const Block& at) {
    const int p = at.len - c.T + at.tok, mask = (1 << c.page_shift) - 1;
    const bool len_ok = at.len >= 0 && at.len <= ((long long)c.max_pages << c.page_shift);
    const bool real = len_ok && p >= 0;
    const int page = real ? c.table[(size_t)ASX_AT(at.lane, c.lanes, 105) * c.max_pages + ASX_AT(p >> c.page_shift, c.max_pages, 106)] : 0;
    const bool in = page >= 0 && page < c.n_pages;
    if (!len_ok || !in) flag_lane(c.lane_status, at.lane, AS_ERR_INVALID_ARG);
    return real && in ? c.pages + (((size_t)page * c.heads + ASX_AT(at.head, c.heads, 107)) * (mask + 1 >> 4) + ((p & mask) >> 4)) * Tile4<D>::BYTES : nullptr;
}

// Store: a thread takes 16 neighbouring dimensions of a token (one scale): code = nearest e2m1 of x / (head scale x scale), scale
// = e4m3 of the largest |x| / 6.  Bound by issue slots (81 % busy, DRAM 33 %): 8 x 4096 tokens of 8 + 8 heads x 128 in 52 us (168 MB: 3.2 TB/s),
// one token each of 256 lanes in 4.5 us.
template <int DT, int D, bool VEC>
__global__ void __launch_bounds__(C4_NT)
append_kernel(const __grid_constant__ CacheArgs c, const typename Io<DT>::type* __restrict__ k, long long k_ld,
              const typename Io<DT>::type* __restrict__ v, long long v_ld) {
    using Ti = Tile4<D>;
    each_block<D>(c, [&](const Block& at) {
        const typename Io<DT>::type* src = (at.is_v ? v : k) + ((long long)ASX_AT(at.lane, c.lanes, 108) * c.T + at.tok) * (at.is_v ? v_ld : k_ld) +
                                           ASX_AT(at.head, c.heads, 109) * D + ASX_AT(at.b, D / 16, 110) * 16;
        const typename Io<DT>::raw16 raw = Io<DT>::load16(src, VEC);
        char* tile = tile_of<D>(c, at);
        if (!tile) return;
        const float* hs = at.is_v ? c.v_scale : c.k_scale;
        const float inv = hs ? __frcp_rn(hs[at.head]) : 1.f;
        const int t = (at.len - c.T + at.tok) & 15;
        float x[16], top = 0.f;
        Io<DT>::widen16(raw, x);
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = __fmul_rn(x[e], inv);
            odd |= !(fabsf(x[e]) <= 3.402823466e38f);
            x[e] = x[e] == x[e] ? x[e] : 0.f;
            top = fmaxf(top, fabsf(x[e]));
        }
        if (odd) flag_lane(c.lane_status, at.lane, AS_ERR_NUMERIC);
        const uint32_t s8 = to_e4m3(__fmul_rn(top, 1.f / 6.f));
        const float s = e4m3_value(s8);
        const float rs = s > 0.f ? __frcp_rn(s) : 0.f;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            // (an infinite value with a zero factor cannot occur: its block's scale is the largest)
            w[e >> 3] |= to_codes(__fmul_rn(x[e], rs), __fmul_rn(x[e + 1], rs)) << (4 * (e & 7));
        }
        *reinterpret_cast<uint2*>(tile + (at.is_v ? Ti::v_code(t, at.b) : Ti::k_code(t, at.b))) = make_uint2(w[0], w[1]);
        tile[at.is_v ? Ti::v_scale(t, at.b) : Ti::k_scale(t, at.b)] = (char)s8;
    });
}

// Load: the same threads the other way, 42 us for 8 x 4096 tokens (4.0 TB/s); issue slots 82 % busy.
template <int DT, int D>
__global__ void __launch_bounds__(C4_NT)
load_kernel(const __grid_constant__ CacheArgs c, typename Io<DT>::type* __restrict__ k, typename Io<DT>::type* __restrict__ v) {
    using Ti = Tile4<D>;
    each_block<D>(c, [&](const Block& at) {
        const char* tile = tile_of<D>(c, at);
        const float* hs = at.is_v ? c.v_scale : c.k_scale;
        const float g = hs ? hs[at.head] : 1.f;
        const int t = (at.len - c.T + at.tok) & 15;
        uint2 q = make_uint2(0, 0);
        uint32_t s8 = 0;                                // zeros where there is no token
        if (tile) {
            q = *reinterpret_cast<const uint2*>(tile + (at.is_v ? Ti::v_code(t, at.b) : Ti::k_code(t, at.b)));
            s8 = (uint8_t)tile[at.is_v ? Ti::v_scale(t, at.b) : Ti::k_scale(t, at.b)];
        }
        const float s = e4m3_value(s8);
        float x[16];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t h[4];
            codes_f16x2(i ? q.y : q.x, h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
                x[8 * i + 2 * e] = f.x * s * g;         // code * scale is exact, one rounding
                x[8 * i + 2 * e + 1] = f.y * s * g;
            }
        }
        Io<DT>::write16((at.is_v ? v : k) + ((size_t)ASX_AT(at.lane, c.lanes, 111) * c.T + at.tok) * c.heads * D + ASX_AT(at.head, c.heads, 112) * D +
                            ASX_AT(at.b, D / 16, 113) * 16, x);
    });
}

}  // namespace asx
