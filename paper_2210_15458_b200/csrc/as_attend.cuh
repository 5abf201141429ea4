// Attention over the 4-bit cache.
#pragma once
#include "as_cache4.cuh"

namespace asx {

struct AttendArgs {
    CacheArgs c;
    const void* q;
    long long q_ld;
    int q_heads;
    float scale;
    int N;
    const int* shared;
    void* out;
    float* lse;
};

// One warp takes one query row (token, head): it walks the lane's tokens with the running maximum
// and sum of a softmax; lane l of the warp holds dimensions l * D/32 and up.
template <int DT, int D>
__global__ void __launch_bounds__(128) attend_rows_kernel(const AttendArgs a) {
    using Ti = Tile4<D>;
    constexpr int PER = D / 32;
    const CacheArgs& c = a.c;
    const int l = threadIdx.x & 31;
    const long long rows = (long long)c.lanes * c.T * a.q_heads;
    for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * 4) {
        const int h = (int)(r % a.q_heads);
        const long long row = r / a.q_heads;
        const int lane = (int)(row / c.T), tok = (int)(row % c.T);
        const int head = h / (a.q_heads / c.heads);
        int len = c.len[lane];
        if (len < 0 || len > ((long long)c.max_pages << c.page_shift)) { if (l == 0) flag_lane(c.lane_status, lane, AS_ERR_INVALID_ARG); len = 0; }
        const int limit = len - c.T + 1 + tok;
        const typename Io<DT>::type* q = reinterpret_cast<const typename Io<DT>::type*>(a.q) + row * a.q_ld + h * D + l * PER;
        const float kg = c.k_scale ? c.k_scale[head] : 1.f, vg = c.v_scale ? c.v_scale[head] : 1.f;
        float x[PER], o[PER], m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int e = 0; e < PER; ++e) { x[e] = (float)q[e] * (a.scale * kg); o[e] = 0.f; }
        const int b = l * PER / 16, inb = l * PER % 16;
        for (int p = 0; p < limit; ++p) {
            bool bad = false;
            const char* tile = tile_of<D>(c, lane, head, p, bad);
            if (bad) {
                if (l == 0) flag_lane(c.lane_status, lane, AS_ERR_INVALID_ARG);
                tile = c.pages + ((size_t)head * (1 << (c.page_shift - 4)) + ((p & ((1 << c.page_shift) - 1)) >> 4)) * Ti::BYTES;
            }
            const int t = p & 15;
            const float ks = e4m3_value((uint8_t)tile[Ti::k_scale(t, b)]), vs = e4m3_value((uint8_t)tile[Ti::v_scale(t, b)]);
            float s = 0.f, val[PER];
#pragma unroll
            for (int e = 0; e < PER; e += 2) {
                const uint32_t kh = codes_f16x2((uint8_t)tile[Ti::k_code(t, b) + (inb + e) / 2]);
                const uint32_t vh = codes_f16x2((uint8_t)tile[Ti::v_code(t, b) + (inb + e) / 2]);
                const float2 kf = __half22float2(*reinterpret_cast<const __half2*>(&kh));
                const float2 vf = __half22float2(*reinterpret_cast<const __half2*>(&vh));
                s += x[e] * kf.x + x[e + 1] * kf.y;
                val[e] = vf.x * vs; val[e + 1] = vf.y * vs;
            }
            s *= ks;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
            const float m2 = fmaxf(m, s), f = __expf(m - m2), w = __expf(s - m2);
            sum = sum * f + w;
#pragma unroll
            for (int e = 0; e < PER; ++e) o[e] = o[e] * f + w * val[e];
            m = m2;
        }
        const float inv = sum > 0.f ? vg / sum : 0.f;
        typename Io<DT>::type* out = reinterpret_cast<typename Io<DT>::type*>(a.out) + r * D + l * PER;
#pragma unroll
        for (int e = 0; e < PER; ++e) out[e] = o[e] * inv;
        if (a.lse && l == 0) a.lse[r] = sum > 0.f ? m + logf(sum) : -INFINITY;
    }
}

}  // namespace asx
