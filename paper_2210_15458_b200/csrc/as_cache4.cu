// C-ABI entry points of the 4-bit cache and of attention over it.
#include "as_attend_host.cuh"

namespace asx {

ASX_BOUNDS_READER(bounds_cache4)

static unsigned block_grid(const CacheArgs& a, int D) { return grid_of((long long)a.lanes * a.T * 2 * a.heads * (D / 16), C4_NT); }
template <int DT, int D>
static void launch_append(const CacheArgs& a, const void* k, long long k_ld, const void* v, long long v_ld, bool vec, cudaStream_t st) {
    using E = typename Io<DT>::type;
    auto kern = vec ? append_kernel<DT, D, true> : append_kernel<DT, D, false>;
    kern<<<block_grid(a, D), C4_NT, 0, st>>>(a, static_cast<const E*>(k), k_ld, static_cast<const E*>(v), v_ld);
}
template <int DT, int D>
static void launch_load(const CacheArgs& a, void* k, void* v, cudaStream_t st) {
    using E = typename Io<DT>::type;
    load_kernel<DT, D><<<block_grid(a, D), C4_NT, 0, st>>>(a, static_cast<E*>(k), static_cast<E*>(v));
}

}  // namespace asx

using namespace asx;

extern "C" {

size_t as_cache4_bytes(int n_pages, int heads, int head_dim, int page_size) {
    if (n_pages < 1 || heads < 1 || head_dim < 1 || page_size < 1) return 0;
    return (size_t)n_pages * heads * (page_size / 16) * 18 * head_dim;
}

int as_cache4_append(const as_cache4* cache, const void* d_k, long long k_ld, const void* d_v, long long v_ld, int dtype, int lanes,
                     int T, const int32_t* d_table, int max_pages, const int32_t* d_len, int32_t* d_lane_status, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    const long long row = (long long)cache->heads * cache->head_dim;
    if (k_ld < row || v_ld < row) return set_err(AS_ERR_INVALID_ARG, "k_ld = %lld or v_ld = %lld is smaller than heads * head_dim = %lld", k_ld, v_ld, row);
    if (lanes == 0) return AS_OK;
    if (!d_k || !d_v) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is NULL");
    const int es = dtype == AS_F32 ? 4 : 2;
    const uintptr_t at = reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_v);
    if (at % es) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is not element-aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = clear_status(d_lane_status, lanes, st)) != AS_OK) return rc;
    const bool vec = ((at | (uintptr_t)(k_ld * es) | (uintptr_t)(v_ld * es)) & 15) == 0;
    const CacheArgs a = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    if (dtype == AS_F32) {
        if (cache->head_dim == 64) launch_append<AS_F32, 64>(a, d_k, k_ld, d_v, v_ld, vec, st);
        else launch_append<AS_F32, 128>(a, d_k, k_ld, d_v, v_ld, vec, st);
    } else {
        if (cache->head_dim == 64) launch_append<AS_BF16, 64>(a, d_k, k_ld, d_v, v_ld, vec, st);
        else launch_append<AS_BF16, 128>(a, d_k, k_ld, d_v, v_ld, vec, st);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "cache append kernel launch");
}

int as_cache4_load(const as_cache4* cache, void* d_k, void* d_v, int dtype, int lanes, int T, const int32_t* d_table, int max_pages,
                   const int32_t* d_len, int32_t* d_lane_status, void* stream) {
    int rc = check_cache(cache);
    if (rc != AS_OK) return rc;
    if ((rc = check_lanes(dtype, lanes, T, d_table, max_pages, d_len, cache->page_size)) != AS_OK) return rc;
    if (lanes == 0) return AS_OK;
    if (!d_k || !d_v) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is NULL");
    if ((reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_v)) & 15) return set_err(AS_ERR_INVALID_ARG, "d_k or d_v is not 16-byte aligned");
    const DeviceInfo* di;
    if ((rc = device_info(&di)) != AS_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = clear_status(d_lane_status, lanes, st)) != AS_OK) return rc;
    const CacheArgs a = cache_args(cache, lanes, T, d_table, max_pages, d_len, d_lane_status);
    if (dtype == AS_F32) {
        if (cache->head_dim == 64) launch_load<AS_F32, 64>(a, d_k, d_v, st);
        else launch_load<AS_F32, 128>(a, d_k, d_v, st);
    } else {
        if (cache->head_dim == 64) launch_load<AS_BF16, 64>(a, d_k, d_v, st);
        else launch_load<AS_BF16, 128>(a, d_k, d_v, st);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "cache load kernel launch");
}

size_t as_cache4_attend_work_bytes(const as_cache4* cache, int dtype, int lanes, int T, int q_heads, int N) {
    // (a shape that the call refuses may not even be planned: its rows may pass 32 bits)
    if (!cache || cache->heads < 1 || (cache->head_dim != 64 && cache->head_dim != 128) || (dtype != AS_F32 && dtype != AS_BF16)) return 0;
    if (lanes < 1 || T < 1 || q_heads < 1 || q_heads % cache->heads || N < 1 || lanes % N) return 0;
    if ((long long)lanes * T > (1LL << 30) || (long long)lanes * T * q_heads > 0x7FFFFFFFLL) return 0;
    return plan_attend(dtype, lanes, T, cache->heads, q_heads, cache->head_dim, N, nullptr).bytes;
}

int as_cache4_attend(const as_cache4* cache, const void* d_q, long long q_ld, int dtype, int lanes, int T, int q_heads,
                     const int32_t* d_table, int max_pages, const int32_t* d_len, double scale, int N, const int32_t* d_shared,
                     void* d_out, float* d_lse, int32_t* d_lane_status, void* d_work, size_t work_bytes, void* stream) {
    return attend<false>(cache, d_q, q_ld, dtype, lanes, T, q_heads, d_table, max_pages, d_len, scale, N, d_shared, 0, 0, d_out, d_lse, d_lane_status, d_work,
                         work_bytes, stream);
}

}  // extern "C"
