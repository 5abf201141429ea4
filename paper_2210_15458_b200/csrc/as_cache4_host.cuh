// Host side that the calls on the 4-bit cache share: checks of arguments, what the kernels get.
#pragma once
#include "as_cache4.cuh"

namespace asx {

inline int check_cache(const as_cache4* c) {
    if (!c) return set_err(AS_ERR_INVALID_ARG, "cache is NULL");
    if (c->n_pages < 1 || c->heads < 1) return set_err(AS_ERR_INVALID_ARG, "n_pages = %d and heads = %d must be >= 1", c->n_pages, c->heads);
    if (c->head_dim != 64 && c->head_dim != 128) return set_err(AS_ERR_UNSUPPORTED, "head_dim = %d is not 64 or 128", c->head_dim);
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return set_err(AS_ERR_UNSUPPORTED, "page_size = %d is not 16, 32, 64 or 128", c->page_size);
    if (!c->d_pages) return set_err(AS_ERR_INVALID_ARG, "d_pages is NULL");
    if (reinterpret_cast<uintptr_t>(c->d_pages) & 15) return set_err(AS_ERR_INVALID_ARG, "d_pages is not 16-byte aligned");
    return AS_OK;
}

inline int check_lanes(int dtype, int lanes, int T, const void* table, int max_pages, const void* len, int page_size) {
    if (dtype != AS_F32 && dtype != AS_BF16) return set_err(AS_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (lanes < 0) return set_err(AS_ERR_INVALID_ARG, "lanes = %d must be >= 0", lanes);
    if (T < 1) return set_err(AS_ERR_INVALID_ARG, "T = %d must be >= 1", T);
    if (max_pages < 1) return set_err(AS_ERR_INVALID_ARG, "max_pages = %d must be >= 1", max_pages);
    if ((long long)max_pages * page_size > (1LL << 30) || (long long)lanes * T > (1LL << 30))
        return set_err(AS_ERR_UNSUPPORTED, "max_pages * page_size and lanes * T must not exceed 2^30");
    if (lanes > 0 && (!table || !len)) return set_err(AS_ERR_INVALID_ARG, "d_table or d_len is NULL");
    return AS_OK;
}

inline CacheArgs cache_args(const as_cache4* c, int lanes, int T, const int* table, int max_pages, const int* len, int* status) {
    CacheArgs a;
    a.pages = static_cast<char*>(c->d_pages);
    a.n_pages = c->n_pages; a.heads = c->heads;
    a.page_shift = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
    a.k_scale = c->d_k_scale; a.v_scale = c->d_v_scale;
    a.table = table; a.max_pages = max_pages; a.len = len; a.lane_status = status;
    a.lanes = lanes; a.T = T;
    a.by_T.set(T);
    a.by_heads.set(c->heads);
    return a;
}

inline int clear_status(int* status, int lanes, cudaStream_t st) {
    if (!status) return AS_OK;
    const cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int) * (size_t)lanes, st);
    return e == cudaSuccess ? AS_OK : cuda_fail(e, "lane status");
}

inline unsigned grid_of(long long threads, int nt) {
    const long long n = (threads + nt - 1) / nt;
    return (unsigned)(n < (1 << 14) ? n : (1 << 14));       // (the kernels loop)
}

}  // namespace asx
