// Host-side helpers that the translation units share; defined in as_api.cu.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace asx {

int set_err(int code, const char* fmt, ...);        // records the calling thread's error text, returns code
int cuda_fail(cudaError_t e, const char* what);     // the same for a CUDA runtime error

struct DeviceInfo {
    int sms = 0;
    bool ok = false;
};
int device_info(const DeviceInfo** out);            // the current device's, looked up once

int check_scalars(int dtype, int V, long long ld, double temp, double top_p);   // what the step calls check of their logits
int check_data(const void* data, int dtype);

long long wait_cycles_now();                        // bound on every on-device wait, in clock cycles (AS_TUNE_WAIT_KCYCLES)
bool window_groups_now();                           // shared beginnings by groups whatever the window (AS_TUNE_WINDOW_GROUPS)

constexpr size_t SMEM_OPTIN_MAX = 232448;           // 227 KB per CTA on sm_100

// Launches a kernel that may be set up while the one before it on the stream drains: it waits for that one's completion
// itself (griddepcontrol.wait) before it touches global memory.
template <class K, class... A>
inline cudaError_t launch_after(K kern, dim3 grid, unsigned block, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

// Checked builds: each translation unit keeps its own record of out-of-range indices; these copy
// it out (failures, first site, index, bound) and reset it.
#ifdef AS_BOUNDS_CHECK
int bounds_edit(int* h_out4, int reset);
int bounds_cache4(int* h_out4, int reset);
int bounds_pages(int* h_out4, int reset);
int bounds_window(int* h_out4, int reset);
int bounds_weigh(int* h_out4, int reset);
int bounds_evict(int* h_out4, int reset);
int bounds_verify(int* h_out4, int reset);
#endif

}  // namespace asx
