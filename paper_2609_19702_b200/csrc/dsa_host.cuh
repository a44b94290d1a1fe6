// Host-side helpers that the translation units with entry points share (defined in dsa_api.cu).
#pragma once
#include "../../include/dsa.h"

#include <atomic>

#include "dsa_launch.cuh"

namespace dsa {

// cuTensorMapEncodeTiled, looked up through the runtime (the library does not link the driver).
using TensorMapEncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                       const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                       CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

constexpr int kMaxSplits = 8192;                 // split weights of the combine kernel: 32 KB of shared memory

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int32_t host_cuda_fail(cudaError_t e);                       // remembers the code for dsa_last_cuda_error
int host_sm_count();
int32_t host_check_problem(const dsa_problem* p);
int32_t host_check_diag(const dsa_problem* p, const dsa_diag_params* d);
cudaError_t host_wait_timeouts_address(int** out);
TensorMapEncodeFn host_tensor_map_encoder();                 // nullptr: not available
void host_cache_args(const dsa_problem* p, AttnArgs* a);     // cache addressing, lengths, heads and scale; dense mask
// merge split partials that the launch in front writes (programmatic serialisation)
int32_t host_launch_combine(const float* out_part, const float* lse_part, int64_t rows, int D, int n_split, void* out,
                            float* lse, int dtype, cudaStream_t st);

cudaError_t tree_prepare();                                  // configure the drafted-token kernels for the current device
cudaError_t verify_prepare();

// Kernels that use more than 48 KB of dynamic shared memory must be told so once per device (idempotent).
template <class Kern>
cudaError_t configure_smem(Kern kern, int bytes, std::atomic<bool>* done /* [kMaxDevices] */) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !done[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
    }
    return cudaSuccess;
}

}  // namespace dsa
