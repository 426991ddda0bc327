// vie_api.h - what the translation units that hold C entry points share: the
// calling thread's error message, and the library-wide device flag word.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "vie_head.h"

namespace vie {

// Sets vie_last_error() and returns st.
vie_status fail(vie_status st, const char *fmt, ...);
// The same for a CUDA error (VIE_ERR_OOM or VIE_ERR_CUDA).
vie_status fail_cuda(cudaError_t e, const char *what);

// Device address of the flag word that vie_device_status reads, on the
// current device.
cudaError_t device_flag_word(uint32_t **word);

// Runs set(), which prepares a kernel for the current device, on the first call
// for that device (again after a failure).
class PerDevice {
  public:
    template <typename F>
    cudaError_t once(const F &set) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
        if (done_.load(std::memory_order_acquire) & bit) return cudaSuccess;
        e = set();
        if (e == cudaSuccess) done_.fetch_or(bit, std::memory_order_release);
        return e;
    }

  private:
    std::atomic<uint64_t> done_{0};
};

// SMs of the current device.
inline cudaError_t sm_count(int *sms) {
    static std::atomic<int> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool kept = dev >= 0 && dev < 64;
    if (kept && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess && kept) known[dev].store(*sms, std::memory_order_relaxed);
    return e;
}

inline bool aligned_to(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

inline int dtype_size(vie_dtype t) { return t == VIE_DTYPE_BF16 ? 2 : 4; }
inline bool dtype_known(vie_dtype t) { return t == VIE_DTYPE_BF16 || t == VIE_DTYPE_F32; }

// VIE_OK if p can hold `rows` rows of `cols` values of type t, `ld` values
// apart: known type, aligned to a value, ld >= cols, no overflow.
vie_status check_matrix(const char *fn, const char *name, const void *p, vie_dtype t, int64_t rows, int64_t cols,
                        int64_t ld);

}  // namespace vie
