// vie_api.h - what the translation units that hold C entry points share: the
// calling thread's error message, and the library-wide device flag word.
#pragma once

#include <cuda_runtime.h>

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

inline bool aligned_to(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

inline int dtype_size(vie_dtype t) { return t == VIE_DTYPE_BF16 ? 2 : 4; }
inline bool dtype_known(vie_dtype t) { return t == VIE_DTYPE_BF16 || t == VIE_DTYPE_F32; }

// VIE_OK if p can hold `rows` rows of `cols` values of type t, `ld` values
// apart: known type, aligned to a value, ld >= cols, no overflow.
vie_status check_matrix(const char *fn, const char *name, const void *p, vie_dtype t, int64_t rows, int64_t cols,
                        int64_t ld);

}  // namespace vie
