// Declarations shared by the translation units of libflux_ffn_mi355.so.
#pragma once
#include <hip/hip_runtime.h>
#include "flux_ffn.h"

namespace flux_ffn {

// Remembers a failed runtime call for flux_ffn_last_hip_error and returns the status for it.
int hip_failed(hipError_t e);
#define FFN_HIP(call) do { const hipError_t e_ = (call); if (e_ != hipSuccess) return ::flux_ffn::hip_failed(e_); } while (0)

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline long long row_bytes(long long K) { return (K + 31) / 32 * 16; }
inline long long scale_row_bytes(long long K) { return ((K + 31) / 32 + 15) / 16 * 16; }

}  // namespace flux_ffn
