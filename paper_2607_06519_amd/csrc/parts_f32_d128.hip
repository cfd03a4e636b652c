// Decode over parts: kernels of one cache type and head dimension (parts.h).
#include "parts.h"

namespace fdkv {
hipError_t launch_parts_f32_d128(const PartsParams& P, hipStream_t s) { return launch_parts_ty<128, parts::kTyF32>(P, s); }
}  // namespace fdkv
