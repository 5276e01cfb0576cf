// The driver's tensor-map encoder for entry points that need no context.  Internal to the library.
#pragma once
#include <cuda.h>

namespace beagle {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled tensor_map_encoder();       // NULL when the driver has none

}  // namespace beagle
