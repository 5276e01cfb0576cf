// What entry points without a context ask of the device: the driver's tensor-map encoder, the SM count.  Internal to the library.
#pragma once
#include <cuda.h>

namespace beagle {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled tensor_map_encoder();       // NULL when the driver has none
int device_sm_count();                  // of the current device (148 when there is none to ask)

}  // namespace beagle
