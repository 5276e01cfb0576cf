// Host-side pieces shared by the paged-cache entry points.  Internal to the library.
#pragma once
#include "../../include/beagle.h"
#include "common.cuh"

namespace beagle {

struct PageSlots { int32_t slot[kMaxCallBatch]; };      // the slots of one call, by value in the kernel parameters

bool pages_valid_shape(const beagle_pages* p);
beagle_status pages_check(const beagle_pages* p);
beagle_status pages_check_slots(const beagle_pages* p, int n, const int32_t* slots, PageSlots* out);

}  // namespace beagle
