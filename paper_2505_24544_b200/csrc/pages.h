// Host-side pieces shared by the paged-cache entry points.  Internal to the library.
#pragma once
#include "../../include/beagle.h"
#include "common.cuh"

namespace beagle {

struct PageSlots { int32_t slot[kMaxCallBatch]; };      // the slots of one call, by value in the kernel parameters

struct AppendRows {                                     // row b of an append: `count` source rows from row `start` on
    long long start[kMaxCallBatch];
    int32_t count[kMaxCallBatch];
};

bool pages_valid_shape(const beagle_pages* p);
beagle_status pages_check(const beagle_pages* p);
beagle_status pages_check_slots(const beagle_pages* p, int n, const int32_t* slots, PageSlots* out);

// The append with any rows (beagle_pages_append takes T rows each); n_new_dev, where given, cuts every row's count.
beagle_status pages_append_rows(const beagle_pages* p, int batch, const int32_t* slot_host, const AppendRows& rows, const int32_t* n_new_dev,
                                const void* k_new_dev, long long k_stride, const void* v_new_dev, long long v_stride, int32_t* ok_dev, cudaStream_t stream);
bool paged_attn_fits(const beagle_pages* p, int batch);      // a call's tiles are counted in 32 bits
// A workspace that suits beagle_paged_attn on every cache of this type and width.
size_t paged_attn_workspace_most(int dtype, int head_dim);

}  // namespace beagle
