// Device helpers of the windowed attention kernels on tcgen05.
#pragma once
#include "common.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.h"

namespace beagle {
namespace tc {

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One lane of a converged warp, the same one every time.  The roles that issue asynchronous work run with all 32 lanes and let
// this one issue: addresses and descriptors then stay in uniform registers, where a branch of a single lane has to move
// every operand of every instruction there (measured: the issue of eight products 550-750 -> 100-200 cycles).
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag) { return mbar_wait(bar, parity, abort_flag); }
// A warp's bounded wait: true for every lane, or false for every lane.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    bool ok = mbar_try_wait(bar, parity);
    if (!__all_sync(0xffffffffu, ok)) ok = __all_sync(0xffffffffu, ok || mbar_wait_slow(bar, parity, abort_flag));
    else ok = true;
    return ok;
}

// Both waits, their first tests in flight together (a test that succeeds takes some hundred cycles).
__device__ __forceinline__ bool warp_wait2(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1, volatile int* abort_flag) {
    const uint32_t a = mbar_try_wait(bar0, parity0), b = mbar_try_wait(bar1, parity1);
    if (__all_sync(0xffffffffu, a & b)) return true;
    return warp_wait(bar0, parity0, abort_flag) && warp_wait(bar1, parity1, abort_flag);
}

// Products and commits of a converged warp, issued by its elected lane (a predicate, not a branch).
__device__ __forceinline__ void umma_ss(bool leader, uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate), "r"((uint32_t)leader)
        : "memory");
}
// A operand in tensor memory: rows are lanes, a column holds two consecutive bf16 of the contraction.
__device__ __forceinline__ void umma_ts(bool leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accumulate), "r"((uint32_t)leader)
        : "memory");
}
__device__ __forceinline__ void commit_el(bool leader, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"((uint32_t)leader)
        : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
// Untiled copy: both addresses 16-byte aligned, `bytes` a multiple of 16.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
// Tile of shared memory to global memory (generic writes before it: fence_async_smem); store_done: the shared memory may be
// written again.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* tm, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tm), "r"(src), "r"(c0), "r"(c1) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void store_done() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
// Two fp32 values in one 64-bit register and the packed arithmetic on them (one issue slot for two operations).
__device__ __forceinline__ uint64_t pk2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void un2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.ftz.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Scores of 32 columns -> their maximum (masked: only where `vis` has a bit; the others become -inf).
template <bool MASK>
__device__ __forceinline__ float chunk_max(uint32_t* r, uint32_t vis, float mx) {
    if (MASK) {
#pragma unroll
        for (int x = 0; x < 32; ++x) r[x] = (vis >> x & 1u) ? r[x] : 0xff800000u;
    }
    float y = -INFINITY;
#pragma unroll
    for (int x = 0; x < 32; x += 4) {                            // two chains
        mx = max3(mx, __uint_as_float(r[x]), __uint_as_float(r[x + 1]));
        y = max3(y, __uint_as_float(r[x + 2]), __uint_as_float(r[x + 3]));
    }
    return fmaxf(mx, y);
}
// exp2(S * scale + neg) of 32 columns as bf16 pairs; their sum (of the unrounded weights) is added to `sum`.
__device__ __forceinline__ void chunk_exp(const uint32_t* r, uint64_t scale2, uint64_t neg2, uint32_t* p, uint64_t& sum0, uint64_t& sum1) {
#pragma unroll
    for (int x = 0; x < 32; x += 4) {
        float e[4];
        un2(fma2(pk2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), scale2, neg2), e[0], e[1]);
        un2(fma2(pk2(__uint_as_float(r[x + 2]), __uint_as_float(r[x + 3])), scale2, neg2), e[2], e[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = exp2f(e[i]);
        sum0 = add2(sum0, pk2(e[0], e[1]));
        sum1 = add2(sum1, pk2(e[2], e[3]));
        p[x >> 1] = pack_bf16(e[0], e[1]);
        p[(x >> 1) + 1] = pack_bf16(e[2], e[3]);
    }
}
// Zeroes rows [from, to) of an operand tile of `rows` rows x DH bf16 (64-column blocks of rows * 128 bytes; whole rows, so the
// swizzle inside a row does not matter).  One warp.
template <int DH>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int rows, int from, int to, int lane) {
    from = max(from, 0);
    const int n = (to - from) * 8;                       // 16-byte pieces per block
#pragma unroll
    for (int hf = 0; hf < DH / 64; ++hf)
        for (int i = lane; i < n; i += 32) *reinterpret_cast<uint4*>(tile + (size_t)hf * rows * 128 + from * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
}

}  // namespace tc

// Tensor map of a bf16 matrix [rows, cols] with rows `ld` elements apart: boxes of 64 columns (128-byte swizzle) or 32 (64-byte
// swizzle) x box_rows, out-of-range rows read as zero.
inline bool win_map(CUtensorMap* out, const void* base, long long rows, long long cols, long long ld, int box_rows, int box_cols = 64) {
    const EncodeTiled encode = tensor_map_encoder();
    if (encode == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace beagle
