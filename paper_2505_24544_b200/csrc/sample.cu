// One token per row of logits from a given uniform number, after temperature, top-k, top-p and min-p (beagle_sample).
//
// All three filters keep a leading run of the tokens in order of (logit falling, id rising), so the kept set is one threshold on the
// 64-bit entry (order-preserving logit bits, inverted id).  The draw is an inverse CDF in order of id.
//
// Weights exp((l - largest) / T) are formed in double precision and rounded to integers, 2^45 for the largest: sums of up to 2^18 of
// them fit 64 bits and do not depend on their order, so neither the number of thread blocks of a row nor timing has an influence on
// the result, and a token differs from exact arithmetic's only if a sum comes within some 2^-45 of a border.
//
// A row belongs to a cluster of up to 8 thread blocks, each of which keeps its slice of the logits in shared memory: they are read
// from memory once (the floor of the call), all passes after that stay on chip and take two fp32 operations a token where nothing more is
// known of it.  What costs is the double-precision weight (some 25 instructions), so it is formed
//   - of all tokens, once, only if top-k does not limit them: the total is needed then.  top-p: a histogram of fp32 weights says beforehand
//     in which few bins of distance the border lies, so that the same pass finds the exact weight before them and lists their tokens;
//   - by code where the logits are bf16 and have few values (1408 codes of either sign; the few logits nearer to 0 are computed): a table
//     holds the weight of every code.  top-p, and top-k beyond kPairs: the tokens of every code are counted, each block adds up its share of the codes,
//     and the border falls on one code, exactly, of whose tokens the first so many in order of id are kept;
//   - otherwise of candidates alone, those a bound in fp32 does not exclude.  top-k: at least k groups of a few neighbours (the ones read as
//     one 16-byte piece) have their largest in the leading bins of a histogram, so the k-th token is in those too.  min-p: its distance.
// Up to kGather candidates or tokens of the border's bins, nearly always, go to the first block: up to kPairs are compared pairwise, more
// selected by histograms of their keys.  More than kGather of them: the cluster finds each border with a histogram whose counts bracket the
// weights, one exact pass, and a list of the tokens in the few bins left, compared pairwise; more than kList of those: their range of logit
// bits is divided further, by 2048 a level with exact weights, until few are left, or only equal logits, which are taken in order of id.
//
// Bound by latency: a row is a chain of some ten short passes with a meeting of the cluster after most (a microsecond each, with the words read
// from the other blocks), 20 to 30 us from end to end; two blocks share an SM, so 71 rows of 128256 bf16 logits are under way at a time.  Measured,
// 448 such rows (115 MB): temperature alone 164 us (weights from the table: half of a row's time), top-k of 50 121, top-p of 0.9 224, min-p of 0.05 94, mixed
// filters 169; the same in fp32 (230 MB) 229, 258, 500 and 168; one row of 32000 fp32 logits with top-k 12 us with the call, of 128256 bf16 ones with top-p
// 31 after a flush, 22 in a row.
#include <cooperative_groups.h>
#include <math_constants.h>

#include <atomic>
#include <cstdlib>
#include <type_traits>

#include "../../include/beagle.h"
#include "common.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.h"

namespace beagle {

namespace {

namespace cg = cooperative_groups;
using namespace tc;
typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048, kPerThread = kBins / kThreads;
constexpr int kMassBins = 1024;          // of the first block's selections
constexpr int kGather = 3500;            // candidates that the first block finishes alone
constexpr int kPairs = 256;              // candidates that it compares pairwise
constexpr int kList = kThreads;          // tokens that a block compares pairwise (the cluster's search)
constexpr int kSide = 1408;              // bf16 codes of one sign with a place of their own: eleven binades below the largest magnitude
constexpr int kFew = 64;                 // entries that a selection of the first block compares pairwise
constexpr int kMaxCluster = 8;
constexpr int kMaxVocab = 1 << 18;
constexpr int kMaxGroups = kMaxVocab / kMaxCluster / 128 + 8;      // of 32 16-byte pieces (128 fp32 logits, 256 bf16) in a block's slice
constexpr double kOne = 35184372088832.0;        // 2^45
constexpr double kFar = 47.0;            // log2 distance from which on the weight is 0 (2^45 * 2^-47 rounds to 0)
constexpr float kMost = 3.402823466e38f;

// 2^-r on [-1/64, 1/64] by Chebyshev interpolation of degree 5 (error 2^-49), and the numbers around it; in constant memory, where an instruction
// takes them as they are (immediate doubles cost two moves each time).
__constant__ double c_exp[9] = {-1.3338724772135417e-3, 9.618110954761505e-3, -5.550410848400134e-2, 2.4022650696921724e-1, -6.931471805599585e-1, 1.0,
                               6755399441055744.0 /* 1.5 * 2^52 */, 4503599627370496.0 /* 2^52 */, -0.03125};

struct SampleArgs {
    const void* logits;
    long long stride;
    int rows, vocab, slice;              // slice: tokens of a block (a multiple of 8)
    int more;                            // more rows than clusters fit the GPU
    uint32_t tries;                      // limit of the wait for another row
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* tokens;
    float* logp;
};

struct Shared {
    uint4 answer;                        // to the request for another row (first block)
    u64 answer_bar;
    int next;                            // that row, -1 for none or kNoAnswer
    union {
        u64 entry[kGather];              // the candidates of the row (first block)
        uint32_t codes[2 * kSide];       // bf16: tokens of every code
        double code_w[2 * kSide];        // and the weight of one
        struct { u64 mass[kBins], list[kList], list_w[kList]; } wide;
    };
    union {
        uint32_t count[kBins];
        u64 mass[kMassBins];
        struct { u64 key[kFew], w[kFew]; } few;
    };
    uint16_t cand[kGather];              // this block's candidates: positions in its slice
    u64 group[kMaxGroups];               // weight of every group of 32 pieces
    u64 scan[2 * kWarps];
    double root[32];                     // 2^(45 - j / 32)
    double c2, most;                     // 1 / (temperature ln 2); the distance that min_p allows, log2
    u64 sum[2], all, all_n, total, thr, found, middle, middle_n;
    uint32_t n_gather[2];                // candidates of the cluster (first block), of this row and of the one before
    uint32_t top, least, id, lo, hi, n_cand, n_list, n_in, bin[2], mid[2], want, ties;
};

__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(bf16 v) { return __bfloat162float(v); }
// Order-preserving bits; -0, +0 and subnormal values are equal (the fp32 operations here flush those).
__device__ __forceinline__ uint32_t bits_of(float v) {
    uint32_t u = __float_as_uint(v);
    u = (u & 0x7f800000u) == 0u ? 0u : u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float of_bits(uint32_t u) { return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u); }
__device__ __forceinline__ u64 entry_of(uint32_t bits, int id) { return ((u64)bits << 32) | (0xffffffffu - (uint32_t)id); }
__device__ __forceinline__ float value_of_entry(u64 e) { return of_bits((uint32_t)(e >> 32)); }
__device__ __forceinline__ int id_of_entry(u64 e) { return (int)(0xffffffffu - (uint32_t)e); }

// Exclusive sum over the block's threads; the block's total for every thread.
template <typename N>
__device__ __forceinline__ N block_exclusive(N v, u64* scratch, N& total) {
    N* s = reinterpret_cast<N*>(scratch);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    N incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    __syncthreads();
    if (lane == 31) s[warp] = incl;
    __syncthreads();
    N before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        before += i < warp ? s[i] : 0;
        total += s[i];
    }
    return before + incl - v;
}

// The same for three fp32 values, side by side.  s: 3 * kWarps words.
__device__ __forceinline__ void block_exclusive3(float* v, float* total, float* s) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float incl[3];
#pragma unroll
    for (int y = 0; y < 3; ++y) incl[y] = v[y];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int y = 0; y < 3; ++y) {
            const float x = __shfl_up_sync(0xffffffffu, incl[y], o);
            if (lane >= o) incl[y] += x;
        }
    __syncthreads();
#pragma unroll
    for (int y = 0; y < 3; ++y)
        if (lane == 31) s[y * kWarps + warp] = incl[y];
    __syncthreads();
#pragma unroll
    for (int y = 0; y < 3; ++y) {
        float before = 0.f;
        total[y] = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            before += i < warp ? s[y * kWarps + i] : 0.f;
            total[y] += s[y * kWarps + i];
        }
        v[y] = before + incl[y] - v[y];
    }
}

// The block's sum for every thread.
__device__ __forceinline__ u64 block_sum(u64 v, u64* scratch) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    u64 all = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) all += scratch[i];
    return all;
}

// Of n items, each with a key of its own and a measure (0: not there), in order of falling key: the key at which the shortest leading run with at
// least `goal` ends, 0 if all of them have less.  Whole block.  Ranges of more than kFew items are divided by kMassBins a level.
template <typename Key, typename Measure>
__device__ __forceinline__ u64 block_select(Shared& s, int n, Key key, Measure measure, u64 goal) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    u64 lo = ~0ull, hi = 0, before = 0;
    if (n > kFew) {
        for (int i = t; i < n; i += kThreads)
            if (measure(i) != 0) { const u64 k = key(i); lo = k < lo ? k : lo; hi = k > hi ? k : hi; }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const u64 a = __shfl_xor_sync(0xffffffffu, lo, o), b = __shfl_xor_sync(0xffffffffu, hi, o);
            lo = a < lo ? a : lo;
            hi = b > hi ? b : hi;
        }
        __syncthreads();
        if (lane == 0) { s.scan[warp] = lo; s.scan[kWarps + warp] = hi; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWarps; ++i) { lo = s.scan[i] < lo ? s.scan[i] : lo; hi = s.scan[kWarps + i] > hi ? s.scan[kWarps + i] : hi; }
    } else {
        lo = 0;
        hi = ~0ull;
    }
    for (;;) {
        __syncthreads();
        if (t == 0) { s.n_list = 0; s.found = 0; s.bin[0] = 0xffffffffu; }
        __syncthreads();
        // (those that fit are listed at once)
        for (int i = t; i < n; i += kThreads) {
            const u64 k = key(i);
            if (k < lo || k > hi) continue;
            const u64 w = measure(i);
            if (w == 0) continue;
            const uint32_t at = atomicAdd(&s.n_list, 1u);
            if (at < kFew) { s.few.key[at] = k; s.few.w[at] = w; }
        }
        __syncthreads();
        const int m = (int)s.n_list;
        if (m <= kFew) {
            if (t < m) {
                const u64 k = s.few.key[t];
                u64 cum = before;
#pragma unroll 4
                for (int i = 0; i < m; ++i) cum += s.few.key[i] > k ? s.few.w[i] : 0;
                if (cum < goal && cum + s.few.w[t] >= goal) s.found = k;
            }
            __syncthreads();
            return s.found;
        }
        const int shift = max(0, 54 - __clzll((long long)(hi - lo)));            // (hi - lo) >> shift < 1024
        for (int i = t; i < kMassBins; i += kThreads) s.mass[i] = 0;
        __syncthreads();
        for (int i = t; i < n; i += kThreads) {
            const u64 k = key(i);
            if (k < lo || k > hi) continue;
            const u64 w = measure(i);
            if (w != 0) atomicAdd(&s.mass[(hi - k) >> shift], w);
        }
        __syncthreads();
        const u64 a = s.mass[2 * t], b = s.mass[2 * t + 1];
        u64 unused;
        const u64 at = before + block_exclusive<u64>(a + b, s.scan, unused);
        if (at < goal && at + a + b >= goal) {
            const bool second = at + a < goal;
            s.bin[0] = 2 * t + (second ? 1 : 0);
            s.sum[0] = second ? at + a : at;
        }
        __syncthreads();
        const uint32_t bin = s.bin[0];
        if (bin == 0xffffffffu) return 0;
        before = s.sum[0];
        const u64 top = hi - ((u64)bin << shift), width = (1ull << shift) - 1;
        lo = top - lo > width ? top - width : lo;
        hi = top;
    }
}

// What the passes over all tokens do with a 16-byte piece without looking at each: its largest and least (not NaN), and which tokens are not below a bound.
template <typename T> struct Piece;
template <> struct Piece<float> {
    static __device__ __forceinline__ float largest(const uint4& x) { return fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w))); }
    static __device__ __forceinline__ float least(const uint4& x) { return fminf(fminf(__uint_as_float(x.x), __uint_as_float(x.y)), fminf(__uint_as_float(x.z), __uint_as_float(x.w))); }
    float bound;
    __device__ __forceinline__ explicit Piece(float b) : bound(b) {}
    __device__ __forceinline__ uint32_t mask(const uint4& x) const {
        return (__uint_as_float(x.x) >= bound ? 1u : 0u) | (__uint_as_float(x.y) >= bound ? 2u : 0u) | (__uint_as_float(x.z) >= bound ? 4u : 0u) | (__uint_as_float(x.w) >= bound ? 8u : 0u);
    }
};
template <> struct Piece<bf16> {
    static __device__ __forceinline__ __nv_bfloat162 two(uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); }
    static __device__ __forceinline__ float largest(const uint4& x) {
        const __nv_bfloat162 m = __hmax2(__hmax2(two(x.x), two(x.y)), __hmax2(two(x.z), two(x.w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ float least(const uint4& x) {
        const __nv_bfloat162 m = __hmin2(__hmin2(two(x.x), two(x.y)), __hmin2(two(x.z), two(x.w)));
        return fminf(__low2float(m), __high2float(m));
    }
    __nv_bfloat162 bound;
    __device__ __forceinline__ explicit Piece(float b) : bound(__bfloat162bfloat162(__float2bfloat16_rd(b))) {}       // (not above the bound)
    __device__ __forceinline__ uint32_t mask(const uint4& x) const {
        const uint32_t a = __hge2_mask(two(x.x), bound), b = __hge2_mask(two(x.y), bound), c = __hge2_mask(two(x.z), bound), d = __hge2_mask(two(x.w), bound);
        if ((a | b | c | d) == 0) return 0;
        return (a & 1u) | (a >> 30 & 2u) | (b & 1u) << 2 | (b >> 30 & 2u) << 2 | (c & 1u) << 4 | (c >> 30 & 2u) << 4 | (d & 1u) << 6 | (d >> 30 & 2u) << 6;
    }
};

// A row is a cluster of the launch.  A cluster that works on one asks for another that has not begun, to do it too; one thread of its first
// block.  (Starting a cluster takes some 0.3 us of the whole GPU, and rows take between 12 and 35 us, so that a fixed share of them
// leaves clusters idle: 448 mixed rows 200 against 182 us.)
__device__ __forceinline__ void ask_for_row(Shared& s) {
    const uint32_t bar = smem_u32(&s.answer_bar);
    mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(&s.answer)), "r"(bar) : "memory");
}
// The first block's index of the cluster that was given, -1 for none, or kNoAnswer: the wait is bounded like every other (the answer comes within a
// microsecond or two), and if it runs out some row may be done by nobody, it is not known which.  The cluster then marks all of them (sample_kernel).
constexpr int kNoAnswer = -2;
__device__ __forceinline__ int row_given(Shared& s, int parity, uint32_t tries) {
    const uint32_t bar = smem_u32(&s.answer_bar);
    bool ok = false;
    for (uint32_t i = 0; i < tries && !ok; ++i) ok = mbar_try_wait(bar, parity);
    if (!ok)                             // an answer on its way still lands (bounded): this memory is the block's until then
        for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(bar, parity); ++i) {}
    uint32_t given = 0, block = 0;
    if (ok)
        asm volatile("{\n.reg .pred p;\n.reg .b128 r;\nld.shared.b128 r, [%2];\n"
                     "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\nselp.u32 %0, 1, 0, p;\nmov.u32 %1, 0;\n"
                     "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n}"
                     : "=r"(given), "=r"(block)
                     : "r"(smem_u32(&s.answer))
                     : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");         // (the next answer is written there)
    return !ok ? kNoAnswer : given ? (int)block : -1;
}

// One row; next: the row that the cluster does after it, -1 or kNoAnswer.  What the blocks read of one another's shared memory stays until the cluster has met in the next row (or at the kernel's end): words that
// are set before that meeting have had a meeting after their last reading.
template <typename T>
__device__ __forceinline__ void sample_row(const SampleArgs& a, const cg::cluster_group& cluster, Shared& s, uint8_t* area, int row, int& next, int parity) {
    constexpr int VN = 16 / (int)sizeof(T);
    T* slice = reinterpret_cast<T*>(area);
    const int C = cluster.num_blocks(), rank = cluster.block_rank(), t = threadIdx.x, lane = t & 31, warp = t >> 5;

    // ---- the slice into shared memory, at the same distance from a 16-byte border as in memory; -infinity around it.  Token i is
    // slice[pad + i]; pieces of VN tokens are read whole from here on.
    const int first = min(rank * a.slice, a.vocab), n = min(a.slice, a.vocab - first);
    const T* src = static_cast<const T*>(a.logits) + (size_t)row * a.stride + first;
    const int pad = (int)(((uintptr_t)src & 15) / sizeof(T)), pieces = (pad + n + VN - 1) / VN, id0 = first - pad;
    auto raw_piece = [&](int p) { return *reinterpret_cast<const uint4*>(slice + p * VN); };
    auto piece = [&](int p, float* v) { unpack16<T>(raw_piece(p), v); };         // in fp32
    // the row's parameters are on their way meanwhile
    const uint32_t temp_bits = a.temperature != nullptr ? __float_as_uint(__ldcg(a.temperature + row)) : __float_as_uint(1.f);
    int k = a.top_k != nullptr ? __ldcg(a.top_k + row) : 0;
    float top_p = a.top_p != nullptr ? __ldcg(a.top_p + row) : 1.f;
    const float min_p = a.min_p != nullptr ? __ldcg(a.min_p + row) : 0.f, uf = __ldcg(a.u + row);
    float top = -CUDART_INF_F, least = CUDART_INF_F;
    if (t == kThreads - 1) {
        // (temperatures above 1e30 do what 1e30 does to logits that are not of that size themselves)
        s.c2 = fmin(1.4426950408889634074 / fmin((double)__uint_as_float(temp_bits), 1e30), 1e300);
        s.most = min_p > 0.f ? -log2((double)min_p) : CUDART_INF;
    }
    {
        const int head = min(n, (VN - pad) % VN), vecs = (n - head) / VN, tail = head + vecs * VN;
        const int p0 = (pad + head) / VN;                        // first whole piece
        for (int i0 = t; i0 < vecs; i0 += 4 * kThreads) {
            uint4 v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (i0 + x * kThreads < vecs) v[x] = ld_act_stream16(src + head + (i0 + x * kThreads) * VN);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (i0 + x * kThreads < vecs) {
                    *reinterpret_cast<uint4*>(slice + (size_t)(p0 + i0 + x * kThreads) * VN) = v[x];
                    top = fmaxf(top, Piece<T>::largest(v[x]));
                    least = fminf(least, Piece<T>::least(v[x]));
                }
        }
        if (t < 2 * VN) {                                        // the two ragged ends, in order
            const int at = t < VN ? t : (pad + tail) / VN * VN + t - VN;         // place in the slice
            const bool edge = t < VN ? at < pad + head : at >= pad + tail && at < pieces * VN;
            if (edge) {
                const int i = at - pad;
                const bool in = i >= 0 && i < n;
                slice[at] = in ? src[i] : from_float<T>(-CUDART_INF_F);
                if (in) { top = fmaxf(top, value_of(src[i])); least = fminf(least, value_of(src[i])); }
            }
        }
    }
    if (t == 0) { s.top = 0; s.least = 0xffffffffu; s.id = 0xffffffffu; s.n_cand = 0; }
    for (int i = t; i < kBins; i += kThreads) s.count[i] = 0;
    __syncthreads();
    {
        const uint32_t hi = __reduce_max_sync(0xffffffffu, bits_of(top)), lo = __reduce_min_sync(0xffffffffu, bits_of(least));
        if (lane == 0) { atomicMax(&s.top, hi); atomicMin(&s.least, lo); }
    }
    if (a.more && rank == 0 && t == 0) {
        const int block = row_given(s, parity, a.tries);
        s.next = block >= 0 ? block / C : block;
    }
    cluster.sync();
    {                                                            // a lane reads a block's word, all in one trip
        const uint32_t* from = lane < C ? cluster.map_shared_rank(&s.top, lane) : lane >= kMaxCluster && lane < kMaxCluster + C ? cluster.map_shared_rank(&s.least, lane - kMaxCluster)
                             : cluster.map_shared_rank(reinterpret_cast<uint32_t*>(&s.next), 0);
        const uint32_t x = *from;
        top = of_bits(__reduce_max_sync(0xffffffffu, lane < C ? x : 0));
        least = of_bits(__reduce_min_sync(0xffffffffu, lane >= kMaxCluster && lane < kMaxCluster + C ? x : 0xffffffffu));
        next = a.more ? (int)__shfl_sync(0xffffffffu, x, 31) : -1;
    }
    if (next >= 0)                                               // it comes from L2
        for (int i = t * 128; i < n * (int)sizeof(T); i += kThreads * 128)
            prefetch_l2(reinterpret_cast<const char*>(static_cast<const T*>(a.logits) + (size_t)next * a.stride + first) + i);
    if (t == 0) s.n_gather[parity ^ 1] = 0;                      // everyone has read the last row's

    // Sum of a word of the blocks' shared memory over the cluster, or over the blocks in front of `end`; whole warps, a lane reads a block's.
    auto sum_lanes = [&](u64 x) {
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        return __shfl_sync(0xffffffffu, x, 0);
    };
    auto cluster_sum = [&](u64* x, int end) { return sum_lanes(lane < end ? *cluster.map_shared_rank(x, lane) : 0); };
    // The same of two words in one trip, over the cluster and over the blocks in front of this one.
    struct Two { u64 x, y, x_before, y_before; };
    auto cluster_sums = [&](u64* x, u64* y) {
        const int i = lane % kMaxCluster;
        u64 v = lane < 2 * kMaxCluster && i < C ? *cluster.map_shared_rank(lane < kMaxCluster ? x : y, i) : 0, w = i < rank ? v : 0;
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
            v += __shfl_xor_sync(0xffffffffu, v, o);
            w += __shfl_xor_sync(0xffffffffu, w, o);
        }
        return Two{__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, kMaxCluster), __shfl_sync(0xffffffffu, w, 0), __shfl_sync(0xffffffffu, w, kMaxCluster)};
    };

    const bool drawn = temp_bits - 1u < 0x7f800000u;             // temperature above 0, infinity included
    if (top_p <= 0.f || min_p > 1.f) k = 1;                      // only the first
    if (!drawn || k == 1 || top == -CUDART_INF_F) {              // its lowest id
        const bool none = top == -CUDART_INF_F;
        uint32_t id = 0xffffffffu;
        if (!none)
            for (int p = t; p < pieces; p += kThreads) {
                float v[VN];
                piece(p, v);
#pragma unroll
                for (int i = VN - 1; i >= 0; --i)
                    if (v[i] == top) id = min(id, (uint32_t)(id0 + p * VN + i));
            }
        id = __reduce_min_sync(0xffffffffu, id);
        if (lane == 0 && id != 0xffffffffu) atomicMin(cluster.map_shared_rank(&s.id, 0), id);
        cluster.sync();
        if (rank == 0 && t == 0) {
            a.tokens[row] = none ? -1 : (int)s.id;
            if (a.logp != nullptr) a.logp[row] = none ? CUDART_NAN_F : 0.f;
        }
        return;
    }
    if (k >= a.vocab || k < 0) k = 0;
    if (!(top_p < 1.f)) top_p = 1.f;
    if (top == CUDART_INF_F) {                                   // the infinite ones share the weight: 0 and -infinity do the same
        __syncthreads();
        for (int i = t; i < pieces * VN; i += kThreads) slice[i] = from_float<T>(value_of(slice[i]) == top ? 0.f : -CUDART_INF_F);
        top = least = 0.f;
        __syncthreads();
    }
    const double c2 = s.c2, most = s.most, dtop = (double)top;
    // A value not above any logit that is at most x away (log2); at least the least finite fp32
    auto value_at = [&](double x) { return fmaxf(__double2float_rd(fmax(dtop - x / c2, -(double)kMost)), -kMost); };
    const float far = fmaxf(__double2float_ru(fmax(dtop - kFar / c2, -(double)kMost)), -kMost);          // logits from here on have a weight, if any
    auto near = [&](float v) { return v >= far; };               // (false for NaN and -infinity)
    auto distance = [&](float v) { return (dtop - (double)v) * c2; };            // log2, of a near token
    // round(2^45 * 2^-x), 0 <= x <= 47.1, as a double: x = j / 32 + r
    auto weight_d = [&](double x) {
        const double m = fma(x, 32.0, c_exp[6]);
        const int j = __double2loint(m);
        const double r = fma(m - c_exp[6], c_exp[8], x);
        double p = fma(r, c_exp[0], c_exp[1]);
        p = fma(r, p, c_exp[2]);
        p = fma(r, p, c_exp[3]);
        p = fma(r, p, c_exp[4]);
        p = fma(r, p, c_exp[5]);
        const double w = s.root[j & 31];                         // times 2^-(j / 32) in whole powers: its exponent less
        return fma(p, __hiloint2double(__double2hiint(w) - ((j << 15) & 0xfff00000), __double2loint(w)), c_exp[7]) - c_exp[7];
    };
    auto weight = [&](double x) { return (u64)weight_d(x); };
    u64 thr = 0;                                                 // kept so far: entries from thr on

    // Weight of every group of 32 pieces, of the tokens that are near or, if `limited`, kept (not below thr and within the limit); the row's total
    // for every thread.  (Excluded tokens run through the arithmetic as the largest, without a branch.  A lane's sum stays below 2^53: exact.)
    auto weigh = [&](auto limited, double limit) {
        constexpr bool kLimited = decltype(limited)::value;
        const float thr_v = kLimited && thr != 0 ? value_of_entry(thr) : -CUDART_INF_F;
        const int thr_id = kLimited && thr != 0 ? id_of_entry(thr) : 0x7fffffff, groups = (pieces + 31) / 32;
        u64 all = 0;
        for (int g = warp; g < groups; g += kWarps) {
            const int p = 32 * g + lane;
            double sum = 0.0;
            if (p < pieces) {
                float v[VN];
                piece(p, v);
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    bool in = near(v[i]);
                    if (kLimited) in = in && (v[i] > thr_v || (v[i] == thr_v && id0 + p * VN + i <= thr_id));
                    const double x = distance(in ? v[i] : top);
                    if (kLimited) in = in && (x <= limit || v[i] == top);
                    const double y = weight_d(x);
                    if (in) sum += y;
                }
            }
            u64 w = (u64)sum;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
            if (lane == 0) s.group[g] = w;
            all += w;
        }
        __syncthreads();
        u64 total;
        block_exclusive<u64>(lane == 0 ? all : 0, s.scan, total);
        if (t == 0) s.total = total;
        cluster.sync();
        return cluster_sum(&s.total, C);
    };
    auto values = [&](int p, float* v) {                         // of a piece, or of none
#pragma unroll
        for (int i = 0; i < VN; ++i) v[i] = -CUDART_INF_F;
        if (p < pieces) piece(p, v);
    };
    // A warp with a group's pieces, one a lane, their measures and what lies before them: the first token at which the target is exceeded.
    auto within = [&](int p, const float* v, const u64* w, u64 start, u64 target, auto hit) {
        u64 all = 0;
#pragma unroll
        for (int i = 0; i < VN; ++i) all += w[i];
        u64 incl = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        u64 cum = start + incl - all;
        if (cum <= target && target < cum + all) {
            bool found = false;
#pragma unroll
            for (int i = 0; i < VN; ++i) {
                cum += w[i];
                if (!found && cum > target) { found = true; hit(entry_of(bits_of(v[i]), id0 + p * VN + i)); }
            }
        }
    };
    // Smallest id whose cumulative measure exceeds the target (below the total).  s.group holds the groups' sums and s.total the block's;
    // measure(value, id) as they were formed.  The thread that has the token calls hit(its entry).
    auto locate = [&](auto measure, u64 target, auto hit) {
        u64 before = cluster_sum(&s.total, rank), sum;
        if (target < before || target >= before + s.total) return;               // (the same for the whole block)
        const int groups = (pieces + 31) / 32;
        const u64 mine = t < groups ? s.group[t] : 0;
        before += block_exclusive<u64>(mine, s.scan, sum);
        const uint32_t owner = __ballot_sync(0xffffffffu, before <= target && target < before + mine);
        if (owner == 0) return;
        const int l = __ffs(owner) - 1, p = 32 * (warp * 32 + l) + lane;         // one warp: a lane takes a piece
        float v[VN];
        u64 w[VN];
        values(p, v);
#pragma unroll
        for (int i = 0; i < VN; ++i) w[i] = measure(v[i], id0 + p * VN + i);
        within(p, v, w, __shfl_sync(0xffffffffu, before, l), target, hit);
    };
    auto emit = [&](u64 e, u64 total) {
        a.tokens[row] = id_of_entry(e);
        if (a.logp != nullptr) a.logp[row] = (float)(-(distance(value_of_entry(e)) * 0.69314718055994530942 + log((double)total / kOne)));
    };
    const double u = uf > 0.f ? (double)uf : 0.0;
    auto target_of = [&](u64 total) {
        const u64 x = (u64)(u * (double)total);
        return x < total ? x : total - 1;
    };
    auto share_of = [&](u64 total) {                             // the weight that top-p asks for
        const u64 x = (u64)ceil((double)top_p * (double)total);
        return x > 1 ? x : 1;
    };
    auto kept = [&](float v, int id) {                           // the last step's measure
        if (!near(v) || entry_of(bits_of(v), id) < thr) return (u64)0;
        const double x = distance(v);
        return x <= most || v == top ? weight(x) : (u64)0;
    };
    // The entry of the `want`th token, in order of id, among those with these bits that are kept (the last one's if there are not so many).
    auto tie_border = [&](uint32_t bits, u64 want) {
        const u64 keep_thr = thr;
        auto tie = [&](float v, int id) { return (u64)(bits_of(v) == bits && entry_of(bits, id) >= keep_thr); };
        const int groups = (pieces + 31) / 32;
        u64 mine_all = 0;
        for (int g = warp; g < groups; g += kWarps) {
            const int p = 32 * g + lane;
            uint32_t x = 0;
            if (p < pieces) {
                float v[VN];
                piece(p, v);
#pragma unroll
                for (int i = 0; i < VN; ++i) x += (uint32_t)tie(v[i], id0 + p * VN + i);
            }
            x = __reduce_add_sync(0xffffffffu, x);
            if (lane == 0) { s.group[g] = x; mine_all += x; }
        }
        mine_all = block_sum(lane == 0 ? mine_all : 0, s.scan);
        if (t == 0) s.total = mine_all;
        cluster.sync();
        const u64 ties = cluster_sum(&s.total, C);
        locate(tie, min(want, ties) - 1, [&](u64 e) { *cluster.map_shared_rank(&s.thr, 0) = e; });
        cluster.sync();
        const u64 e = *cluster.map_shared_rank(&s.thr, 0);
        cluster.sync();                                          // (s.total and s.thr may be written again)
        return e;
    };
    // (s.total is not written again before the next row's first meeting of the cluster)
    auto draw = [&](u64 total) { locate(kept, target_of(total), [&](u64 e) { emit(e, total); }); };

    u64 total = 0;
    const float bottom = fmaxf(far, least);                      // (a masked token makes it `far`)
    if constexpr (sizeof(T) == 2) {
        // ---- bf16, limited by top-p or by a large top-k: codes.  (k = 400 / 3000 with top-p 0.95, us: one row by candidates 39 / 64, by code 33 / 33,
        // 142 rows 88 / 168 and 86 / 90; k = 50 by candidates 23 and 53.)  Positive ones from the largest downwards, then negative ones up to the largest magnitude that is
        // near; `code` numbers them in order of falling logit.
        const int top_code = top > 0.f ? (int)(__float_as_uint(top) >> 16) : -1, low_mag = bottom < 0.f ? (int)(__float_as_uint(-bottom) >> 16) : -1;
        constexpr int kLeast = kSide + 128;                      // (no subnormal values among them)
        if ((k == 0 || k > kPairs) && (top_p < 1.f || !(min_p > 0.f)) && (top_code < 0 || top_code >= kLeast) && (low_mag < 0 || low_mag >= kLeast) && top_code + low_mag >= 0) {
            const int neg0 = 32768 - low_mag + 2 * kSide - 1;
            // the place of a code (sign-extended), or -1: none of its own
            auto code = [&](int x) {
                const int b = x >= 0 ? top_code - x : x + neg0;
                return (uint32_t)(b - (x < 0 ? kSide : 0)) < (uint32_t)kSide ? b : -1;
            };
            auto value_of_code = [&](int b) {
                const uint32_t m = b < kSide ? (uint32_t)(top_code - b) : 0x8000u | (uint32_t)(low_mag - (2 * kSide - 1 - b));
                return __uint_as_float(m << 16);
            };
            auto code_exists = [&](int b) { return b < kSide ? top_code >= 0 : low_mag >= 0; };
            auto code_at = [&](const uint4& x, int i) {
                const uint32_t w = i < 2 ? x.x : i < 4 ? x.y : i < 6 ? x.z : x.w;
                return (i & 1) ? (int)w >> 16 : (int)(w << 16) >> 16;
            };
            static_assert(kSide % kMaxCluster == 0, "shares of the codes");
            const int groups = (pieces + 31) / 32;
            bool cuts = false, search = false;                                 // the border is not on a code of its own
            if (top_p < 1.f || k > 0) {
                for (int i = t; i < 2 * kSide; i += kThreads) s.codes[i] = 0;
                if (t == 0) { s.found = 0; s.bin[0] = 0xffffffffu; }
                __syncthreads();
                u64 middle = 0, middle_n = 0;                    // weight and number of the logits without a place: nearer to 0 than all the others
                for (int p = t; p < pieces; p += kThreads) {
                    const uint4 x = raw_piece(p);
                    uint32_t none = 0;
#pragma unroll
                    for (int i = 0; i < VN; ++i) {
                        const int b = code(code_at(x, i));
                        if (b >= 0) atomicAdd(&s.codes[b], 1u);
                        else none |= 1u << i;
                    }
                    for (; none != 0; none &= none - 1) {
                        const float v = value_of(slice[p * VN + __ffs(none) - 1]);
                        if (near(v)) { middle += weight(distance(v)); ++middle_n; }
                    }
                }
                middle = block_sum(middle, s.scan);
                middle_n = block_sum(middle_n, s.scan);
                if (t == 0) { s.middle = middle; s.middle_n = middle_n; }
                cluster.sync();
                // exact cumulative weight over the codes: a block takes as many of them as the others, a thread q
                const int share = 2 * kSide / C, q = (share + kThreads - 1) / kThreads;          // (kSide is a multiple of the cluster's size)
                const int b0 = rank * share + min(t * q, share), b1 = rank * share + min(t * q + q, share);
                // near tokens of a code, and the weight of one
                auto of_code = [&](int b, uint32_t& n) {
                    n = 0;
                    for (int r = 0; r < C; r += 4) {             // (four on their way at once)
                        uint32_t x[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y) x[y] = r + y < C ? cluster.map_shared_rank(s.codes, r + y)[b] : 0;
                        n += x[0] + x[1] + x[2] + x[3];
                    }
                    const float v = value_of_code(b);
                    if (!near(v)) n = 0;
                    return n != 0 ? weight(distance(v)) : 0;
                };
                u64 sum = 0, all;
                uint32_t sum_n = 0, all_n;
#pragma unroll 1
                for (int b = b0; b < b1; ++b) {
                    uint32_t n;
                    const u64 w = of_code(b, n);
                    sum += n * w;
                    sum_n += n;
                }
                const Two middles = cluster_sums(&s.middle, &s.middle_n);
                const u64 mid = middles.x;
                const uint32_t mid_n = (uint32_t)middles.y;
                u64 cum = block_exclusive<u64>(sum, s.scan, all);
                uint32_t cum_n = block_exclusive<uint32_t>(sum_n, s.scan, all_n);
                if (t == 0) { s.all = all; s.all_n = all_n; }
                cluster.sync();
                {
                    const Two sums = cluster_sums(&s.all, &s.all_n);
                    cum += sums.x_before;
                    cum_n += (uint32_t)sums.y_before;
                    total = sums.x + mid;
                    all_n = (uint32_t)sums.y + mid_n;
                }
                // f(code, its tokens, the weight of one, weight and tokens before), of this thread's codes
                auto for_codes = [&](auto f) {
                    u64 c = cum;
                    uint32_t c_n = cum_n;
#pragma unroll 1
                    for (int b = b0; b < b1; ++b) {
                        uint32_t n;
                        const u64 w = of_code(b, n);
                        f(b, n, w, c + (b >= kSide ? mid : 0), c_n + (b >= kSide ? mid_n : 0));
                        c += n * w;
                        c_n += n;
                    }
                };
                auto border = [&](int b, uint32_t want) {
                    for (int r = 0; r < C; ++r) {
                        *cluster.map_shared_rank(&s.bin[0], r) = b;
                        *cluster.map_shared_rank(&s.want, r) = want;
                    }
                };
                const uint32_t most_n = k > 0 && (uint32_t)k < all_n ? (uint32_t)k : 0xffffffffu;
                cuts = top_p < 1.f || most_n != 0xffffffffu;
                if (most_n != 0xffffffffu) {                     // top-k's border; top-p is a share of what is in front of it
                    if (cum_n < most_n && cum_n + sum_n + mid_n >= most_n)
                        for_codes([&](int b, uint32_t n, u64 w, u64 before, uint32_t before_n) {
                            if (before_n >= most_n || before_n + n < most_n) return;
                            if (top_p == 1.f) border(b, most_n - before_n);
                            for (int r = 0; r < C; ++r) *cluster.map_shared_rank(&s.found, r) = before + (most_n - before_n) * w;
                        });
                    cluster.sync();
                    total = s.found;                             // (0: it lies among the logits without a place)
                }
                if (top_p < 1.f && total != 0) {
                    const u64 goal = share_of(total);
                    if (cum < goal && cum + sum + mid >= goal)
                        for_codes([&](int b, uint32_t n, u64 w, u64 before, uint32_t before_n) {
                            const uint32_t there = min(n, most_n - min(most_n, before_n));
                            if (before < goal && before + there * w >= goal) border(b, (uint32_t)((goal - before + w - 1) / w));
                        });
                }
                cluster.sync();                                  // (and the codes' counts have been read)
                search = cuts && s.bin[0] == 0xffffffffu;        // among the logits without a place
                if (cuts && !search) thr = entry_of(bits_of(value_of_code((int)s.bin[0])), kMaxVocab);
            }
            if (!search) {
                // weights by code; what is not kept weighs nothing
                for (int b = t; b < 2 * kSide; b += kThreads) {
                    double w = 0.0;
                    if (code_exists(b)) {
                        const float v = value_of_code(b);
                        if (near(v) && (thr == 0 || bits_of(v) >= (uint32_t)(thr >> 32))) {
                            const double x = distance(v);
                            if (x <= most || v == top) w = weight_d(x);
                        }
                    }
                    s.code_w[b] = w;
                }
                __syncthreads();
                // the border's tokens, of which the first s.want in order of id are kept, are counted apart
                const float thr_v = thr != 0 ? value_of_entry(thr) : -kMost;
                const Piece<T> test(thr_v);
                uint16_t* ties = s.cand;                         // of every group
                u64 sums = 0;
                uint32_t tie_sums = 0;
                for (int g = warp; g < groups; g += kWarps) {
                    const int p = 32 * g + lane;
                    double sum = 0.0;
                    uint32_t n_ties = 0;
                    if (p < pieces) {
                        const uint4 x = raw_piece(p);
                        uint32_t rest = 0;                       // looked at one by one
                        if (thr == 0) {
#pragma unroll
                            for (int i = 0; i < VN; ++i) {
                                const int b = code(code_at(x, i));
                                sum += s.code_w[max(b, 0)] * (b >= 0 ? 1.0 : 0.0);
                                rest |= b < 0 ? 1u << i : 0u;
                            }
                        } else {
                            rest = test.mask(x);
                        }
                        for (; rest != 0; rest &= rest - 1) {
                            const int at = p * VN + __ffs(rest) - 1, b = code((int)reinterpret_cast<const int16_t*>(slice)[at]);
                            const float v = value_of(slice[at]);
                            if (v == thr_v) ++n_ties;
                            else if (b >= 0) sum += s.code_w[b];
                            else sum += (double)kept(v, id0 + at);
                        }
                    }
                    u64 w = (u64)sum;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
                    if (thr != 0) n_ties = __reduce_add_sync(0xffffffffu, n_ties);
                    if (lane == 0) { s.group[g] = w; ties[g] = (uint16_t)n_ties; }
                    sums += w;
                    tie_sums += n_ties;
                }
                sums = block_sum(lane == 0 ? sums : 0, s.scan);
                if (t == 0) s.total = sums;
                auto by_code = [&](float v, int id) {
                    const int b = code((int)__float_as_uint(v) >> 16);
                    return b >= 0 ? (u64)s.code_w[b] : kept(v, id);
                };
                if (thr == 0) {
                    cluster.sync();
                    total = cluster_sum(&s.total, C);
                    locate(by_code, target_of(total), [&](u64 e) { emit(e, total); });
                    return;
                }
                const uint32_t here = (uint32_t)block_sum(lane == 0 ? tie_sums : 0, s.scan), want = s.want;
                const u64 w_tie = (u64)s.code_w[s.bin[0]];       // (0 where min-p excludes it)
                if (t == 0) s.ties = here;
                cluster.sync();
                auto kept_ties = [&](uint32_t before, uint32_t n) { return min(n, want - min(want, before)); };
                u64 start, mine;
                uint32_t ties_start;
                {                                                // a lane does a block's
                    const uint32_t y = lane < C ? *cluster.map_shared_rank(&s.ties, lane) : 0;
                    u64 x = lane < C ? *cluster.map_shared_rank(&s.total, lane) : 0;
                    uint32_t before = y;
#pragma unroll
                    for (int o = 1; o < kMaxCluster; o <<= 1) {
                        const uint32_t z = __shfl_up_sync(0xffffffffu, before, o);
                        if (lane >= o) before += z;
                    }
                    before -= y;
                    x += kept_ties(before, y) * w_tie;
                    total = sum_lanes(x);
                    start = sum_lanes(lane < rank ? x : 0);
                    mine = __shfl_sync(0xffffffffu, x, rank);
                    ties_start = __shfl_sync(0xffffffffu, before, rank);
                }
                const u64 target = target_of(total);
                if (target < start || target >= start + mine) return;            // (the same for the whole block)
                const uint32_t y = t < groups ? ties[t] : 0;
                uint32_t unused;
                ties_start += block_exclusive<uint32_t>(y, s.scan, unused);
                const u64 x = t < groups ? s.group[t] + kept_ties(ties_start, y) * w_tie : 0;
                start += block_exclusive<u64>(x, s.scan, mine);
                const uint32_t owner = __ballot_sync(0xffffffffu, start <= target && target < start + x);
                if (owner == 0) return;
                const int l = __ffs(owner) - 1, p = 32 * (warp * 32 + l) + lane;
                float v[VN];
                u64 w[VN];
                values(p, v);
                uint32_t n_ties = 0;
#pragma unroll
                for (int i = 0; i < VN; ++i) n_ties += v[i] == thr_v ? 1 : 0;
                uint32_t at = n_ties;                            // ties before this lane's
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t z = __shfl_up_sync(0xffffffffu, at, o);
                    if (lane >= o) at += z;
                }
                at += __shfl_sync(0xffffffffu, ties_start, l) - n_ties;
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    w[i] = by_code(v[i], 0);
                    if (v[i] == thr_v) w[i] = at++ < want ? w_tie : 0;
                }
                within(p, v, w, __shfl_sync(0xffffffffu, start, l), target, [&](u64 e) { emit(e, total); });
                return;
            }
            for (int i = t; i < kBins; i += kThreads) s.count[i] = 0;
            __syncthreads();
        }
    }

    // ---- no filter
    if (k == 0 && top_p == 1.f && !(min_p > 0.f)) {
        draw(weigh(std::false_type(), CUDART_INF));
        return;
    }

    // bins of distance, by a product that rises with it
    const float span = top - bottom;
    const float inv = span > 1e-30f && span < 1e36f ? (float)kBins / span : 0.f;
    auto place = [&](float v) { return (top - v) * inv; };
    auto bin_of = [&](float v) { return min(kBins - 1, (int)place(v)); };
    const float unit = (float)c2;                                // log2 distance of 1
    uint32_t c[kPerThread];
    auto gather_counts = [&]() {                                 // the cluster's counts of this thread's bins
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) c[i] = 0;
        for (int r = 0; r < C; r += 4) {                         // (four on their way at once)
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = r + i < C ? *reinterpret_cast<const uint4*>(cluster.map_shared_rank(s.count, r + i) + t * kPerThread) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) { c[0] += x[i].x; c[1] += x[i].y; c[2] += x[i].z; c[3] += x[i].w; }
        }
        static_assert(kPerThread == 4, "one 16-byte read of the counts");
    };
    auto list = [&](int p, uint32_t mask) {                      // tokens of a piece among the block's candidates
        uint32_t at = atomicAdd(&s.n_cand, (uint32_t)__popc(mask));
        for (; mask != 0; mask &= mask - 1, ++at)
            if (at < kGather) s.cand[at] = (uint16_t)(p * VN + __ffs(mask) - 1);
    };
    // The blocks' candidates into the first one's memory, if they fit; their number.  (Their order there has no influence.)
    auto send = [&]() {
        __syncthreads();
        const uint32_t mine = s.n_cand;
        if (t == 0) s.n_in = atomicAdd(cluster.map_shared_rank(&s.n_gather[parity], 0), mine);
        __syncthreads();
        const uint32_t base = s.n_in;
        if (base + mine <= kGather) {
            u64* to = cluster.map_shared_rank(s.entry, 0) + base;
            for (int i = t; i < (int)mine; i += kThreads) to[i] = entry_of(bits_of(value_of(slice[s.cand[i]])), id0 + s.cand[i]);
        }
        cluster.sync();
        return (int)*cluster.map_shared_rank(&s.n_gather[parity], 0);
    };
    auto key_at = [&](int i) { return s.entry[i]; };

    // ---- top-p alone (or with min-p): the border's bins, then one pass over the weights
    if (k == 0 && top_p < 1.f) {
        for (int p = t; p < pieces; p += kThreads) {
            float v[VN];
            piece(p, v);
#pragma unroll
            for (int i = 0; i < VN; ++i)
                if (near(v[i])) atomicAdd(&s.count[bin_of(v[i])], 1u);
        }
        if (t < 2) s.bin[t] = s.mid[t] = kBins - 1;
        if (t == 0) { s.all = 0; s.total = 0; s.n_in = 0; }
        cluster.sync();
        gather_counts();
        {
            // A bin's weights lie between those of its two ends (1.6 % apart at most), which bounds the cumulative weight; their middle is closer
            // where many tokens count.
            const float w = inv > 0.f ? unit / inv : 0.f;
            float x[3][kPerThread], cum[3] = {0.f, 0.f, 0.f}, all[3];
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                const int b = t * kPerThread + i;
                x[0][i] = (float)c[i] * exp2f(-(float)b * w);
                x[1][i] = b == kBins - 1 ? 0.f : (float)c[i] * exp2f(-(float)(b + 1) * w);
                x[2][i] = 0.5f * (x[0][i] + x[1][i]);
#pragma unroll
                for (int y = 0; y < 3; ++y) cum[y] += x[y][i];
            }
            block_exclusive3(cum, all, reinterpret_cast<float*>(s.scan));
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
#pragma unroll
                for (int y = 0; y < 3; ++y) cum[y] += x[y][i];
                const uint32_t b = (uint32_t)(t * kPerThread + i);
                if (c[i] > 0) {
                    if (cum[0] * 1.0001f >= top_p * all[1]) atomicMin(&s.bin[0], b);
                    if (cum[1] >= top_p * all[0] * 1.0001f) atomicMin(&s.bin[1], b);
                    if (cum[2] >= (top_p - 1e-3f) * all[2]) atomicMin(&s.mid[0], b);
                    if (cum[2] >= (top_p + 1e-3f) * all[2]) atomicMin(&s.mid[1], b);
                }
            }
        }
        __syncthreads();
        int b0 = s.bin[0], b1 = s.bin[1];
        {
            uint32_t in = 0;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) in += t * kPerThread + i >= b0 && t * kPerThread + i <= b1 ? c[i] : 0;
            in = __reduce_add_sync(0xffffffffu, in);
            if (lane == 0 && in != 0) atomicAdd(&s.n_in, in);
        }
        __syncthreads();
        if (s.n_in > kGather) { b0 = s.mid[0]; b1 = s.mid[1]; }  // (a border outside of them is noticed below)
        const float from = b0 > 0 ? (float)b0 : -CUDART_INF_F, to = b1 == kBins - 1 ? CUDART_INF_F : (float)(b1 + 1);
        double all_d = 0.0;                                      // (of some hundred tokens: exact)
        u64 sum_before = 0;
        const int groups = (pieces + 31) / 32;
        for (int g = warp; g < groups; g += kWarps) {
            const int p = 32 * g + lane;
            double first_d = 0.0;
            if (p < pieces) {
                float v[VN];
                piece(p, v);
                uint32_t mask = 0;
#pragma unroll
                for (int i = 0; i < VN; ++i) {
                    const float y = place(v[i]);
                    const bool in = near(v[i]), first = in && y < from;
                    const double w = weight_d(distance(in ? v[i] : top));
                    if (in) all_d += w;
                    if (first) first_d += w;
                    mask |= in && !first && y < to ? 1u << i : 0u;
                }
                if (mask != 0) list(p, mask);
            }
            u64 before = (u64)first_d;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
            if (lane == 0) { s.group[g] = before; sum_before += before; }
        }
        u64 sum_all = (u64)all_d;
        for (int o = 16; o > 0; o >>= 1) sum_all += __shfl_xor_sync(0xffffffffu, sum_all, o);
        if (lane == 0) { atomicAdd(&s.all, sum_all); atomicAdd(&s.total, sum_before); }
        const int m = send();
        const Two sums = cluster_sums(&s.total, &s.all);
        const u64 before = sums.x;
        total = sums.y;
        const u64 goal = share_of(total);
        if (m <= kGather && before < goal) {
            if (rank == 0) {
                const u64 e = block_select(s, m, key_at, [&](int i) { return weight(distance(value_of_entry(s.entry[i]))); }, goal - before);
                if (t == 0) s.thr = e;
            }
            cluster.sync();
            thr = *cluster.map_shared_rank(&s.thr, 0);
            if (thr != 0) {
                if (distance(value_of_entry(thr)) <= most) {
                    // what is kept of the bins joins its groups' sums
                    u64 mine = 0;
                    for (int i = t; i < (int)s.n_cand; i += kThreads) {
                        const float v = value_of(slice[s.cand[i]]);
                        if (entry_of(bits_of(v), id0 + s.cand[i]) >= thr) {
                            const u64 x = weight(distance(v));
                            atomicAdd(&s.group[s.cand[i] / (32 * VN)], x);
                            mine += x;
                        }
                    }
                    mine = block_sum(mine, s.scan);
                    if (t == 0) s.total += mine;
                    cluster.sync();
                    total = cluster_sum(&s.total, C);
                } else {                                         // min-p cuts deeper
                    total = weigh(std::true_type(), most);
                }
                draw(total);
                return;
            }
        }
        cluster.sync();
    }

    // ---- top-k, min-p: candidates, tokens that may be kept
    float bound = far;
    if (min_p > 0.f && top_p == 1.f) bound = fmaxf(bound, value_at(most + 1e-6));        // (top-p counts the weight of what min-p drops)
    if (k > 0) {
        for (int p = t; p < pieces; p += kThreads) {
            const float m = Piece<T>::largest(raw_piece(p));
            if (near(m)) atomicAdd(&s.count[bin_of(m)], 1u);
        }
        if (t == 0) s.bin[0] = kBins;
        cluster.sync();
        gather_counts();
        uint32_t all, cum = block_exclusive<uint32_t>(c[0] + c[1] + c[2] + c[3], s.scan, all);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            if (cum < (uint32_t)k && cum + c[i] >= (uint32_t)k) s.bin[0] = t * kPerThread + i;
            cum += c[i];
        }
        __syncthreads();
        // the logits of the bins up to that one: not below this (rounded down; one bin more for the product's rounding)
        if (inv > 0.f && s.bin[0] < kBins - 2) bound = fmaxf(bound, top - (float)(s.bin[0] + 2) / inv * 1.000001f);
    }
    if (!(k == 0 && top_p < 1.f)) {                              // (top-p alone comes here only if the cluster has to search for its border)
        const Piece<T> test(bound);
        for (int p = t; p < pieces; p += kThreads) {
            const uint32_t mask = test.mask(raw_piece(p));
            if (mask != 0) list(p, mask);
        }
        const int m = send();
        if (m <= kGather) {
            if (rank != 0) return;
            // ---- the first block alone
            auto w_at = [&](int i) { const float v = value_of_entry(s.entry[i]); return near(v) ? weight(distance(v)) : (u64)0; };
            if (m <= kPairs) {                                   // compared pairwise, `per` threads a candidate
                int shift = 1;
                while (shift < 5 && (m << shift) <= kThreads / 2) ++shift;
                const int per = 1 << shift, i = t >> shift;
                const bool there = i < m, speaks = there && (t & (per - 1)) == 0;        // (one of them speaks for the candidate)
                const u64 e = there ? s.entry[i] : 0;
                u64 w = there ? w_at(i) : 0, before = 0;
                if (speaks) s.mass[i] = w;
                __syncthreads();
                int front = 0;                                   // how many, and how much weight, lie in front of it
                if (there)
                    for (int y = t & (per - 1); y < m; y += per)
                        if (s.entry[y] > e) { ++front; before += s.mass[y]; }
                for (int o = per / 2; o > 0; o >>= 1) {
                    front += __shfl_xor_sync(0xffffffffu, front, o);
                    before += __shfl_xor_sync(0xffffffffu, before, o);
                }
                if (k > 0 && front >= k) w = 0;
                if (top_p < 1.f && before >= share_of(block_sum(speaks ? w : 0, s.scan))) w = 0;         // (k > 0)
                const float v = value_of_entry(e);
                if (w != 0 && !(distance(v) <= most || v == top)) w = 0;
                const u64 whole = block_sum(speaks ? w : 0, s.scan), target = target_of(whole);
                if (speaks) s.mass[i] = w;
                __syncthreads();
                before = 0;                                      // weight of the lower ids that are kept
                if (there)
                    for (int y = t & (per - 1); y < m; y += per)
                        if ((uint32_t)s.entry[y] > (uint32_t)e) before += s.mass[y];
                for (int o = per / 2; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
                if (speaks && before <= target && target < before + w) emit(e, whole);
                return;
            }
            if (k > 0 && m > k) thr = block_select(s, m, key_at, [&](int) { return (u64)1; }, (u64)k);
            if (top_p < 1.f) {                                   // (k > 0)
                u64 mine = 0;
                for (int i = t; i < m; i += kThreads) mine += s.entry[i] >= thr ? w_at(i) : 0;
                const u64 goal = share_of(block_sum(mine, s.scan)), was = thr;
                thr = block_select(s, m, key_at, [&](int i) { return s.entry[i] >= was ? w_at(i) : (u64)0; }, goal);
            }
            auto kept_at = [&](int i) { return kept(value_of_entry(s.entry[i]), id_of_entry(s.entry[i])); };
            u64 mine = 0;
            for (int i = t; i < m; i += kThreads) mine += kept_at(i);
            const u64 all = block_sum(mine, s.scan);
            // in order of id: the inverted id as the key
            const u64 id = block_select(s, m, [&](int i) { return s.entry[i] & 0xffffffffull; }, kept_at, target_of(all) + 1);
            for (int i = t; i < m; i += kThreads)
                if ((s.entry[i] & 0xffffffffull) == id) emit(s.entry[i], all);
            return;
        }
        cluster.sync();
    }

    // ---- more candidates: the whole cluster.  Moves thr to the end of the shortest leading run whose measure is at least the goal:
    // weight (by_mass) or tokens.
    auto select = [&](bool by_mass, u64 goal) {
        for (int i = t; i < kBins; i += kThreads) s.count[i] = 0;
        if (t < 2) s.bin[t] = kBins - 1;
        if (t == 0) { s.hi = 0; s.lo = 0xffffffffu; s.n_list = 0; s.sum[0] = 0; }
        __syncthreads();
        const float thr_v = thr != 0 ? value_of_entry(thr) : -kMost;
        // f(value, id, bin) of the tokens that can be kept
        auto for_tokens = [&](auto f) {
            for (int p = t; p < pieces; p += kThreads) {
                float v[VN];
                piece(p, v);
#pragma unroll
                for (int i = 0; i < VN; ++i)
                    if (v[i] >= bound && near(v[i]) && v[i] >= thr_v) {
                        const int id = id0 + p * VN + i;
                        if (thr == 0 || entry_of(bits_of(v[i]), id) >= thr) f(v[i], id, bin_of(v[i]));
                    }
            }
        };
        for_tokens([&](float, int, int b) { atomicAdd(&s.count[b], 1u); });
        cluster.sync();
        gather_counts();
        const uint32_t mine = c[0] + c[1] + c[2] + c[3];
        uint32_t all;
        const uint32_t count_before = block_exclusive<uint32_t>(mine, s.scan, all);
        if (!by_mass && all <= goal) { cluster.sync(); return; }         // everything that has weight is kept
        if (by_mass) {
            // a bin's weights lie between those of its two ends: bounds of the cumulative weight, with a margin for their rounding
            const float w = inv > 0.f ? unit / inv : 0.f, want = (float)((double)goal / kOne);
            float up[kPerThread], down[kPerThread], up_mine = 0.f, down_mine = 0.f, unused;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                const int b = t * kPerThread + i;
                up[i] = (float)c[i] * exp2f(-(float)b * w);
                down[i] = b == kBins - 1 ? 0.f : (float)c[i] * exp2f(-(float)(b + 1) * w);
                up_mine += up[i]; down_mine += down[i];
            }
            float cu = block_exclusive<float>(up_mine, s.scan, unused), cd = block_exclusive<float>(down_mine, s.scan, unused);
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                cu += up[i]; cd += down[i];
                if (c[i] > 0 && cu * 1.001f >= want) atomicMin(&s.bin[0], t * kPerThread + i);
                if (c[i] > 0 && cd * 0.999f >= want) atomicMin(&s.bin[1], t * kPerThread + i);
            }
        } else {
            uint32_t cum = count_before;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                if (cum < goal && cum + c[i] >= goal) s.bin[0] = s.bin[1] = t * kPerThread + i;
                cum += c[i];
            }
        }
        __syncthreads();
        const int b0 = s.bin[0], b1 = s.bin[1];
        // tokens inside: few enough for the list?  (the same number in every block)
        uint32_t in = 0, n_in;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) in += t * kPerThread + i >= b0 && t * kPerThread + i <= b1 ? c[i] : 0;
        block_exclusive<uint32_t>(in, s.scan, n_in);
        auto measure = [&](float v) { return by_mass ? weight(distance(v)) : (u64)1; };
        auto put = [&](u64 e) {
            const uint32_t at = atomicAdd(cluster.map_shared_rank(&s.n_list, 0), 1u);
            if (at < kList) cluster.map_shared_rank(s.wide.list, 0)[at] = e;
        };
        u64 part = 0;                                            // measure before
        uint32_t lo = 0xffffffffu, hi = 0;
        for_tokens([&](float v, int id, int b) {
            if (b < b0) part += measure(v);
            else if (b <= b1) {
                const uint32_t x = bits_of(v);
                lo = min(lo, x);
                hi = max(hi, x);
                if (n_in <= kList) put(entry_of(x, id));
            }
        });
        for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) { atomicAdd(&s.sum[0], part); atomicMin(&s.lo, lo); atomicMax(&s.hi, hi); }
        cluster.sync();
        u64 before = cluster_sum(&s.sum[0], C);
        lo = __reduce_min_sync(0xffffffffu, lane < C ? *cluster.map_shared_rank(&s.lo, lane) : 0xffffffffu);
        hi = __reduce_max_sync(0xffffffffu, lane < C ? *cluster.map_shared_rank(&s.hi, lane) : 0);
        // divide the range of logit bits until the list holds what is left, or one value is
        while (n_in > kList && lo < hi) {
            const int shift = max(0, 21 - __clz(hi - lo));       // (hi - lo) >> shift < 2048
            for (int i = t; i < kBins; i += kThreads) { s.count[i] = 0; s.wide.mass[i] = 0; }
            if (t == 0) s.bin[0] = 0xffffffffu;
            cluster.sync();                                      // (everyone has read the counts and sums of the step before)
            for_tokens([&](float v, int, int) {
                const uint32_t x = bits_of(v);
                if (x < lo || x > hi) return;
                const int b = (int)((hi - x) >> shift);
                atomicAdd(&s.count[b], 1u);
                if (by_mass) atomicAdd(&s.wide.mass[b], measure(v));
            });
            cluster.sync();
            gather_counts();
            u64 m[kPerThread], m_mine = 0, m_all;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                m[i] = by_mass ? 0 : c[i];
                for (int r = 0; r < C && by_mass; ++r) m[i] += cluster.map_shared_rank(s.wide.mass, r)[t * kPerThread + i];
                m_mine += m[i];
            }
            u64 cum = before + block_exclusive<u64>(m_mine, s.scan, m_all);
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                if (cum < goal && cum + m[i] >= goal) {
                    s.bin[0] = t * kPerThread + i;
                    s.sum[0] = cum;
                    s.sum[1] = c[i];
                }
                cum += m[i];
            }
            __syncthreads();
            const uint32_t b = s.bin[0];
            if (b == 0xffffffffu) break;                         // (the border lies behind: all of it is kept)
            before = s.sum[0];
            n_in = (uint32_t)s.sum[1];
            const uint32_t top_key = hi - (b << shift);
            lo = max(lo, top_key - min(top_key, (1u << shift) - 1u));
            hi = top_key;
            if (n_in <= kList) {
                if (t == 0) s.n_list = 0;
                cluster.sync();
                for_tokens([&](float v, int id, int) {
                    const uint32_t x = bits_of(v);
                    if (x >= lo && x <= hi) put(entry_of(x, id));
                });
            }
            cluster.sync();
        }
        if (n_in <= kList) {
            if (rank == 0) {
                // entry i is the border if the measure up to it reaches the goal and the measure before it does not
                const int m = min((int)n_in, (int)s.n_list);
                if (t == 0) s.thr = thr;
                if (t < m) s.wide.list_w[t] = measure(value_of_entry(s.wide.list[t]));
                __syncthreads();
                if (t < m) {
                    const u64 e = s.wide.list[t];
                    u64 cum = before;
                    for (int i = 0; i < m; ++i) cum += s.wide.list[i] > e ? s.wide.list_w[i] : 0;
                    if (cum < goal && cum + s.wide.list_w[t] >= goal) s.thr = e;
                }
            }
            cluster.sync();
            thr = *cluster.map_shared_rank(&s.thr, 0);
        } else if (lo == hi) {
            // equal logits: the first so many of them in order of id
            const u64 w = measure(of_bits(lo));
            thr = tie_border(lo, goal > before + w ? (goal - before + w - 1) / w : 1);
        }
        cluster.sync();
    };

    if (k > 0) {
        select(false, (u64)k);
        if (top_p < 1.f) total = weigh(std::true_type(), CUDART_INF);
    }
    if (top_p < 1.f) select(true, share_of(total));
    draw(weigh(std::true_type(), most));
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    Shared& s = *reinterpret_cast<Shared*>(smem);
    const cg::cluster_group cluster = cg::this_cluster();
    const int C = cluster.num_blocks();
    if (threadIdx.x < 32) s.root[threadIdx.x] = exp2(45.0 - (double)threadIdx.x / 32.0);
    if (threadIdx.x < 2) s.n_gather[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&s.answer_bar), 1);
        fence_barrier_init();
    }
    pdl_launch_dependents();
    pdl_wait();
    int row = blockIdx.x / C;
    for (int parity = 0, next; row >= 0; row = next, parity ^= 1) {
        __syncthreads();                                         // (the row before is done with the block's memory)
        if (a.more && threadIdx.x == 0 && cluster.block_rank() == 0) ask_for_row(s);
        sample_row<T>(a, cluster, s, smem + (sizeof(Shared) + 15) / 16 * 16, row, next, parity);
    }
    cluster.sync();                                              // nobody reads a block's memory after it has ended
    // No row keeps what its places held before the call: a row that was done, by this cluster or by another up to now, counts as undone too.
    if (row == kNoAnswer && cluster.block_rank() == 0)
        for (int i = threadIdx.x; i < a.rows; i += kThreads) {
            a.tokens[i] = -1;
            if (a.logp != nullptr) a.logp[i] = CUDART_NAN_F;
        }
}

constexpr size_t kHalfSm = 113 * 1024 - 128;     // dynamic shared memory of a block that shares its SM with another

// Blocks of a row: slices of up to 64 KB, so that two blocks share an SM; more blocks while the GPU has room for them.  Slices of 32 KB: 448 rows of
// 128256 bf16 logits 233 instead of 166 us (temperature) and 354 instead of 225 (top-p), the same where rows are few.  As few blocks as the slices
// need: one row of 32000 bf16 logits 25 instead of 16 us (temperature) and 34 instead of 25 (top-p), 32 rows of 128256 33 instead of 31
// and 41 instead of 38 (but 23 instead of 29 with top-k, where one block does most of the work).
int blocks_of_row(int rows, int vocab, int elt) {
    int c = 1;
    while (c < kMaxCluster && ((long long)vocab * elt > (long long)c * 64 * 1024 || (vocab > c * 4096 && (long long)rows * c < device_sm_count()))) c *= 2;
    return c;
}

// Clusters of c = 1, 2, 4, 8 blocks that the current device holds at once, with blocks of kHalfSm bytes or (large) more.
template <typename T>
int resident_clusters(const cudaLaunchConfig_t& cfg, int c, bool large) {
    static std::atomic<int> known[PerDeviceOnce::kMaxDevices][2][4];
    int dev = 0, n = 0, slot = c == 1 ? 0 : c == 2 ? 1 : c == 4 ? 2 : 3;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= PerDeviceOnce::kMaxDevices) return 1;
    std::atomic<int>& k = known[dev][large ? 1 : 0][slot];
    n = k.load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveClusters(&n, sample_kernel<T>, &cfg) != cudaSuccess || n <= 0) { cudaGetLastError(); n = device_sm_count() / c; }
        k.store(n > 0 ? n : 1, std::memory_order_relaxed);
    }
    return n > 0 ? n : 1;
}

template <typename T>
beagle_status launch_sample(SampleArgs a, cudaStream_t stream) {
    const int c = blocks_of_row(a.rows, a.vocab, (int)sizeof(T));
    a.slice = ((a.vocab + c - 1) / c + 7) / 8 * 8;
    const size_t bytes = (sizeof(Shared) + 15) / 16 * 16 + (size_t)(a.slice + 32) * sizeof(T);
    const bool large = bytes > kHalfSm;
    static PerDeviceOnce attr;
    constexpr size_t kLarge = 200 * 1024;
    static_assert((sizeof(Shared) + 15) / 16 * 16 + (kMaxVocab / kMaxCluster + 40) * sizeof(T) <= kLarge, "the largest slice");
    if (!attr.ensure([] { return cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLarge) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)c);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = large ? kLarge : kHalfSm;     // (what the number below is known for)
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = c;
    attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = 1;
    const int fit = resident_clusters<T>(cfg, c, large);
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    a.more = a.rows > fit;
    cfg.dynamicSmemBytes = bytes;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a) == cudaSuccess && cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

}  // namespace

}  // namespace beagle

using namespace beagle;

extern "C" beagle_status beagle_sample(const void* logits_dev, int32_t logits_dtype, int32_t rows, int32_t vocab, int64_t row_stride,
                                       const float* temperature_dev, const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev,
                                       const float* u_dev, int32_t* tokens_out_dev, float* logp_out_dev, void* stream) {
    if (logits_dtype != BEAGLE_FP32 && logits_dtype != BEAGLE_BF16) return BEAGLE_ERR_INVALID_ARG;
    if (rows < 0 || vocab <= 0 || row_stride < vocab) return BEAGLE_ERR_INVALID_ARG;
    if (vocab > kMaxVocab) return BEAGLE_ERR_SHAPE;
    if (rows > 0x7fffffff / kMaxCluster) return BEAGLE_ERR_CAPACITY;     // (rows and blocks are counted in 32 bits)
    if (rows == 0) return BEAGLE_OK;
    if (logits_dev == nullptr || u_dev == nullptr || tokens_out_dev == nullptr) return BEAGLE_ERR_INVALID_ARG;
    if (((uintptr_t)logits_dev & (logits_dtype == BEAGLE_BF16 ? 1 : 3)) ||
        (((uintptr_t)temperature_dev | (uintptr_t)top_k_dev | (uintptr_t)top_p_dev | (uintptr_t)min_p_dev | (uintptr_t)u_dev | (uintptr_t)tokens_out_dev |
          (uintptr_t)logp_out_dev) & 3))
        return BEAGLE_ERR_INVALID_ARG;
    SampleArgs a{logits_dev, row_stride, rows, vocab, 0, 0, kSpinLimit, temperature_dev, top_p_dev, min_p_dev, u_dev, top_k_dev, tokens_out_dev, logp_out_dev};
#ifdef BEAGLE_BOUNDS_CHECK
    if (const char* tries = getenv("BEAGLE_SAMPLE_TRIES")) a.tries = (uint32_t)strtoul(tries, nullptr, 10);      // (tests of the wait that runs out)
#endif
    return logits_dtype == BEAGLE_BF16 ? launch_sample<bf16>(a, static_cast<cudaStream_t>(stream)) : launch_sample<float>(a, static_cast<cudaStream_t>(stream));
}
