// One token per row of logits from a given uniform number, after temperature, top-k, top-p and min-p (beagle_sample).
//
// All three filters keep a leading run of the tokens in order of (logit falling, id rising), so the kept set is one threshold on the
// 64-bit entry (order-preserving logit bits, inverted id), found without sorting; the draw is an inverse CDF in order of id.
//
// Weights exp((l - largest) / T) are formed in double precision and rounded to integers, 2^45 for the largest: sums of up to 2^18 of
// them fit 64 bits and do not depend on their order, so neither the number of thread blocks of a row nor timing has an influence on
// the result, and a token differs from exact arithmetic's only if a sum comes within some 2^-45 of a border.
//
// A row belongs to a cluster of up to 8 thread blocks, each of which keeps its slice of the logits in shared memory: they are read
// from memory once (the floor of the call), all passes after that stay on chip.  Per filter: a histogram of the tokens' distance from
// the largest (2048 bins, 32-bit counts); for top-p the bins' counts bracket their weights, which leaves a few bins in which the
// border can lie; one pass forms the exact weights before, inside and behind them; the tokens inside (usually a few dozen) are gathered
// by the first block, which finds the border by comparing all pairs.  More than kList of them: their range of logit bits is
// divided further, by 2048 a level with exact weights, until few are left, or only equal logits, which are taken in order of id.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "../../include/beagle.h"
#include "common.cuh"
#include "tensor_map.h"

namespace beagle {

namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048, kPerThread = kBins / kThreads;
constexpr int kList = kThreads;          // tokens that the first block compares pairwise
constexpr int kMaxCluster = 8;
constexpr int kMaxVocab = 1 << 18;
constexpr double kOne = 35184372088832.0;        // 2^45
constexpr float kFar = 47.f;             // log2 distance from which on the weight is 0 (2^45 * 2^-47 rounds to 0)

struct SampleArgs {
    const void* logits;
    long long stride;
    int vocab, slice;                    // slice: tokens of a block (a multiple of 8)
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* tokens;
    float* logp;
};

struct Shared {
    u64 mass[kBins];
    uint32_t count[kBins];
    u64 list[kList], list_w[kList];
    double root[32];                     // 2^(-j / 32)
    u64 scan[kWarps + 1];
    u64 best, sum[3], total, thr, found;
    uint32_t least, lo, hi, n_list, bin[2];
};

__device__ __forceinline__ float value_of(float v) { return v != v ? -CUDART_INF_F : v; }
__device__ __forceinline__ float value_of(bf16 v) { return value_of(__bfloat162float(v)); }
// Order-preserving bits; -0 and +0 are equal.
__device__ __forceinline__ uint32_t bits_of(float v) {
    uint32_t u = __float_as_uint(v);
    u = u == 0x80000000u ? 0u : u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float of_bits(uint32_t u) { return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u); }
__device__ __forceinline__ u64 entry_of(uint32_t bits, int id) { return ((u64)bits << 32) | (0xffffffffu - (uint32_t)id); }

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

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const __grid_constant__ SampleArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    Shared& s = *reinterpret_cast<Shared*>(smem);
    constexpr int VN = 16 / (int)sizeof(T);
    T* slice = reinterpret_cast<T*>(smem + (sizeof(Shared) + 15) / 16 * 16);
    cg::cluster_group cluster = cg::this_cluster();
    const int C = cluster.num_blocks(), rank = cluster.block_rank(), row = blockIdx.x / C, t = threadIdx.x, lane = t & 31;
    pdl_launch_dependents();
    pdl_wait();

    // ---- the slice into shared memory, at the same distance from a 16-byte border as in memory; the largest and the least finite logit
    const int first = min(rank * a.slice, a.vocab), n = min(a.slice, a.vocab - first);
    const T* src = static_cast<const T*>(a.logits) + (size_t)row * a.stride + first;
    const int pad = (int)(((uintptr_t)src & 15) / sizeof(T));
    slice += pad;
    u64 best = 0;
    float least = CUDART_INF_F;
    auto look = [&](T raw, int i) {
        const float v = value_of(raw);
        const u64 k = argmax_key(v, first + i);
        best = k > best ? k : best;
        if (v > -CUDART_INF_F) least = fminf(least, v);
    };
    {
        const int head = min(n, (VN - pad) % VN), vecs = (n - head) / VN, tail = head + vecs * VN;
        if (t < head) { slice[t] = src[t]; look(src[t], t); }
        if (t < n - tail) { slice[tail + t] = src[tail + t]; look(src[tail + t], tail + t); }
        for (int i0 = t; i0 < vecs; i0 += 4 * kThreads) {
            uint4 v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (i0 + x * kThreads < vecs) v[x] = ld_act_stream16(src + head + (i0 + x * kThreads) * VN);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (i0 + x * kThreads < vecs) {
                    const int at = head + (i0 + x * kThreads) * VN;
                    *reinterpret_cast<uint4*>(slice + at) = v[x];
                    const T* e = reinterpret_cast<const T*>(&v[x]);
#pragma unroll
                    for (int y = 0; y < VN; ++y) look(e[y], at + y);
                }
        }
    }
    if (t == 0) { s.best = 0; s.least = 0xffffffffu; }
    if (t < 32) s.root[t] = exp2(-(double)t / 32.0);
    __syncthreads();
    best = warp_max_u64(best);
    for (int o = 16; o > 0; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
    if (lane == 0) { atomicMax(&s.best, best); atomicMin(&s.least, bits_of(least)); }
    cluster.sync();
    uint32_t least_bits = 0xffffffffu;
    for (int i = 0; i < C; ++i) {
        const u64 b = *cluster.map_shared_rank(&s.best, i);
        best = b > best ? b : best;
        least_bits = min(least_bits, *cluster.map_shared_rank(&s.least, i));
    }
    const float top = of_bits((uint32_t)(best >> 32));           // (argmax_key's bits are bits_of's)
    const int top_id = argmax_key_index(best);

    // ---- the row's parameters
    const uint32_t temp_bits = a.temperature != nullptr ? __float_as_uint(__ldcg(a.temperature + row)) : __float_as_uint(1.f);
    const bool drawn = temp_bits - 1u < 0x7f800000u;             // above 0, infinity included
    int k = a.top_k != nullptr ? __ldcg(a.top_k + row) : 0;
    const float top_p = a.top_p != nullptr ? __ldcg(a.top_p + row) : 1.f;
    const float min_p = a.min_p != nullptr ? __ldcg(a.min_p + row) : 0.f;
    if (top_p <= 0.f || min_p > 1.f) k = 1;                      // only the first
    if (!drawn || k == 1 || top == -CUDART_INF_F) {
        if (rank == 0 && t == 0) {
            a.tokens[row] = top == -CUDART_INF_F ? -1 : top_id;
            if (a.logp != nullptr) a.logp[row] = top == -CUDART_INF_F ? CUDART_NAN_F : 0.f;
        }
        cluster.sync();                                          // the others have read this block's words
        return;
    }
    const double c2 = 1.4426950408889634074 / (double)__uint_as_float(temp_bits), dtop = (double)top;
    const double most = min_p > 0.f ? -log2((double)min_p) : CUDART_INF;         // distance that min_p allows

    // log2 distance from the largest; infinity for a token without weight (the comparison first: inf - inf, 0 * inf)
    auto distance = [&](float v) { return v == top ? 0.0 : v == -CUDART_INF_F ? CUDART_INF : (dtop - (double)v) * c2; };
    auto near = [&](double x) { return x <= (double)kFar; };     // (false for NaN: infinite temperature below an infinite logit)
    // round(2^45 * 2^-x), 0 <= x <= 47: x = k / 32 + r, 2^-r from its Taylor series, |r ln 2| <= 0.011: error 2e-15
    auto weight = [&](double x) {
        constexpr double kMagic = 6755399441055744.0;            // 1.5 * 2^52
        const double m = fma(x, 32.0, kMagic);
        const int j = __double2loint(m);
        const double r = fma(m - kMagic, -0.03125, x);
        double p = fma(r, -1.3333558146428443e-3, 9.6181291076284772e-3);
        p = fma(r, p, -5.5504108664821580e-2);
        p = fma(r, p, 2.4022650695910071e-1);
        p = fma(r, p, -6.9314718055994531e-1);
        p = fma(r, p, 1.0);
        const double scale = __longlong_as_double((long long)(1023 + 45 - (j >> 5)) << 52);
        return (u64)(__double_as_longlong(fma(p * s.root[j & 31], scale, 4503599627370496.0)) - 0x4330000000000000ll);
    };
    // Each thread walks over a run of neighbouring tokens, of odd length: no bank conflicts between the threads.
    const int run = ((n + kThreads - 1) / kThreads) | 1;
    const int begin = min(t * run, n), end = min(begin + run, n);
    u64 thr = 0;                                                 // kept so far: entries from thr on

    // Smallest id whose cumulative measure exceeds floor(u * total) + skip, and the measure's total.  Every thread of the cluster.
    auto locate = [&](auto measure, double u, u64 skip, u64& total) {
        u64 mine = 0, sum;
        for (int i = begin; i < end; ++i) mine += measure(value_of(slice[i]), first + i);
        u64 before = block_exclusive<u64>(mine, s.scan, sum);
        if (t == 0) s.total = sum;
        cluster.sync();
        total = 0;
        for (int i = 0; i < C; ++i) {
            const u64 x = *cluster.map_shared_rank(&s.total, i);
            before += i < rank ? x : 0;
            total += x;
        }
        u64 target = (u64)(u * (double)total) + skip;
        target = target < total ? target : total - 1;
        const uint32_t owner = __ballot_sync(0xffffffffu, before <= target && target < before + mine);
        if (owner != 0) {                                        // one warp of the cluster: its lanes share the run
            const int l = __ffs(owner) - 1, b = __shfl_sync(0xffffffffu, begin, l), e = __shfl_sync(0xffffffffu, end, l);
            u64 acc = __shfl_sync(0xffffffffu, before, l);
            for (int i0 = b; i0 < e; i0 += 32) {
                const u64 m = i0 + lane < e ? measure(value_of(slice[i0 + lane]), first + i0 + lane) : 0;
                u64 incl = m;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 x = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += x;
                }
                const uint32_t hit = __ballot_sync(0xffffffffu, acc + incl > target);
                if (hit != 0) {
                    if (lane == __ffs(hit) - 1) *cluster.map_shared_rank(&s.found, 0) = entry_of(bits_of(value_of(slice[i0 + lane])), first + i0 + lane);
                    break;
                }
                acc += __shfl_sync(0xffffffffu, incl, 31);
            }
        }
        cluster.sync();
        return *cluster.map_shared_rank(&s.found, 0);
    };

    // Moves thr to the end of the shortest leading run whose measure is at least the goal: by_mass the share p of all kept weight, else k
    // tokens.  Every thread of the cluster.
    auto select = [&](bool by_mass, double p) {
        const float span = fminf(kFar, (float)distance(of_bits(least_bits)));
        const float inv = span > 0.f ? (float)kBins / span : 0.f;
        auto bin_of = [&](double x) { return min(kBins - 1, (int)((float)x * inv)); };       // rises with x
        for (int i = t; i < kBins; i += kThreads) s.count[i] = 0;
        __syncthreads();
        for (int i = begin; i < end; ++i) {
            const float v = value_of(slice[i]);
            const double x = distance(v);
            if (near(x) && entry_of(bits_of(v), first + i) >= thr) atomicAdd(&s.count[bin_of(x)], 1u);
        }
        if (t < 2) s.bin[t] = kBins - 1;
        if (t == 0) { s.hi = 0; s.lo = 0xffffffffu; s.n_list = 0; s.sum[0] = s.sum[1] = s.sum[2] = 0; }
        cluster.sync();
        uint32_t c[kPerThread] = {}, mine = 0, all;
        for (int i = 0; i < C; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(s.count, i) + t * kPerThread);
            c[0] += x.x; c[1] += x.y; c[2] += x.z; c[3] += x.w;
        }
        static_assert(kPerThread == 4, "one 16-byte read of the counts");
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) mine += c[i];
        const uint32_t count_before = block_exclusive<uint32_t>(mine, s.scan, all);
        if (!by_mass && all <= (uint32_t)k) { cluster.sync(); return; }          // everything that has weight is kept
        if (by_mass) {
            // a bin's weights lie between those of its two ends: bounds of the cumulative weight, with a margin for their rounding
            const float w = inv > 0.f ? 1.f / inv : 0.f;
            float up[kPerThread], down[kPerThread], up_mine = 0.f, down_mine = 0.f, up_all, down_all;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                const int b = t * kPerThread + i;
                up[i] = (float)c[i] * exp2f(-(float)b * w);
                down[i] = b == kBins - 1 && span >= kFar ? 0.f : (float)c[i] * exp2f(-(float)(b + 1) * w);
                up_mine += up[i]; down_mine += down[i];
            }
            float cu = block_exclusive<float>(up_mine, s.scan, up_all), cd = block_exclusive<float>(down_mine, s.scan, down_all);
            const float from = (float)p * down_all * 0.999f, to = (float)p * up_all * 1.001f;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                cu += up[i]; cd += down[i];
                if (c[i] > 0 && cu >= from) atomicMin(&s.bin[0], t * kPerThread + i);
                if (c[i] > 0 && cd >= to) atomicMin(&s.bin[1], t * kPerThread + i);
            }
        } else {
            uint32_t cum = count_before;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                if (cum < (uint32_t)k && cum + c[i] >= (uint32_t)k) s.bin[0] = s.bin[1] = t * kPerThread + i;
                cum += c[i];
            }
        }
        __syncthreads();
        const int b0 = s.bin[0], b1 = s.bin[1];
        // tokens inside: few enough for the list?  (the same number in every block)
        uint32_t cand = 0, n_cand;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) cand += t * kPerThread + i >= b0 && t * kPerThread + i <= b1 ? c[i] : 0;
        block_exclusive<uint32_t>(cand, s.scan, n_cand);
        auto measure = [&](double x) { return by_mass ? weight(x) : (u64)1; };
        auto put = [&](u64 e) {
            const uint32_t at = atomicAdd(cluster.map_shared_rank(&s.n_list, 0), 1u);
            if (at < kList) cluster.map_shared_rank(s.list, 0)[at] = e;
        };
        u64 part[3] = {0, 0, 0};                                 // measure before, inside, behind
        uint32_t lo = 0xffffffffu, hi = 0;
        for (int i = begin; i < end; ++i) {
            const float v = value_of(slice[i]);
            const double x = distance(v);
            const u64 e = entry_of(bits_of(v), first + i);
            if (!near(x) || e < thr) continue;
            const int b = bin_of(x);
            const bool inside = b >= b0 && b <= b1;
            if (by_mass || b < b0) part[b < b0 ? 0 : inside ? 1 : 2] += measure(x);
            if (inside) {
                lo = min(lo, bits_of(v));
                hi = max(hi, bits_of(v));
                if (n_cand <= kList) put(e);
            }
        }
#pragma unroll
        for (int x = 0; x < 3; ++x) {
            for (int o = 16; o > 0; o >>= 1) part[x] += __shfl_xor_sync(0xffffffffu, part[x], o);
            if (lane == 0 && part[x] != 0) atomicAdd(&s.sum[x], part[x]);
        }
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) { atomicMin(&s.lo, lo); atomicMax(&s.hi, hi); }
        cluster.sync();
        u64 before = 0, total = 0;
        for (int i = 0; i < C; ++i) {
            const u64* x = cluster.map_shared_rank(s.sum, i);
            before += x[0];
            total += x[0] + x[1] + x[2];
            lo = min(lo, *cluster.map_shared_rank(&s.lo, i));
            hi = max(hi, *cluster.map_shared_rank(&s.hi, i));
        }
        const double goal = by_mass ? p * (double)total : (double)k;
        // divide the range of logit bits until the list holds what is left, or one value is
        while (n_cand > kList && lo < hi) {
            const int shift = max(0, 21 - __clz(hi - lo));       // (hi - lo) >> shift < 2048
            for (int i = t; i < kBins; i += kThreads) { s.count[i] = 0; s.mass[i] = 0; }
            cluster.sync();                                      // everyone has read the counts and sums of the step before
            for (int i = begin; i < end; ++i) {
                const float v = value_of(slice[i]);
                const uint32_t key = bits_of(v);
                if (key < lo || key > hi || entry_of(key, first + i) < thr) continue;
                const double x = distance(v);
                if (!near(x)) continue;
                const int b = (int)((hi - key) >> shift);
                atomicAdd(&s.count[b], 1u);
                if (by_mass) atomicAdd(&s.mass[b], weight(x));
            }
            if (t == 0) s.bin[0] = 0xffffffffu;
            cluster.sync();
            u64 m[kPerThread] = {}, m_mine = 0, m_all;
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                c[i] = 0;
                for (int r = 0; r < C; ++r) {
                    c[i] += cluster.map_shared_rank(s.count, r)[t * kPerThread + i];
                    if (by_mass) m[i] += cluster.map_shared_rank(s.mass, r)[t * kPerThread + i];
                }
                if (!by_mass) m[i] = c[i];
                m_mine += m[i];
            }
            u64 cum = before + block_exclusive<u64>(m_mine, s.scan, m_all);
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                if ((double)cum < goal && (double)(cum + m[i]) >= goal) {
                    s.bin[0] = t * kPerThread + i;
                    s.sum[0] = cum;
                    s.sum[1] = c[i];
                }
                cum += m[i];
            }
            __syncthreads();
            const uint32_t b = s.bin[0];
            if (b == 0xffffffffu) break;                         // (rounding of the goal at the very end of the range: all of it is kept)
            before = s.sum[0];
            n_cand = (uint32_t)s.sum[1];
            const uint32_t top_key = hi - (b << shift);
            lo = max(lo, top_key - min(top_key, (1u << shift) - 1u));
            hi = top_key;
            if (n_cand <= kList) {
                if (t == 0) s.n_list = 0;
                cluster.sync();
                for (int i = begin; i < end; ++i) {
                    const uint32_t key = bits_of(value_of(slice[i]));
                    const u64 e = entry_of(key, first + i);
                    if (key >= lo && key <= hi && e >= thr) put(e);
                }
            }
            cluster.sync();
        }
        if (n_cand <= kList) {
            if (rank == 0) {
                // entry i is the border if the measure up to it reaches the goal and the measure before it does not
                const int m = min((int)n_cand, (int)s.n_list);
                if (t == 0) s.thr = thr;
                if (t < m) s.list_w[t] = measure(distance(of_bits((uint32_t)(s.list[t] >> 32))));
                __syncthreads();
                if (t < m) {
                    const u64 e = s.list[t];
                    u64 cum = before;
                    for (int i = 0; i < m; ++i) cum += s.list[i] > e ? s.list_w[i] : 0;
                    if ((double)cum < goal && (double)(cum + s.list_w[t]) >= goal) s.thr = e;
                }
            }
            cluster.sync();
            thr = *cluster.map_shared_rank(&s.thr, 0);
        } else if (lo == hi) {
            // equal logits: the first so many of them in order of id
            const u64 w = measure(distance(of_bits(lo)));
            u64 want = 1;
            const double miss = goal - (double)before;
            if (miss > (double)w) want = (u64)ceil(miss / (double)w);
            u64 ties;
            const u64 keep_thr = thr;
            const u64 e = locate([&](float v, int id) { return (u64)(bits_of(v) == lo && entry_of(lo, id) >= keep_thr); }, 0.0, want - 1, ties);
            thr = e;
        }
        cluster.sync();
    };

    if (k > 0 && k < a.vocab) select(false, 0.0);
    if (top_p < 1.f) select(true, (double)top_p);
    u64 total;
    const float uf = __ldcg(a.u + row);
    const u64 e = locate(
        [&](float v, int id) {
            if (entry_of(bits_of(v), id) < thr) return (u64)0;
            const double x = distance(v);
            return near(x) && (x <= most || x == 0.0) ? weight(x) : (u64)0;
        },
        uf > 0.f ? (double)uf : 0.0, 0, total);
    if (rank == 0 && t == 0) {
        a.tokens[row] = (int)(0xffffffffu - (uint32_t)e);
        if (a.logp != nullptr)
            a.logp[row] = (float)(-(distance(of_bits((uint32_t)(e >> 32))) * 0.69314718055994530942 + log((double)total / kOne)));
    }
    cluster.sync();
}

// Blocks of a row: as many as the slice needs, more while the GPU has room for them.
int blocks_of_row(int rows, int vocab, int elt) {
    const int most_bytes = 128 * 1024;
    int c = 1;
    while (c < kMaxCluster && (((long long)vocab * elt > (long long)c * most_bytes) || (vocab > c * 4096 && (long long)rows * c < device_sm_count()))) c *= 2;
    return c;
}

template <typename T>
beagle_status launch_sample(SampleArgs a, int rows, cudaStream_t stream) {
    const int c = blocks_of_row(rows, a.vocab, (int)sizeof(T));
    a.slice = ((a.vocab + c - 1) / c + 7) / 8 * 8;
    const size_t bytes = (sizeof(Shared) + 15) / 16 * 16 + (size_t)(a.slice + 16) * sizeof(T);
    static PerDeviceOnce attr;
    if (!attr.ensure([] { return cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)rows * c);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = c;
    attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attrs;
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
    if (rows > 0x7fffffff / kMaxCluster) return BEAGLE_ERR_CAPACITY;
    if (rows == 0) return BEAGLE_OK;
    if (logits_dev == nullptr || u_dev == nullptr || tokens_out_dev == nullptr) return BEAGLE_ERR_INVALID_ARG;
    if (((uintptr_t)logits_dev & (logits_dtype == BEAGLE_BF16 ? 1 : 3)) ||
        (((uintptr_t)temperature_dev | (uintptr_t)top_k_dev | (uintptr_t)top_p_dev | (uintptr_t)min_p_dev | (uintptr_t)u_dev | (uintptr_t)tokens_out_dev |
          (uintptr_t)logp_out_dev) & 3))
        return BEAGLE_ERR_INVALID_ARG;
    SampleArgs a{logits_dev, row_stride, vocab, 0, temperature_dev, top_p_dev, min_p_dev, u_dev, top_k_dev, tokens_out_dev, logp_out_dev};
    return logits_dtype == BEAGLE_BF16 ? launch_sample<bf16>(a, rows, static_cast<cudaStream_t>(stream)) : launch_sample<float>(a, rows, static_cast<cudaStream_t>(stream));
}
