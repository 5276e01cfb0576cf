// Attention of one new token per sequence over a paged key/value cache (beagle_paged_attn).
//
//   o_h = sum_j softmax_j(<q_h, K_j> / sqrt(dh)) V_j   over the visible positions j < n:  all of them, or, with a window,
//   j >= n - window (the newest `window`, the token's own key included) and j < sinks.
//
// Bound by memory: G query heads do G * 4 flop per cached 2 * 2-byte pair, so the kernel is a stream over the visible cache.
// The lengths live on the device, so the work is divided there: the visible tiles of 64 positions of all (sequence, K/V head)
// pairs, one after the other, are cut into equal runs, one per CTA of a grid that fills the GPU once.  A ragged batch, a
// single long sequence and a batch of short ones are then balanced by the same rule.  A pair that lies inside one run is
// finished there; the others leave unnormalised partials (fp32, with their maximum and sum) that a second, dependent launch
// joins in the order of the runs, so results do not depend on timing.  No counter and no initialised workspace is needed.
// Where the cache's capacity or the window leave a pair only a few tiles (kWholeTiles), every pair is a run of its own and
// the second launch, most of such a call's latency, is left out.
//
// bf16, head_dim 64 / 128: a producer warp copies the tiles' pages by TMA (128-byte swizzle) into a ring of three stages (two
// CTAs per SM, about 190 KB in flight per SM); four consumer warps own 16 positions of each tile and keep their own running
// reference point, sum and O accumulator in registers over the whole run, so they meet only where a pair ends.  Products on
// mma.sync m16n8k16 with the G <= 8 query heads as rows: tcgen05 tiles have 64 rows at least, and the CUDA cores cannot do
// G * 4 flop per 4 bytes next to unpacking at memory speed.
// Other types and widths: paged_attn_simt_kernel, the same ring in front of the CUDA cores.
//
// beagle_paged_attn_shared, rows in groups with a common part, walks entries (paged_attn.cuh) in place of rows: here with the same two kernels if all
// groups are small or the type is not the tensor cores', else in paged_grouped.cu; paged_shared_join_kernel adds up what the runs leave of a
// row's own positions and of its group's common part, one (row, head) to four warps, the runs in order.
//
// Measured: 32 sequences of 512 to 8192, 32 heads over 8 of 128: 103 us of stream (5.8 to 6.0 TB/s of cache) and 5 us of join; 16
// sequences of 65000 to 131072: 1012 us, the rate of a plain copy; the smallest fp32 call: 4 us on the GPU.  fp32, 32 sequences of 2000,
// 8 K/V heads of 128 (524 MB): 111 us with one query head each, 118 with four, 142 with eight (loading straight into registers, without the
// ring, took 165, 212 and 490).  bf16, 537 MB, on the same CUDA-core kernel: head_dim 256 with 1 / 4 query heads a pair 112 / 138 us, head_dim 32 with
// 1 / 4 / 8 192 / 210 / 288: at 64 bytes a row there are four times as many scores and weights to form per byte as at 256.  No pipe is saturated there (issue slots
// 0.49 to 0.54, DRAM 0.35 to 0.50 of nominal); the consumer warps wait for their own shared-memory reads and shuffles half of the time.
//
// Masked positions (past the length, outside the window) have their weight and their V row replaced by zero before use, so
// whatever the pool holds there (NaN included) has no effect.
#include <cuda.h>

#include <atomic>
#include <cstring>

#include "pages.h"
#include "paged_rows.cuh"
#include "tensor_map.h"

using namespace beagle;

namespace beagle {
namespace {

// The G heads of a pair without a visible position: o = 0, lse = -inf.  Whole CTA.
template <typename T>
__device__ __forceinline__ void empty_pair(const PagedArgs& a, int b, int kvh, int dh) {
    T* out = static_cast<T*>(a.o) + ((size_t)b * a.Hq + (size_t)kvh * a.G) * dh;
    for (int i = threadIdx.x; i < a.G * dh; i += blockDim.x) out[i] = from_float<T>(0.f);
    if (a.lse != nullptr && threadIdx.x < a.G) a.lse[(size_t)b * a.Hq + kvh * a.G + threadIdx.x] = -INFINITY;
}


// The units of this CTA's run; in whole mode, of its pair.  Also zeroes the pairs without a visible position (shared out over the
// CTAs) and leaves the run's join item.  Whole CTA.
template <typename T>
__device__ __forceinline__ void begin_run(const PagedArgs& a, const Schedule& s, int dh, int& u0, int& u1) {
    if (a.whole) {
        const int b = blockIdx.x / a.Hkv, kvh = blockIdx.x - b * a.Hkv, n = tiles_of(s, b, a.Hkv);
        u0 = s.start[b] + kvh * n;
        u1 = u0 + n;
        if (n == 0) empty_pair<T>(a, b, kvh, dh);
        return;
    }
    const Runs runs(s.start[kMaxCallBatch], gridDim.x);
    u0 = runs.begin(blockIdx.x);
    u1 = runs.begin(blockIdx.x + 1);
    for (int i = blockIdx.x; i < a.batch * a.Hkv; i += gridDim.x)
        if (s.len[i / a.Hkv] == 0) empty_pair<T>(a, i / a.Hkv, i % a.Hkv, dh);
    if (threadIdx.x < 32) {
        JoinItem it = {-1, 0, 0, 0};
        if (u0 < u1) {
            Walk w;
            w.seek(s, u1 - 1, a.Hkv);
            const int e0 = u1 - 1 - w.i, e1 = e0 + w.n;          // the units of the run's last pair
            if (e0 >= u0 && e1 > u1) it = {w.b * a.Hkv + w.kvh, runs.of(e1 - 1), e0 != u0 ? 1 : 0, runs.total};
        }
        if (threadIdx.x == 0) *reinterpret_cast<int4*>(a.join + blockIdx.x) = make_int4(it.pair, it.last_run, it.second, it.total);
    }
}

template <typename T>
__device__ __forceinline__ void begin_run(const SharedArgs& a, const ScheduleOf<SharedArgs::kEntries>& s, int, int& u0, int& u1) {
    begin_shared(a, s, blockIdx.x, gridDim.x, threadIdx.x, blockDim.x, u0, u1);
}

template <int DH, typename Args>
__global__ void __launch_bounds__((kConsumers + 1) * 32, kCtasPerSm)
paged_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Args a) {
    using SM = PagedSmem<DH>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
    float* join = reinterpret_cast<float*>(gen + kStages * 2 * SM::kTileBytes);
    __shared__ ScheduleOf<Args::kEntries> s;
    __shared__ __align__(8) uint64_t bars[2 * kStages];
    __shared__ float s_m[kConsumers][8], s_l[kConsumers][8];
    __shared__ int s_abort;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kStages;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kConsumers); }
        s_abort = 0;
        fence_barrier_init();
    }
    pdl_launch_dependents();
    pdl_wait();                          // lengths, table, cache and queries may come from the previous launches
    build_schedule(a, s);
    int u0, u1;
    begin_run<bf16>(a, s, DH, u0, u1);
    if (u0 >= u1) return;
    attn_rows<DH>(tmK, tmV, a, s, base, join, full, empty, s_m, s_l, &s_abort, threadIdx.x >> 5, blockIdx.x, u0, u1);
}

// ------------------------------------------------------------------------------------------------
// fp32, and bf16 at head_dim 32 and 256, on the CUDA cores.  The same ring, filled by untiled bulk copies (a page's rows of one
// head are contiguous) of 64 positions, or 32 where a row has 512 bytes.  LPK lanes share a position (16 bytes of its row each),
// a warp's 32 / LPK groups walk its positions side by side with their own reference point, sum and O; they meet where a pair ends.
// The LPK partial sums of the heads' scores are added by halving: a lane hands half of its heads on and keeps the other half, so
// GM heads take about GM exchanges instead of GM log2(LPK), and each weight is formed in one place and handed to the other lanes.
// ------------------------------------------------------------------------------------------------
template <typename T, int DH, int GM>
struct SimtCfg {
    static constexpr int VN = 16 / (int)sizeof(T), LPK = DH / VN, KPW = 32 / LPK;
    static constexpr int kWarps = GM * VN >= 32 ? 4 : 8;                                // consumer warps: a thread keeps 2 GM VN of q and O
    static constexpr int kRow = DH * (int)sizeof(T), kSub = kRow >= 512 ? 32 : 64;       // bytes of a row; positions of a stage
    static constexpr int kPer = kSub / kWarps, kSteps = kPer / KPW;                      // positions of a warp; of each of its groups
    static constexpr int HV = GM > LPK ? GM / LPK : 1, kSpan = GM > LPK ? 1 : LPK / GM;  // heads a lane keeps; lanes that keep the same ones
    static constexpr int kStage = 2 * kSub * kRow, kJoin = (kWarps / 2) * GM * DH * 4;
    static constexpr int kFit = (104 * 1024 - kJoin) / kStage, kRing = kFit < 6 ? kFit : 6;
    static constexpr int kBytes = kRing * kStage + kJoin + 128;                          // + alignment slack
    static_assert(kPer % KPW == 0 && kRing >= 2, "shape");
    static __device__ __forceinline__ int owner(int h) { return GM > LPK ? h / HV : h * kSpan; }      // the lane of a group that keeps head h
};
template <typename T, int DH, int GM, typename Args>
__global__ void __launch_bounds__((SimtCfg<T, DH, GM>::kWarps + 1) * 32, 2) paged_attn_simt_kernel(const __grid_constant__ Args a) {
    using S = SimtCfg<T, DH, GM>;
    constexpr int VN = S::VN, LPK = S::LPK, KPW = S::KPW, HV = S::HV, kSteps = S::kSteps;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
    float* s_o = reinterpret_cast<float*>(ring + S::kRing * S::kStage);                  // [kWarps / 2][GM][DH]
    __shared__ ScheduleOf<Args::kEntries> s;
    __shared__ __align__(8) uint64_t bars[2 * S::kRing];
    __shared__ float s_m[S::kWarps][GM], s_l[S::kWarps][GM];
    __shared__ int s_abort;
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kRing;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane / LPK, sub = lane % LPK;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kRing; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, S::kWarps); }
        s_abort = 0;
        fence_barrier_init();
    }
    pdl_launch_dependents();
    pdl_wait();
    build_schedule(a, s);
    int u0, u1;
    begin_run<T>(a, s, DH, u0, u1);
    if (u0 >= u1) return;
    Walk w;
    w.seek(s, u0, a.Hkv);

    if (warp == S::kWarps) {
        // ---------------- producer: lane p copies page p of the stage
        const int rows = min(1 << a.page_shift, S::kSub), parts = S::kSub / rows;
        const uint32_t bytes = (uint32_t)rows * S::kRow;
        bool ok = true;
        int st = 0, ph = 0, issued = 0;
        for (int u = u0; u < u1 && ok; ++u) {
#pragma unroll 1
            for (int x = 0; x < kTile / S::kSub; ++x) {
                const int pos = w.tile(s) * kTile + x * S::kSub + lane * rows;
                int page = -1;
                // (a part without a visible position stays what it was: its weights and its V rows count as 0)
                if (lane < parts && pos < s.len[w.b] && (pos + rows > s.lo[w.b] || pos < a.sinks))
                    page = __ldcg(a.table + (size_t)slot_of(a, w.b) * a.max_pages + (pos >> a.page_shift));
                if (page >= a.n_pages) page = -1;
                const int copies = __popc(__ballot_sync(0xffffffffu, page >= 0));
                ok = mbar_wait(empty + 8 * st, ph ^ 1, &s_abort);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) {
                    if (copies > 0) mbar_expect_tx(full + 8 * st, 2 * copies * bytes);
                    else mbar_arrive(full + 8 * st);
                }
                __syncwarp();
                if (page >= 0) {
                    const size_t at = (((((size_t)page * a.Hkv + w.kvh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1)))) * S::kRow;
                    const uint32_t dst = smem_u32(ring) + st * S::kStage + lane * bytes;
                    bulk_load(dst, static_cast<const uint8_t*>(a.k) + at, bytes, full + 8 * st);
                    bulk_load(dst + S::kSub * S::kRow, static_cast<const uint8_t*>(a.v) + at, bytes, full + 8 * st);
                }
                ++issued;
                if (++st == S::kRing) { st = 0; ph ^= 1; }
            }
            w.next(s, a.batch, a.Hkv);
        }
        if (!ok)                         // copies already requested still land: wait (bounded) for the last of each stage
            for (int n = max(0, issued - S::kRing); n < issued; ++n)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(full + 8 * (n % S::kRing), (n / S::kRing) & 1); ++i) {}
        return;
    }

    // ---------------- consumers
    auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(S::kWarps * 32) : "memory"); };
    const int base_lane = lane - sub;
    float q[GM][VN], o[GM][VN], m[HV], l[HV];                    // m, l: of this lane's own heads
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < HV; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
#pragma unroll
        for (int h = 0; h < GM; ++h)
#pragma unroll
            for (int i = 0; i < VN; ++i) o[h][i] = 0.f;
    };
    auto of_head = [&](const float* v, int h) {                  // the owner's value of head h
        return GM == 1 ? v[0] : __shfl_sync(0xffffffffu, v[GM > LPK ? h % HV : 0], base_lane + S::owner(h));
    };
    clear();
#pragma unroll
    for (int h = 0; h < GM; ++h)
#pragma unroll
        for (int i = 0; i < VN; ++i) q[h][i] = 0.f;
    int have_q = -1, seg = 0, st = 0, ph = 0;
    bool ok = true, first_pair_open = w.i > 0;
    for (int u = u0; u < u1; ++u) {
        const int pair = w.b * a.Hkv + w.kvh;
        if (pair != have_q) {
            have_q = pair;
#pragma unroll
            for (int h = 0; h < GM; ++h)
                if (h < rows_of(a, w.b)) {
                    const uint4 x = __ldcg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + query_at(a, w.b, w.kvh, h, DH) + sub * VN));
                    unpack16<T>(x, q[h]);
                }
        }
        const int len = s.len[w.b], lo = s.lo[w.b];
#pragma unroll 1
        for (int x0 = 0; x0 < kTile / S::kSub; ++x0) {
            const int pos0 = w.tile(s) * kTile + x0 * S::kSub + warp * S::kPer;
            // A wait that runs out leaves NaN in what depends on it; the warp still meets the others where pairs end.
            if (ok) ok = mbar_wait(full + 8 * st, ph, &s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok)
#pragma unroll
                for (int i = 0; i < HV; ++i) l[i] = __int_as_float(0x7fffffff);
            if (ok && pos0 < len && (pos0 + S::kPer > lo || pos0 < a.sinks)) {
                const bool plain = pos0 + S::kPer <= len && (pos0 >= lo || pos0 + S::kPer <= a.sinks);
                const uint8_t* K = ring + st * S::kStage + (warp * S::kPer + grp) * S::kRow + sub * 16;
                const uint8_t* V = K + S::kSub * S::kRow;
                float sc[kSteps][HV], mx[HV];
#pragma unroll
                for (int i = 0; i < HV; ++i) mx[i] = -INFINITY;
#pragma unroll
                for (int x = 0; x < kSteps; ++x) {
                    float f[VN], v[GM];
                    unpack16<T>(*reinterpret_cast<const uint4*>(K + x * KPW * S::kRow), f);
#pragma unroll
                    for (int h = 0; h < GM; ++h) {
                        v[h] = 0.f;
#pragma unroll
                        for (int i = 0; i < VN; ++i) v[h] = fmaf(q[h][i], f[i], v[h]);
                    }
                    int n = GM;
#pragma unroll
                    for (int d = LPK / 2; d > 0; d >>= 1) {
                        if (n > 1) {
                            n /= 2;
                            const bool upper = (lane & d) != 0;
#pragma unroll
                            for (int h = 0; h < GM / 2; ++h)
                                if (h < n) {
                                    const float give = upper ? v[h] : v[h + n], keep = upper ? v[h + n] : v[h];
                                    v[h] = keep + __shfl_xor_sync(0xffffffffu, give, d);
                                }
                        } else {
                            v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
                        }
                    }
                    const int pos = pos0 + x * KPW + grp;
                    const bool vis = plain || (pos < len && (pos >= lo || pos < a.sinks));
#pragma unroll
                    for (int i = 0; i < HV; ++i) {
                        sc[x][i] = vis ? v[i] * a.scale_log2 : -INFINITY;
                        mx[i] = fmaxf(mx[i], sc[x][i]);
                    }
                }
                // the reference point moves only when a score exceeds it by more than kSlack: weights stay below 2^8
                bool grow = false;
#pragma unroll
                for (int i = 0; i < HV; ++i) grow |= mx[i] > m[i] + kSlack;
                if (__any_sync(0xffffffffu, grow)) {
                    float r[HV];
#pragma unroll
                    for (int i = 0; i < HV; ++i) {
                        const bool g = mx[i] > m[i] + kSlack;
                        r[i] = g && m[i] != -INFINITY ? exp2f(m[i] - mx[i]) : 1.f;
                        if (g) m[i] = mx[i];
                        l[i] *= r[i];
                    }
#pragma unroll
                    for (int h = 0; h < GM; ++h) {
                        const float f = of_head(r, h);
#pragma unroll
                        for (int i = 0; i < VN; ++i) o[h][i] *= f;
                    }
                }
#pragma unroll
                for (int i = 0; i < HV; ++i) {
                    const float neg = m[i] == -INFINITY ? 0.f : -m[i];       // no visible position so far: every weight is 0
#pragma unroll
                    for (int x = 0; x < kSteps; ++x) {
                        sc[x][i] = exp2f(sc[x][i] + neg);
                        l[i] += sc[x][i];
                    }
                }
#pragma unroll
                for (int x = 0; x < kSteps; ++x) {
                    uint4 raw = *reinterpret_cast<const uint4*>(V + x * KPW * S::kRow);
                    if (!plain) {
                        const int pos = pos0 + x * KPW + grp;
                        if (!(pos < len && (pos >= lo || pos < a.sinks))) raw = make_uint4(0u, 0u, 0u, 0u);
                    }
                    float f[VN];
                    unpack16<T>(raw, f);
#pragma unroll
                    for (int h = 0; h < GM; ++h) {
                        const float p = of_head(sc[x], h);
#pragma unroll
                        for (int i = 0; i < VN; ++i) o[h][i] = fmaf(p, f[i], o[h][i]);
                    }
                }
            }
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(empty + 8 * st);
            if (++st == S::kRing) { st = 0; ph ^= 1; }
        }
        const int b = w.b, kvh = w.kvh;
        const bool last = w.i + 1 == w.n;
        w.next(s, a.batch, a.Hkv);
        if (!last && u + 1 < u1) continue;

        // ---- join the warp's groups, then the warps
#pragma unroll
        for (int h = 0; h < GM; ++h) {
            const float mh = of_head(m, h);
            float lh = of_head(l, h), M = mh;
#pragma unroll
            for (int d = LPK; d < 32; d <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
            const float f = mh == -INFINITY ? 0.f : exp2f(mh - M);
            lh = mh == -INFINITY ? lh : lh * f;                  // (no position seen: the sum is 0, or NaN after a wait that ran out)
#pragma unroll
            for (int i = 0; i < VN; ++i) o[h][i] *= f;
#pragma unroll
            for (int d = LPK; d < 32; d <<= 1) {
                lh += __shfl_xor_sync(0xffffffffu, lh, d);
#pragma unroll
                for (int i = 0; i < VN; ++i) o[h][i] += __shfl_xor_sync(0xffffffffu, o[h][i], d);
            }
            if (lane == 0) { s_m[warp][h] = M; s_l[warp][h] = lh; }
        }
        meet();
        // the upper half of the warps hand theirs to the lower half, which add and leave the sums for all
        constexpr int kHalf = S::kWarps / 2;
#pragma unroll
        for (int h = 0; h < GM; ++h) {
            float M = -INFINITY;
#pragma unroll
            for (int x = 0; x < S::kWarps; ++x) M = fmaxf(M, s_m[x][h]);
            const float f = s_m[warp][h] == -INFINITY ? 0.f : exp2f(s_m[warp][h] - M);
#pragma unroll
            for (int i = 0; i < VN; ++i) {
                o[h][i] *= f;
                if (warp >= kHalf && grp == 0) s_o[((warp - kHalf) * GM + h) * DH + sub * VN + i] = o[h][i];
            }
        }
        meet();
        if (warp < kHalf && grp == 0)
#pragma unroll
            for (int h = 0; h < GM; ++h)
#pragma unroll
                for (int i = 0; i < VN; ++i) s_o[(warp * GM + h) * DH + sub * VN + i] += o[h][i];
        meet();
        const bool whole = !Args::kShared && last && !first_pair_open;
        for (int i = threadIdx.x; i < rows_of(a, b) * DH; i += S::kWarps * 32) {
            const int h = i / DH, d = i % DH;
            float M = -INFINITY, L = 0.f, acc = 0.f;
#pragma unroll
            for (int x = 0; x < S::kWarps; ++x) M = fmaxf(M, s_m[x][h]);
#pragma unroll
            for (int x = 0; x < S::kWarps; ++x) L += s_m[x][h] == -INFINITY ? s_l[x][h] : s_l[x][h] * exp2f(s_m[x][h] - M);
#pragma unroll
            for (int x = 0; x < kHalf; ++x) acc += s_o[(x * GM + h) * DH + d];
            const int head = kvh * a.G + h;
            if (whole) {
                static_cast<T*>(a.o)[((size_t)b * a.Hq + head) * DH + d] = from_float<T>(L != 0.f ? acc / L : 0.f);
                if (d == 0 && a.lse != nullptr) a.lse[(size_t)b * a.Hq + head] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
            } else {
                float* dst = a.part + ((size_t)part_at(a, b * a.Hkv + kvh, !first_pair_open, seg, blockIdx.x) * 8 + h) * (DH + 2);
                dst[d] = acc;
                if (d == 0) { dst[DH] = M; dst[DH + 1] = L; }
            }
        }
        meet();
        clear();
        first_pair_open = false;
        seg = 1;
    }
}

// ------------------------------------------------------------------------------------------------
// Joins the partials of every (sequence, query head) that more than one run worked on.
// blockIdx.x = run: the CTA joins head blockIdx.y of the pair that begins in this run and ends in a later one (there is at most
// one, and the run left word of it); eight warps share the partials, then meet in shared memory, always in the same order.
// ------------------------------------------------------------------------------------------------
constexpr int kJoinWarps = 8;
template <typename T, int DH>
__global__ void __launch_bounds__(kJoinWarps * 32) paged_attn_join_kernel(const __grid_constant__ PagedArgs a) {
    constexpr int kPer = (DH + 31) / 32;
    __shared__ float s_o[kJoinWarps][DH], s_m[kJoinWarps], s_l[kJoinWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();
    const int r0 = blockIdx.x, g = blockIdx.y;
    const int4 it = __ldcg(reinterpret_cast<const int4*>(a.join + r0));
    if (it.x < 0) return;
    const int b = it.x / a.Hkv, kvh = it.x - b * a.Hkv, r1 = it.y, head = kvh * a.G + g;
    T* out = static_cast<T*>(a.o) + ((size_t)b * a.Hq + head) * DH;
    const Runs runs(it.w, gridDim.x);
    const bool gaps = runs.total < runs.runs;                    // fewer tiles than runs: some runs between are empty and left no partial
    auto part = [&](int r) { return a.part + ((size_t)(2 * r + (r == r0 ? it.z : 0)) * 8 + g) * (DH + 2); };
    float M = -INFINITY, L = 0.f, acc[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
    for (int r = r0 + warp * 32 + lane; r <= r1; r += kJoinWarps * 32)
        if (!gaps || runs.begin(r) < runs.begin(r + 1)) M = fmaxf(M, __ldcg(part(r) + DH));
    M = warp_max(M);
    if (lane == 0) s_m[warp] = M;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kJoinWarps; ++i) M = fmaxf(M, s_m[i]);
#pragma unroll 4
    for (int r = r0 + warp; r <= r1; r += kJoinWarps) {
        if (gaps && runs.begin(r) >= runs.begin(r + 1)) continue;
        const float* p = part(r);
        const float m = __ldcg(p + DH);
        const float f = m == -INFINITY ? 0.f : exp2f(m - M);
        L += m == -INFINITY ? __ldcg(p + DH + 1) : f * __ldcg(p + DH + 1);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (lane + 32 * i < DH) acc[i] = fmaf(f, __ldcg(p + lane + 32 * i), acc[i]);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (lane + 32 * i < DH) s_o[warp][lane + 32 * i] = acc[i];
    if (lane == 0) s_l[warp] = L;
    __syncthreads();
    for (int d = threadIdx.x; d < DH; d += kJoinWarps * 32) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int i = 0; i < kJoinWarps; ++i) { x += s_o[i][d]; y += s_l[i]; }
        out[d] = from_float<T>(y != 0.f ? x / y : 0.f);
        if (d == 0 && a.lse != nullptr) a.lse[(size_t)b * a.Hq + head] = y != 0.f ? (M + log2f(y)) * kLn2 : -INFINITY;
    }
}

// Warps of a head in the join, and partials that each has in flight.  Calls of 32 rows over 8192 / four groups of 16 over 2094 to 3511, us: 4 and 4 28.9 / 81, 8 and 4
// 30.4 / 85, 4 and 8 29.2 / 83, 8 and 8 34 / 91, 4 and 2 30.6 / 80, 2 and 4 31.8 / 81.
constexpr int kSharedJoinWarps = 4;
constexpr int kJoinFlight = 4;
// The same for rows of groups, two (row of the call, query head) items a CTA; the partials of the row's own positions and those of the
// common part, which lie with the row's launch or (`prefix.on`) with the tensor cores'.
struct PrefixParts {
    const int2* span;
    const float* part;
    int n_pairs, part_rows, block;
    uint8_t on[kMaxCallBatch], entry[kMaxCallBatch];
};
template <typename T, int DH>
__global__ void __launch_bounds__(2 * kSharedJoinWarps * 32) paged_shared_join_kernel(const __grid_constant__ SharedArgs a, const __grid_constant__ PrefixParts prefix) {
    // a lane holds kPer neighbouring components, four warps share a head's partials
    constexpr int kPer = DH >= 128 ? 4 : DH >= 64 ? 2 : 1, kSteps = (DH + 32 * kPer - 1) / (32 * kPer), W = kSharedJoinWarps;
    __shared__ float s_o[2][W][DH], s_m[2][W], s_l[2][W];
    const int half = threadIdx.x / (W * 32), warp = threadIdx.x / 32 % W, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();
    const int item = 2 * blockIdx.x + half, b = item / a.Hq, head = item - b * a.Hq, kvh = head / a.G, h = head - kvh * a.G;
    const bool there = b < a.rows;
    const int group = there ? a.group_of[b] : 255;
    const bool common = group != 255, cores = common && prefix.on[group];
    // the row's own positions and the common part.  Partial i of a source is the (i % split)th of run r0 + i / split; the first run's lie by pair, the
    // others' by run, one behind the other: head + i * size for i < split, else rest + i * size.
    struct Source {
        const float *head, *rest;        // at the row's O
        int size, ml;                    // floats of a partial; from the row's O to its (maximum, sum)
        int n, split;
    };
    auto source = [&](bool first) {
        const bool tc = !first && cores;
        int e = b, at = h;
        if (!first) {
            const int j = common ? (b - a.group_row0[group]) * a.G + h : 0, block = tc ? prefix.block : a.block;
            e = common ? (tc ? prefix.entry[group] : a.prefix_entry[group]) + j / block : 0;
            at = j % block;
        }
        const int rows = tc ? prefix.part_rows : 8, pair = e * a.Hkv + kvh, split = tc ? 1 : a.split, size = rows * (DH + 2), o = tc ? at * DH : at * (DH + 2);
        const int2 runs = there && (first || common) ? __ldcg((tc ? prefix.span : a.span) + pair) : make_int2(0, -1);
        const float* part = (tc ? prefix.part : a.part) + o;
        return Source{part + (size_t)pair * split * size, part + (size_t)((tc ? prefix.n_pairs : a.n_pairs) + runs.x) * split * size, size,
                      (tc ? rows * DH + 2 * at : at * (DH + 2) + DH) - o, (runs.y - runs.x + 1) * split, split};
    };
    const Source own = source(true), shared = source(false);
    const int all = own.n + shared.n;
    float M = -INFINITY, L = 0.f, acc[kSteps][kPer];
#pragma unroll
    for (int x = 0; x < kSteps; ++x)
#pragma unroll
        for (int y = 0; y < kPer; ++y) acc[x][y] = 0.f;
    for (int i0 = warp; i0 < all; i0 += W * kJoinFlight) {
        float2 ml[kJoinFlight];
        float o[kJoinFlight][kSteps][kPer];
#pragma unroll
        for (int z = 0; z < kJoinFlight; ++z) {
            const int i = i0 + z * W;
            const bool some = i < all, mine = i < own.n;
            const int at = mine ? i : i - own.n;
            const float* p = (at < (mine ? own.split : shared.split) ? (mine ? own.head : shared.head) : (mine ? own.rest : shared.rest)) + (size_t)(uint32_t)at * (mine ? own.size : shared.size);
            ml[z] = some ? __ldcg(reinterpret_cast<const float2*>(p + (mine ? own.ml : shared.ml))) : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int d = 0; d < kSteps; ++d)
#pragma unroll
                for (int y = 0; y < kPer; y += kPer > 1 ? 2 : 1) {       // (rows of partials begin on 8 bytes)
                    const int c = (d * 32 + lane) * kPer + y;
                    if (kPer > 1) {
                        const float2 v = some && c < DH ? __ldcg(reinterpret_cast<const float2*>(p + c)) : make_float2(0.f, 0.f);
                        o[z][d][y] = v.x;
                        o[z][d][y + (kPer > 1 ? 1 : 0)] = v.y;
                    } else {
                        o[z][d][y] = some && c < DH ? __ldcg(p + c) : 0.f;
                    }
                }
        }
        float top = M;
#pragma unroll
        for (int z = 0; z < kJoinFlight; ++z) top = fmaxf(top, ml[z].x);
        const float f0 = M == -INFINITY ? 0.f : exp2f(M - top);
        L = M == -INFINITY ? L : L * f0;                         // (no position seen: the sum is 0, or NaN after a wait that ran out)
#pragma unroll
        for (int x = 0; x < kSteps; ++x)
#pragma unroll
            for (int y = 0; y < kPer; ++y) acc[x][y] *= f0;
#pragma unroll
        for (int z = 0; z < kJoinFlight; ++z) {
            const float f = ml[z].x == -INFINITY ? 0.f : exp2f(ml[z].x - top);
            L += ml[z].x == -INFINITY ? ml[z].y : f * ml[z].y;
#pragma unroll
            for (int x = 0; x < kSteps; ++x)
#pragma unroll
                for (int y = 0; y < kPer; ++y) acc[x][y] = fmaf(f, ml[z].x == -INFINITY ? 0.f : o[z][x][y], acc[x][y]);
        }
        M = top;
    }
#pragma unroll
    for (int x = 0; x < kSteps; ++x)
#pragma unroll
        for (int y = 0; y < kPer; ++y)
            if ((x * 32 + lane) * kPer + y < DH) s_o[half][warp][(x * 32 + lane) * kPer + y] = acc[x][y];
    if (lane == 0) { s_m[half][warp] = M; s_l[half][warp] = L; }
    __syncthreads();
    if (!there) return;
    T* out = static_cast<T*>(a.o) + ((size_t)b * a.Hq + head) * DH;
    for (int d = threadIdx.x % (W * 32); d < DH; d += W * 32) {
        float top = -INFINITY, x = 0.f, y = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) top = fmaxf(top, s_m[half][i]);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float f = s_m[half][i] == -INFINITY ? 0.f : exp2f(s_m[half][i] - top);
            x = fmaf(f, s_o[half][i][d], x);
            y += s_m[half][i] == -INFINITY ? s_l[half][i] : f * s_l[half][i];
        }
        out[d] = from_float<T>(y != 0.f ? x / y : 0.f);
        if (d == 0 && a.lse != nullptr) a.lse[(size_t)b * a.Hq + head] = y != 0.f ? (top + log2f(y)) * kLn2 : -INFINITY;
    }
}

// beagle_pages_shared: blockIdx.x = group.  The first page at which the table rows of its slots differ or the shortest of them ends.
// Bound by latency: row after row, a trip to L2 each (32 rows of 128 pages 9 us, 64 rows of 1024 53, 127 after a flush).
__global__ void __launch_bounds__(256) pages_shared_kernel(const int32_t* table, const int32_t* length, const __grid_constant__ PageSlots slots,
                                                         const __grid_constant__ PageSlots first_row, const __grid_constant__ PageSlots n_rows, int page_size,
                                                         int max_pages, int32_t* shared) {
    __shared__ int s_pages;
    pdl_launch_dependents();
    pdl_wait();
    const int g = blockIdx.x, r0 = first_row.slot[g], n = n_rows.slot[g], t = threadIdx.x;
    if (t == 0) s_pages = n > 1 ? max_pages : 0;
    __syncthreads();
    if (t < n) atomicMin(&s_pages, max(__ldcg(length + slots.slot[r0 + t]), 0) / page_size);
    __syncthreads();
    const int32_t* lead = table + (size_t)slots.slot[r0] * max_pages;
    const int pages = s_pages;
    __syncthreads();
    for (int r = 1; r < n; ++r) {
        const int32_t* row = table + (size_t)slots.slot[r0 + r] * max_pages;
        for (int i = t; i < pages; i += 256)
            if (__ldcg(row + i) != __ldcg(lead + i)) { atomicMin(&s_pages, i); break; }
    }
    __syncthreads();
    if (t == 0) shared[g] = s_pages * page_size;
}

constexpr int kMaxRuns = 2048;           // bound of the workspace; the grid is min(this, CTAs that fit the GPU)
constexpr int kSimtCtasPerSm = 2;
// Pairs of at most this many tiles are not cut: the join launch takes some 3 us, a tile on its own 0.4 (tensor cores), 0.9 (up to four
// heads a pair on the CUDA cores) or 3.5 (more).  Measured whole against cut, us: 4 heads of 64, fp32, 4 tiles, 32 sequences 7.6 against 9.2,
// one sequence 6.4 against 6.3, 6 tiles 8.2 against 6.4; 8 heads a pair of 128, fp32, 2 tiles 12.2 against 12.7, 3 tiles 15.7 against 13.0.
constexpr int kWholeTiles = 8, kWholeTilesSimt = 4, kWholeTilesMany = 2;

bool uses_mma(const beagle_pages* p) { return p->dtype == BEAGLE_BF16 && (p->head_dim == 64 || p->head_dim == 128); }
// The most tiles of one pair, as far as the host can know.
long long most_tiles(const beagle_pages* p, int window, int sinks) {
    const long long cap = ((long long)p->max_pages * p->page_size + kTile - 1) / kTile;
    if (window <= 0) return cap;
    const long long seen = ((long long)window + kTile - 2) / kTile + 1 + ((long long)sinks + kTile - 1) / kTile;
    return seen < cap ? seen : cap;
}
bool whole_pairs(const beagle_pages* p, int Hq, int window, int sinks) {
    return most_tiles(p, window, sinks) <= (uses_mma(p) ? kWholeTiles : Hq / p->n_kv_heads <= 4 ? kWholeTilesSimt : kWholeTilesMany);
}

template <typename T, int DH>
void launch_join(const PagedArgs& a, int runs, cudaStream_t stream) {
    if (!a.whole) launch_pdl(paged_attn_join_kernel<T, DH>, dim3(runs, a.G), dim3(kJoinWarps * 32), 0, stream, a);
}
struct SharedCall : SharedArgs {         // the rows' launch, and where the tensor cores' partials are
    PrefixParts prefix;
};
template <typename T, int DH>
void launch_join(const SharedCall& a, int, cudaStream_t stream) {
    launch_pdl(paged_shared_join_kernel<T, DH>, dim3((a.rows * a.Hq + 1) / 2), dim3(2 * kSharedJoinWarps * 32), 0, stream, static_cast<const SharedArgs&>(a), a.prefix);
}
template <typename Args> struct KernelArgs { typedef PagedArgs type; };
template <> struct KernelArgs<SharedCall> { typedef SharedArgs type; };

template <int DH, typename Args>
beagle_status launch_mma(const beagle_pages* p, const Args& a, int runs, cudaStream_t stream) {
    using SM = PagedSmem<DH>;
    typedef typename KernelArgs<Args>::type KArgs;
    const EncodeTiled encode = tensor_map_encoder();
    if (encode == nullptr) return BEAGLE_ERR_CUDA;
    CUtensorMap mk, mv;
    const int rows = p->page_size < kTile ? p->page_size : kTile;
    const cuuint64_t total = (cuuint64_t)p->n_pages * p->n_kv_heads * p->page_size;
    const cuuint64_t dims[2] = {DH, total}, strides[1] = {DH * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)rows}, one[2] = {1, 1};
    for (int i = 0; i < 2; ++i)
        if (encode(i ? &mv : &mk, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, i ? p->v : p->k, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return BEAGLE_ERR_CUDA;
    static PerDeviceOnce smem_attr;
    if (!smem_attr.ensure([] { return cudaFuncSetAttribute(paged_attn_kernel<DH, KArgs>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::kBytes) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    launch_pdl(paged_attn_kernel<DH, KArgs>, dim3(runs), dim3((kConsumers + 1) * 32), (size_t)SM::kBytes, stream, mk, mv, static_cast<const KArgs&>(a));
    launch_join<bf16, DH>(a, runs, stream);
    return BEAGLE_OK;
}

template <typename T, int DH, int GM, typename Args>
beagle_status launch_simt_heads(const Args& a, int runs, cudaStream_t stream) {
    using S = SimtCfg<T, DH, GM>;
    typedef typename KernelArgs<Args>::type KArgs;
    static PerDeviceOnce smem_attr;
    if (!smem_attr.ensure([] { return cudaFuncSetAttribute(paged_attn_simt_kernel<T, DH, GM, KArgs>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    launch_pdl(paged_attn_simt_kernel<T, DH, GM, KArgs>, dim3(runs), dim3((S::kWarps + 1) * 32), (size_t)S::kBytes, stream, static_cast<const KArgs&>(a));
    return BEAGLE_OK;
}

template <typename T, int DH, typename Args>
beagle_status launch_simt(const Args& a, int runs, cudaStream_t stream) {
    beagle_status st;
    if constexpr (Args::kShared) {                       // entries of the common part have as many rows as a kernel takes
        st = launch_simt_heads<T, DH, DH < 256 ? 8 : 4>(a, runs, stream);
    } else {
        if (a.G == 1) st = launch_simt_heads<T, DH, 1>(a, runs, stream);
        else if (a.G <= 2) st = launch_simt_heads<T, DH, 2>(a, runs, stream);
        else if (a.G <= 4) st = launch_simt_heads<T, DH, 4>(a, runs, stream);
        else if constexpr (DH < 256) st = launch_simt_heads<T, DH, 8>(a, runs, stream);
        else return BEAGLE_ERR_SHAPE;
    }
    if (st != BEAGLE_OK) return st;
    launch_join<T, DH>(a, runs, stream);
    return BEAGLE_OK;
}

template <typename Args>
beagle_status launch_attn(const beagle_pages* p, const Args& a, int runs, cudaStream_t stream) {
    beagle_status st;
    if (uses_mma(p)) st = p->head_dim == 128 ? launch_mma<128>(p, a, runs, stream) : launch_mma<64>(p, a, runs, stream);
    else if (p->dtype == BEAGLE_BF16) st = p->head_dim == 256 ? launch_simt<bf16, 256>(a, runs, stream) : launch_simt<bf16, 32>(a, runs, stream);
    else if (p->head_dim == 128) st = launch_simt<float, 128>(a, runs, stream);
    else if (p->head_dim == 64) st = launch_simt<float, 64>(a, runs, stream);
    else if (p->head_dim == 32) st = launch_simt<float, 32>(a, runs, stream);
    else st = launch_simt<float, 16>(a, runs, stream);
    if (st != BEAGLE_OK) return st;
    return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

beagle_status check_heads(const beagle_pages* p, int Hq) {
    if (Hq <= 0) return BEAGLE_ERR_INVALID_ARG;
    if (Hq % p->n_kv_heads || Hq / p->n_kv_heads > 8) return BEAGLE_ERR_SHAPE;
    // the widest rows with more than four grouped heads: as for the decode step of the draft head, no kernel has that shape
    if (p->dtype == BEAGLE_BF16 && p->head_dim == 256 && Hq / p->n_kv_heads > 4) return BEAGLE_ERR_SHAPE;
    return BEAGLE_OK;
}

// The call's arguments that both forms share, from checked values.
void fill_args(const beagle_pages* p, int Hq, const void* q, int64_t q_stride, void* out, float* lse, PagedArgs* a) {
    a->table = p->table; a->length = p->length; a->k = p->k; a->v = p->v; a->q = q; a->o = out; a->lse = lse;
    a->q_stride = q_stride;
    a->n_pages = p->n_pages; a->max_pages = p->max_pages;
    a->page_shift = 0;
    while ((1 << a->page_shift) < p->page_size) ++a->page_shift;
    a->Hq = Hq; a->Hkv = p->n_kv_heads; a->G = Hq / p->n_kv_heads;
    a->scale_log2 = 1.4426950408889634f / sqrtf((float)p->head_dim);
}
// Checks of the queries, outputs and workspace.
beagle_status check_call(const beagle_pages* p, int Hq, const void* q, int64_t q_stride, const void* out, const float* lse, const void* ws, size_t ws_bytes, size_t need) {
    const int e = p->dtype == BEAGLE_BF16 ? 2 : 4;
    if (q == nullptr || out == nullptr || (need > 0 && ws == nullptr) || q_stride < (int64_t)Hq * p->head_dim) return BEAGLE_ERR_INVALID_ARG;
    if ((((uintptr_t)q | (uintptr_t)out | (uintptr_t)ws) & 15) || (q_stride * e) % 16 || ((uintptr_t)lse & 3)) return BEAGLE_ERR_INVALID_ARG;
    return ws_bytes < need ? BEAGLE_ERR_CAPACITY : BEAGLE_OK;
}
// Slots of a call, in range; a slot may be read by several rows.
beagle_status check_rows(const beagle_pages* p, int batch, const int32_t* slot_host, PageSlots* out) {
    if (batch < 0 || (batch > 0 && slot_host == nullptr)) return BEAGLE_ERR_INVALID_ARG;
    if (batch > kMaxCallBatch) return BEAGLE_ERR_CAPACITY;
    for (int i = 0; i < batch; ++i) {
        if (slot_host[i] < 0 || slot_host[i] >= p->max_slots) return BEAGLE_ERR_INVALID_ARG;
        out->slot[i] = slot_host[i];
    }
    return BEAGLE_OK;
}
beagle_status check_groups(int batch, int n_groups, const int32_t* group_rows) {
    if (batch < 0 || n_groups < 0 || (n_groups > 0 && group_rows == nullptr)) return BEAGLE_ERR_INVALID_ARG;
    if (batch > kMaxCallBatch) return BEAGLE_ERR_CAPACITY;
    int64_t sum = 0;
    for (int i = 0; i < n_groups && i <= kMaxCallBatch; ++i) {
        if (group_rows[i] < 1) return BEAGLE_ERR_INVALID_ARG;
        sum += group_rows[i];
    }
    return sum == batch && n_groups <= batch ? BEAGLE_OK : BEAGLE_ERR_INVALID_ARG;
}

// Groups with more query rows than this (rows times grouped heads) have their common part on the tensor cores' 128-row tiles, the others in
// entries of eight rows, the rows of an mma.sync product.  Measured as entries / on the tensor cores, us, heads of 128, 8 K/V heads: 8 groups
// of 2 query rows over 4096 positions 43 / 49, of 8 47 / 53, 7 groups of 9 66 / 49, one group of 8 over 16384 40 / 38, of 9 49 / 38.
constexpr int kFewRows = 8;

// Query rows of a common part's entry: what the kernel takes as grouped heads.
int entry_rows(const beagle_pages* p) { return p->dtype == BEAGLE_BF16 && p->head_dim == 256 ? 4 : 8; }

// The entries of a call, from checked groups.
void plan_shared(const beagle_pages* p, int Hq, int batch, int n_groups, const int32_t* group_rows, SharedCall* a, PrefixArgs* f) {
    const int G = Hq / p->n_kv_heads;
    a->block = entry_rows(p);
    a->split = uses_mma(p) ? kConsumers : 1;
    f->block = prefix_block(G);
    int e = batch, fe = 0, most = 0;                     // the rows' own entries first
    for (int i = 0, r = 0; i < n_groups; r += group_rows[i++]) {
        const int R = group_rows[i], rows = R * G;
        f->on[i] = a->prefix.on[i] = R > 1 && uses_mma(p) && rows > kFewRows;
        a->group_row0[i] = (uint8_t)r;
        a->prefix_entry[i] = (uint8_t)e;
        a->prefix.entry[i] = (uint8_t)fe;
        for (int x = 0; x < R; ++x) {
            a->group_of[r + x] = R > 1 ? (uint8_t)i : (uint8_t)255;
            a->entry[r + x] = {(uint8_t)(r + x), a->group_of[r + x], 0, (uint8_t)G, 0};
        }
        if (R == 1) continue;
        const int block = f->on[i] ? f->block : a->block;
        for (int j = 0; j < rows; j += block) {
            const int n = rows - j < block ? rows - j : block;
            const SharedEntry x = {(uint8_t)r, (uint8_t)i, 1, (uint8_t)n, (uint16_t)j};
            if (f->on[i]) { f->entry[fe++] = x; most = n > most ? n : most; }
            else a->entry[e++] = x;
        }
    }
    memcpy(f->group_of, a->group_of, sizeof(f->group_of));
    a->batch = e;
    a->rows = f->rows = batch;
    a->n_groups = f->n_groups = n_groups;
    a->n_pairs = e * p->n_kv_heads;
    f->batch = fe;
    f->n_pairs = fe * p->n_kv_heads;
    f->part_rows = (most + 3) / 4 * 4;
}
int shared_runs(const beagle_pages* p) {
    const int runs = device_sm_count() * (uses_mma(p) ? kCtasPerSm : kSimtCtasPerSm);
    return runs < kMaxRuns ? runs : kMaxRuns;
}
// The call's workspace: where each form's runs of the pairs and partials lie, from a border of kWsAlign bytes on; bytes that the caller provides.
// The caller's memory begins on 16 bytes, but a common part's partials leave as 32 bytes at once, whose address has to be a multiple of
// that: the parts lie behind the first such border, and a whole one more is asked for.
constexpr size_t kWsAlign = 256;
char* shared_ws_base(void* ws) { return reinterpret_cast<char*>(((uintptr_t)ws + kWsAlign - 1) / kWsAlign * kWsAlign); }
struct SharedLayout { size_t span, prefix_span, part, prefix_part, bytes; };
SharedLayout shared_ws(const beagle_pages* p, const SharedArgs& a, const PrefixArgs& f) {
    const size_t row = (size_t)(p->head_dim + 2) * sizeof(float);
    auto up = [](size_t n) { return (n + kWsAlign - 1) / kWsAlign * kWsAlign; };
    SharedLayout l;
    l.span = 0;
    l.prefix_span = l.span + up(a.n_pairs * sizeof(int2));
    l.part = l.prefix_span + up(f.n_pairs * sizeof(int2));
    l.prefix_part = l.part + up((size_t)(a.n_pairs + shared_runs(p)) * a.split * 8 * row);
    l.bytes = kWsAlign + l.prefix_part + (f.batch > 0 ? up((size_t)(f.n_pairs + shared_runs(p)) * f.part_rows * row) : 0);
    return l;
}

}  // namespace

bool paged_attn_fits(const beagle_pages* p, int batch) {
    return (long long)batch * p->n_kv_heads * ((long long)p->max_pages * p->page_size / kTile + 2) <= 0x7fffffffll;
}

size_t paged_attn_workspace_most(int dtype, int head_dim) {
    const int per = dtype == BEAGLE_BF16 && (head_dim == 64 || head_dim == 128) ? kCtasPerSm : kSimtCtasPerSm;
    const int sms = device_sm_count(), runs = sms * per < kMaxRuns ? sms * per : kMaxRuns;
    return ((size_t)runs * sizeof(JoinItem) + (size_t)2 * runs * 8 * (head_dim + 2) * sizeof(float) + 255) / 256 * 256;
}

int device_sm_count() {
    static std::atomic<int> counts[PerDeviceOnce::kMaxDevices];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= PerDeviceOnce::kMaxDevices) return 148;
    n = counts[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
        counts[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

EncodeTiled tensor_map_encoder() {
    static std::atomic<void*> cached{nullptr};
    void* fn = cached.load(std::memory_order_acquire);
    if (fn == nullptr) {
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        cached.store(fn, std::memory_order_release);
    }
    return reinterpret_cast<EncodeTiled>(fn);
}

}  // namespace beagle

extern "C" {

beagle_status beagle_paged_attn_workspace_bytes(const beagle_pages* p, int32_t n_q_heads, int32_t window, int32_t sinks, size_t* bytes) {
    if (p == nullptr || bytes == nullptr || p->n_kv_heads <= 0 || p->max_pages <= 0 || window < 0 || sinks < 0) return BEAGLE_ERR_INVALID_ARG;
    if (!pages_valid_shape(p)) return BEAGLE_ERR_SHAPE;
    const beagle_status st = check_heads(p, n_q_heads);
    if (st != BEAGLE_OK) return st;
    if (whole_pairs(p, n_q_heads, window, sinks)) {
        *bytes = 0;
        return BEAGLE_OK;
    }
    *bytes = paged_attn_workspace_most(p->dtype, p->head_dim);
    return BEAGLE_OK;
}

beagle_status beagle_paged_attn(const beagle_pages* p, int32_t batch, const int32_t* slot_host, int32_t n_q_heads, const void* q_dev, int64_t q_stride,
                                int32_t window, int32_t sinks, void* out_dev, float* lse_dev, void* ws_dev, size_t ws_bytes, void* stream_) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    PagedArgs a;
    memset(&a, 0, sizeof(a));
    st = check_rows(p, batch, slot_host, &a.slots);
    if (st != BEAGLE_OK) return st;
    st = check_heads(p, n_q_heads);
    if (st != BEAGLE_OK) return st;
    if (window < 0 || sinks < 0) return BEAGLE_ERR_INVALID_ARG;
    if (batch == 0) return BEAGLE_OK;
    size_t need = 0;
    beagle_paged_attn_workspace_bytes(p, n_q_heads, window, sinks, &need);
    st = check_call(p, n_q_heads, q_dev, q_stride, out_dev, lse_dev, ws_dev, ws_bytes, need);
    if (st != BEAGLE_OK) return st;
    if (!paged_attn_fits(p, batch)) return BEAGLE_ERR_CAPACITY;
    fill_args(p, n_q_heads, q_dev, q_stride, out_dev, lse_dev, &a);
    a.batch = batch;
    a.window = window; a.sinks = sinks;
    // no more runs than the cache's capacity has tiles
    const long long most = (long long)batch * p->n_kv_heads * most_tiles(p, window, sinks);
    a.whole = whole_pairs(p, n_q_heads, window, sinks) ? 1 : 0;
    long long runs = (long long)device_sm_count() * (uses_mma(p) ? kCtasPerSm : kSimtCtasPerSm);
    if (runs > kMaxRuns) runs = kMaxRuns;
    if (runs > most) runs = most;
    if (a.whole) runs = (long long)batch * p->n_kv_heads;
    a.join = static_cast<JoinItem*>(ws_dev);
    a.part = a.whole ? nullptr : reinterpret_cast<float*>(a.join + runs);
    return launch_attn(p, a, (int)runs, static_cast<cudaStream_t>(stream_));
}

beagle_status beagle_pages_shared(const beagle_pages* p, int32_t batch, const int32_t* slot_host, int32_t n_groups, const int32_t* group_rows_host,
                                  int32_t* shared_dev, void* stream) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    PageSlots slots, first, count;
    st = check_rows(p, batch, slot_host, &slots);
    if (st != BEAGLE_OK) return st;
    st = check_groups(batch, n_groups, group_rows_host);
    if (st != BEAGLE_OK || n_groups == 0) return st;
    if (shared_dev == nullptr || ((uintptr_t)shared_dev & 3)) return BEAGLE_ERR_INVALID_ARG;
    for (int i = 0, r = 0; i < n_groups; r += group_rows_host[i++]) { first.slot[i] = r; count.slot[i] = group_rows_host[i]; }
    launch_pdl(pages_shared_kernel, dim3(n_groups), dim3(256), 0, static_cast<cudaStream_t>(stream), p->table, p->length, slots, first, count, p->page_size,
               p->max_pages, shared_dev);
    return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

beagle_status beagle_paged_attn_shared_workspace_bytes(const beagle_pages* p, int32_t batch, int32_t n_q_heads, int32_t n_groups,
                                                       const int32_t* group_rows_host, size_t* bytes) {
    if (p == nullptr || bytes == nullptr || p->n_kv_heads <= 0 || p->max_pages <= 0) return BEAGLE_ERR_INVALID_ARG;
    if (!pages_valid_shape(p)) return BEAGLE_ERR_SHAPE;
    beagle_status st = check_heads(p, n_q_heads);
    if (st != BEAGLE_OK) return st;
    st = check_groups(batch, n_groups, group_rows_host);
    if (st != BEAGLE_OK) return st;
    SharedCall a;
    PrefixArgs f;
    memset(static_cast<void*>(&a), 0, sizeof(a));
    memset(static_cast<void*>(&f), 0, sizeof(f));
    plan_shared(p, n_q_heads, batch, n_groups, group_rows_host, &a, &f);
    *bytes = shared_ws(p, a, f).bytes;
    return BEAGLE_OK;
}

beagle_status beagle_paged_attn_shared(const beagle_pages* p, int32_t batch, const int32_t* slot_host, int32_t n_groups, const int32_t* group_rows_host,
                                       const int32_t* shared_dev, int32_t n_q_heads, const void* q_dev, int64_t q_stride, void* out_dev, float* lse_dev,
                                       void* ws_dev, size_t ws_bytes, void* stream_) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    SharedCall a;
    PrefixArgs f;
    memset(static_cast<void*>(&a), 0, sizeof(a));
    memset(static_cast<void*>(&f), 0, sizeof(f));
    st = check_rows(p, batch, slot_host, &a.slots);
    if (st != BEAGLE_OK) return st;
    st = check_heads(p, n_q_heads);
    if (st != BEAGLE_OK) return st;
    st = check_groups(batch, n_groups, group_rows_host);
    if (st != BEAGLE_OK) return st;
    if (batch == 0) return BEAGLE_OK;
    if (shared_dev == nullptr || ((uintptr_t)shared_dev & 3)) return BEAGLE_ERR_INVALID_ARG;
    plan_shared(p, n_q_heads, batch, n_groups, group_rows_host, &a, &f);
    const SharedLayout l = shared_ws(p, a, f);
    st = check_call(p, n_q_heads, q_dev, q_stride, out_dev, lse_dev, ws_dev, ws_bytes, l.bytes);
    if (st != BEAGLE_OK) return st;
    if (!paged_attn_fits(p, a.batch) || !paged_attn_fits(p, f.batch)) return BEAGLE_ERR_CAPACITY;
    fill_args(p, n_q_heads, q_dev, q_stride, out_dev, lse_dev, &a);
    f.slots = a.slots;
    fill_args(p, n_q_heads, q_dev, q_stride, out_dev, lse_dev, &f);
    a.shared = f.shared = shared_dev;
    char* base = shared_ws_base(ws_dev);
    a.span = reinterpret_cast<int2*>(base + l.span);
    f.span = reinterpret_cast<int2*>(base + l.prefix_span);
    a.part = reinterpret_cast<float*>(base + l.part);
    f.part = reinterpret_cast<float*>(base + l.prefix_part);
    a.prefix.span = f.span; a.prefix.part = f.part;
    a.prefix.n_pairs = f.n_pairs; a.prefix.part_rows = f.part_rows; a.prefix.block = f.block;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int runs = shared_runs(p);
    if (f.batch > 0) {
        st = launch_grouped(p, a, f, runs, stream);
        if (st != BEAGLE_OK) return st;
        if (p->head_dim == 128) launch_join<bf16, 128>(a, runs, stream);
        else launch_join<bf16, 64>(a, runs, stream);
        return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
    }
    const long long most = (long long)a.n_pairs * most_tiles(p, 0, 0);           // (no more runs than the cache's capacity has tiles)
    return launch_attn(p, a, (int)(runs < most ? runs : most), stream);
}

}  // extern "C"
