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
#include "tc_ptx.cuh"
#include "tensor_map.h"

using namespace beagle;

namespace beagle {
namespace {

using namespace tc;

constexpr int kTile = 64;               // cached positions per tile
constexpr int kConsumers = 4;           // warps; each owns 16 positions of a tile
constexpr int kPerWarp = kTile / kConsumers;
constexpr int kStages = 3;
constexpr int kCtasPerSm = 2;
constexpr float kSlack = 8.f;           // how far (log2) a score may exceed the row's reference point before it moves
constexpr float kLn2 = 0.6931471805599453f;

struct JoinItem;
struct PagedArgs {
    const int32_t *table, *length;
    const void *k, *v;                  // pools (the SIMT kernel; the other one has tensor maps)
    const void* q;
    void* o;
    float* lse;                         // [batch, Hq] or NULL
    JoinItem* join;                     // [runs]
    float* part;                        // [2 * runs][8][dh + 2]: unnormalised O, then maximum (log2 units) and sum
    long long q_stride;
    int batch, n_pages, page_shift, max_pages, Hq, Hkv, G, window, sinks;
    int whole;                          // every (sequence, K/V head) pair is one run
    float scale_log2;
    PageSlots slots;
};

// How the visible tiles are divided; computed by every CTA from the lengths (64 values at most).
struct Schedule {
    int len[kMaxCallBatch];             // positions of the sequence
    int lo[kMaxCallBatch];              // first position of the window (0: everything is visible)
    int sink_tiles[kMaxCallBatch];      // tiles in front of the window's first one
    int first[kMaxCallBatch];           // first tile of the window
    int start[kMaxCallBatch + 1];       // prefix sum of (tiles * Hkv)
};

__device__ __forceinline__ int tiles_of(const Schedule& s, int b, int Hkv) { return (s.start[b + 1] - s.start[b]) / Hkv; }
// First unit of run r: floor(total * r / runs), in 32 bits (runs <= 2048).
struct Runs {
    int total, runs, each, rest;
    __device__ __forceinline__ Runs(int t, int n) : total(t), runs(n), each(t / n), rest(t - t / n * n) {}
    __device__ __forceinline__ int begin(int r) const { return each * r + rest * r / runs; }
    __device__ __forceinline__ int of(int unit) const {                         // the run that holds `unit`
        int r = min(runs - 1, (int)((float)unit * (float)runs / (float)total));
        while (r + 1 < runs && begin(r + 1) <= unit) ++r;
        while (r > 0 && begin(r) > unit) --r;
        return r;
    }
};

// Threads 0..63 of the CTA fill `s`; the caller synchronises afterwards.
__device__ __forceinline__ void make_schedule(const PagedArgs& a, Schedule& s) {
    const int t = threadIdx.x;
    if (t >= kMaxCallBatch) return;
    int tiles = 0;
    if (t < a.batch) {
        const int cap = a.max_pages << a.page_shift;
        const int n = min(max(__ldcg(a.length + a.slots.slot[t]), 0), cap);
        const int lo = (a.window > 0 && n > a.window) ? n - a.window : 0;
        const int first = lo / kTile;
        const int front = min((min(a.sinks, lo) + kTile - 1) / kTile, first);
        s.len[t] = n; s.lo[t] = lo; s.first[t] = first; s.sink_tiles[t] = front;
        tiles = (front + (n + kTile - 1) / kTile - first) * a.Hkv;
    }
    // inclusive sum over the 64 threads: two warps
    int incl = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if ((t & 31) >= o) incl += v;
    }
    s.start[t + 1] = incl;
    if (t == 0) s.start[0] = 0;
}
__device__ __forceinline__ void finish_schedule(Schedule& s) {          // second half: the upper warp's offset; between two barriers
    const int t = threadIdx.x;
    if (t >= 32 && t < kMaxCallBatch) s.start[t + 1] += s.start[32];
}

// Walks the units [u, end) of one run: for every tile the pair (b, kvh), the tile's first position and whether the pair ends.
struct Walk {
    int b, kvh, i, n;                   // sequence, K/V head, tile index inside the pair, tiles of the pair
    __device__ __forceinline__ void seek(const Schedule& s, int unit, int Hkv) {          // whole warps
        const int lane = threadIdx.x & 31;
        b = __popc(__ballot_sync(0xffffffffu, s.start[lane + 1] <= unit)) + __popc(__ballot_sync(0xffffffffu, s.start[lane + 33] <= unit));
        n = tiles_of(s, b, Hkv);
        const int in = unit - s.start[b];
        kvh = in / n;
        i = in - kvh * n;
    }
    __device__ __forceinline__ void next(const Schedule& s, int batch, int Hkv) {
        if (++i < n) return;
        i = 0;
        if (++kvh < Hkv) return;
        kvh = 0;
        do { ++b; } while (b < batch && s.start[b + 1] == s.start[b]);
        if (b < batch) n = tiles_of(s, b, Hkv);
    }
    __device__ __forceinline__ int tile(const Schedule& s) const { return i < s.sink_tiles[b] ? i : s.first[b] + i - s.sink_tiles[b]; }
};

// The G heads of a pair without a visible position: o = 0, lse = -inf.  Whole CTA.
template <typename T>
__device__ __forceinline__ void empty_pair(const PagedArgs& a, int b, int kvh, int dh) {
    T* out = static_cast<T*>(a.o) + ((size_t)b * a.Hq + (size_t)kvh * a.G) * dh;
    for (int i = threadIdx.x; i < a.G * dh; i += blockDim.x) out[i] = from_float<T>(0.f);
    if (a.lse != nullptr && threadIdx.x < a.G) a.lse[(size_t)b * a.Hq + kvh * a.G + threadIdx.x] = -INFINITY;
}

// What the join does for a run: the pair that begins in it and ends in a later one, if there is one.
struct JoinItem { int pair, last_run, second, total; };          // pair: b * Hkv + kvh or -1; second: it is the run's second partial; all tiles

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

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
// D (16 x 8, fp32) += A (16 x 16) B (16 x 8); rows 8..15 of A are zero (at most eight query heads share a K/V head)
__device__ __forceinline__ void mma_rows8(float* d, uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
    float z0 = 0.f, z1 = 0.f;
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%5}, {%7,%8}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(z0), "+f"(z1)
                 : "r"(a0), "r"(0u), "r"(a2), "r"(b0), "r"(b1));
}
// Untiled copy: both addresses 16-byte aligned, `bytes` a multiple of 16.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <int DH>
struct PagedSmem {
    static constexpr int kTileBytes = kTile * DH * 2;                       // one of K / V
    static constexpr int kJoin = 2 * 8 * DH * 4;                            // two warps' O rows on their way to the other two
    static constexpr int kBytes = kStages * 2 * kTileBytes + kJoin + 1024;  // + alignment slack
};

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int DH>
__global__ void __launch_bounds__((kConsumers + 1) * 32, kCtasPerSm)
paged_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PagedArgs a) {
    using SM = PagedSmem<DH>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
    float* join = reinterpret_cast<float*>(gen + kStages * 2 * SM::kTileBytes);
    __shared__ Schedule s;
    __shared__ __align__(8) uint64_t bars[2 * kStages];
    __shared__ float s_m[kConsumers][8], s_l[kConsumers][8];
    __shared__ int s_abort;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kStages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kConsumers); }
        s_abort = 0;
        fence_barrier_init();
    }
    pdl_launch_dependents();
    pdl_wait();                          // lengths, table, cache and queries may come from the previous launches
    make_schedule(a, s);
    __syncthreads();
    finish_schedule(s);
    __syncthreads();
    int u0, u1;
    begin_run<bf16>(a, s, DH, u0, u1);
    if (u0 >= u1) return;
    Walk w;
    w.seek(s, u0, a.Hkv);

    if (warp == kConsumers) {
        // ---------------- producer: lane p copies page p of the tile (a tile spans 1, 2, 4 or 8 pages)
        const int rows = min(1 << a.page_shift, kTile);          // rows of one copy
        const int parts = kTile / rows;
        const uint32_t part_bytes = (uint32_t)rows * DH * 2;
        const uint64_t once = policy_evict_first();
        bool ok = true;
        int issued = 0;
        int next_page = -1;
        auto page_of = [&](const Walk& x) {                      // this lane's page of the walk's tile, -1 if it holds no position
            const int pos = x.tile(s) * kTile + lane * rows;
            int id = -1;
            // (a part without a visible position stays what it was: its weights and its V rows count as 0)
            if (lane < parts && pos < s.len[x.b] && (pos + rows > s.lo[x.b] || pos < a.sinks)) id = __ldcg(a.table + (size_t)a.slots.slot[x.b] * a.max_pages + (pos >> a.page_shift));
            return (id >= 0 && id < a.n_pages) ? id : -1;
        };
        next_page = page_of(w);
        for (int u = u0; u < u1; ++u) {
            const int st = issued % kStages;
            const int page = next_page;
            const int pos = w.tile(s) * kTile + lane * rows;
            const int row = page >= 0 ? ((page * a.Hkv + w.kvh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : 0;
            w.next(s, a.batch, a.Hkv);
            if (u + 1 < u1) next_page = page_of(w);              // the next tile's entry is on its way while this one waits for its slot
            const int copies = __popc(__ballot_sync(0xffffffffu, page >= 0));
            ok = mbar_wait(empty + 8 * st, ((issued / kStages) & 1) ^ 1, &s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (lane == 0) {
                if (copies > 0) mbar_expect_tx(full + 8 * st, 2 * copies * part_bytes);
                else mbar_arrive(full + 8 * st);
            }
            __syncwarp();
            if (page >= 0) {
                const uint32_t dst = base + st * 2 * SM::kTileBytes + lane * part_bytes;
#pragma unroll
                for (int h = 0; h < DH / 64; ++h) tma_load_2d_hint(dst + h * rows * 128, &tmK, full + 8 * st, 64 * h, row, once);
#pragma unroll
                for (int h = 0; h < DH / 64; ++h) tma_load_2d_hint(dst + SM::kTileBytes + h * rows * 128, &tmV, full + 8 * st, 64 * h, row, once);
            }
            ++issued;
        }
        if (!ok)                         // copies already requested still land: wait (bounded) for the last of each stage
            for (int n = max(0, issued - kStages); n < issued; ++n)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(full + 8 * (n % kStages), (n / kStages) & 1); ++i) {}
        return;
    }

    // ---------------- consumers
    const int g = lane >> 2, c = lane & 3;
    const int r_log = min(a.page_shift, 6);                      // log2 rows of a copy
    const int half_step = 128 << r_log, part_step = DH * 2 << r_log, r_mask = (1 << r_log) - 1;
    // byte offset of 16-byte piece `chunk` of row r: [copy][64-column half][row][128 bytes], swizzled inside 8 rows
    auto off = [&](int r, int chunk) {
        return (uint32_t)((r >> r_log) * part_step + (chunk >> 3) * half_step + (r & r_mask) * 128 + (((chunk & 7) ^ (r & 7)) << 4));
    };
    const int row0 = warp * kPerWarp;
    float o[DH / 8][2], m = -INFINITY, l = 0.f;
    uint32_t qa[DH / 16][2];
    int have_q = -1;                                             // the pair whose queries are in registers
    int seg = 0;                                                 // partial slot: the run's first pair that continues, else the second
    bool ok = true, first_pair_open = w.i > 0;                   // the first pair began in an earlier run
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = 0.f;
    int step = 0;
    for (int u = u0; u < u1; ++u, ++step) {
        const int pair = w.b * a.Hkv + w.kvh;
        if (pair != have_q) {
            have_q = pair;
            const uint32_t* qrow = reinterpret_cast<const uint32_t*>(static_cast<const bf16*>(a.q) + (size_t)w.b * a.q_stride + (size_t)(w.kvh * a.G + (g < a.G ? g : 0)) * DH);
#pragma unroll
            for (int ks = 0; ks < DH / 16; ++ks) {
                qa[ks][0] = g < a.G ? __ldcg(qrow + ks * 8 + c) : 0u;
                qa[ks][1] = g < a.G ? __ldcg(qrow + ks * 8 + 4 + c) : 0u;
            }
        }
        const int st = step % kStages;
        const int pos0 = w.tile(s) * kTile + row0;               // first position of this warp
        const int len = s.len[w.b], lo = s.lo[w.b];
        const bool plain = pos0 + kPerWarp <= len && (pos0 >= lo || pos0 + kPerWarp <= a.sinks);
        // A wait that runs out leaves NaN in what depends on it; the warp still meets the others where pairs end.
        if (ok) ok = mbar_wait(full + 8 * st, (step / kStages) & 1, &s_abort);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) l = __int_as_float(0x7fffffff);
        const uint32_t sK = base + st * 2 * SM::kTileBytes, sV = sK + SM::kTileBytes;
        if (ok && pos0 < len && (pos0 + kPerWarp > lo || pos0 < a.sinks)) {
            float sc[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
            for (int dg = 0; dg < DH / 32; ++dg)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    uint32_t b0, b1, b2, b3;
                    ldsm4(sK + off(row0 + nt * 8 + (lane & 7), 4 * dg + (lane >> 3)), b0, b1, b2, b3);
                    mma_rows8(sc[nt], qa[2 * dg][0], qa[2 * dg][1], b0, b1);
                    mma_rows8(sc[nt], qa[2 * dg + 1][0], qa[2 * dg + 1][1], b2, b3);
                }
            uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;   // V rows (2c, 2c+1) and (2c+8, 2c+9) as 16-bit lanes
            float mx = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = sc[nt][e] * a.scale_log2;
                    if (!plain) {
                        const int pos = pos0 + nt * 8 + 2 * c + e;
                        const bool vis = pos < len && (pos >= lo || pos < a.sinks);
                        x = vis ? x : -INFINITY;
                        if (!vis) (nt == 0 ? keep0 : keep1) &= e == 0 ? 0xffff0000u : 0x0000ffffu;
                    }
                    sc[nt][e] = x;
                    mx = fmaxf(mx, x);
                }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            // the reference point moves only when a score exceeds it by more than kSlack: weights stay below 2^8
            const bool grow = mx > m + kSlack;
            if (__any_sync(0xffffffffu, grow)) {
                const float f = (grow && m != -INFINITY) ? exp2f(m - mx) : 1.f;
                if (grow) m = mx;
                l *= f;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) { o[i][0] *= f; o[i][1] *= f; }
            }
            const float neg = m == -INFINITY ? 0.f : -m;         // no visible position so far: every score is -inf, every weight 0
            uint32_t pa[2];
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const float p0 = exp2f(sc[nt][0] + neg), p1 = exp2f(sc[nt][1] + neg);
                l += p0 + p1;                                    // fp32, unrounded; the product below takes the weights in bf16
                pa[nt] = pack2(p0, p1);
            }
            const int mi = lane >> 3;
#pragma unroll
            for (int jp = 0; jp < DH / 16; ++jp) {
                uint32_t b0, b1, b2, b3;
                ldsm4_t(sV + off(row0 + 8 * (mi & 1) + (lane & 7), 2 * jp + (mi >> 1)), b0, b1, b2, b3);
                if (!plain) { b0 &= keep0; b1 &= keep1; b2 &= keep0; b3 &= keep1; }
                mma_rows8(o[2 * jp], pa[0], pa[1], b0, b1);
                mma_rows8(o[2 * jp + 1], pa[0], pa[1], b2, b3);
            }
        }
        __syncwarp();
        if (ok && lane == 0) mbar_arrive(empty + 8 * st);
        const int b = w.b, kvh = w.kvh;
        const bool last = w.i + 1 == w.n;
        w.next(s, a.batch, a.Hkv);
        if (!last && u + 1 < u1) continue;

        // ---- the pair (or this run's part of it) is done: join the four warps, rows = heads
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if (c == 0) { s_m[warp][g] = m; s_l[warp][g] = l; }
        consumers_sync();
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int i = 0; i < kConsumers; ++i) M = fmaxf(M, s_m[i][g]);
#pragma unroll
        for (int i = 0; i < kConsumers; ++i) L += s_m[i][g] == -INFINITY ? s_l[i][g] : s_l[i][g] * exp2f(s_m[i][g] - M);      // (no position seen: the sum is 0)
        const float f = m == -INFINITY ? 0.f : exp2f(m - M);
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) { o[i][0] *= f; o[i][1] *= f; }
        // warps 2, 3 hand theirs to 0, 1; then 1 to 0
#pragma unroll
        for (int from = 2; from >= 1; --from) {
            if (warp >= from && warp < 2 * from) {
                float* dst = join + (size_t)(warp - from) * 8 * DH + g * DH + 2 * c;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<float2*>(dst + 8 * i) = make_float2(o[i][0], o[i][1]);
            }
            consumers_sync();
            if (warp < from) {
                const float* src = join + (size_t)warp * 8 * DH + g * DH + 2 * c;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) {
                    const float2 x = *reinterpret_cast<const float2*>(src + 8 * i);
                    o[i][0] += x.x; o[i][1] += x.y;
                }
            }
            consumers_sync();
        }
        if (warp == 0 && g < a.G) {
            const int head = kvh * a.G + g;
            if (last && !first_pair_open) {                      // all of the pair's tiles were in this run
                const float inv = L != 0.f ? 1.f / L : 0.f;
                uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<bf16*>(a.o) + ((size_t)b * a.Hq + head) * DH) + c;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) dst[4 * i] = pack2(o[i][0] * inv, o[i][1] * inv);
                if (c == 0 && a.lse != nullptr) a.lse[(size_t)b * a.Hq + head] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
            } else {
                float* dst = a.part + ((size_t)(2 * blockIdx.x + seg) * 8 + g) * (DH + 2);
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<float2*>(dst + 8 * i + 2 * c) = make_float2(o[i][0], o[i][1]);
                if (c == 0) { dst[DH] = M; dst[DH + 1] = L; }
            }
        }
        first_pair_open = false;
        seg = 1;
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = 0.f;
    }
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
template <typename T, int DH, int GM>
__global__ void __launch_bounds__((SimtCfg<T, DH, GM>::kWarps + 1) * 32, 2) paged_attn_simt_kernel(const __grid_constant__ PagedArgs a) {
    using S = SimtCfg<T, DH, GM>;
    constexpr int VN = S::VN, LPK = S::LPK, KPW = S::KPW, HV = S::HV, kSteps = S::kSteps;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
    float* s_o = reinterpret_cast<float*>(ring + S::kRing * S::kStage);                  // [kWarps / 2][GM][DH]
    __shared__ Schedule s;
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
    make_schedule(a, s);
    __syncthreads();
    finish_schedule(s);
    __syncthreads();
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
                    page = __ldcg(a.table + (size_t)a.slots.slot[w.b] * a.max_pages + (pos >> a.page_shift));
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
                if (h < a.G) {
                    const uint4 x = __ldcg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (size_t)w.b * a.q_stride + (size_t)(w.kvh * a.G + h) * DH + sub * VN));
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
        const bool whole = last && !first_pair_open;
        for (int i = threadIdx.x; i < a.G * DH; i += S::kWarps * 32) {
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
                float* dst = a.part + ((size_t)(2 * blockIdx.x + seg) * 8 + h) * (DH + 2);
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

template <int DH>
beagle_status launch_mma(const beagle_pages* p, const PagedArgs& a, int runs, cudaStream_t stream) {
    using SM = PagedSmem<DH>;
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
    if (!smem_attr.ensure([] { return cudaFuncSetAttribute(paged_attn_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::kBytes) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    launch_pdl(paged_attn_kernel<DH>, dim3(runs), dim3((kConsumers + 1) * 32), (size_t)SM::kBytes, stream, mk, mv, a);
    if (!a.whole) launch_pdl(paged_attn_join_kernel<bf16, DH>, dim3(runs, a.G), dim3(kJoinWarps * 32), 0, stream, a);
    return BEAGLE_OK;
}

template <typename T, int DH, int GM>
beagle_status launch_simt_heads(const PagedArgs& a, int runs, cudaStream_t stream) {
    using S = SimtCfg<T, DH, GM>;
    static PerDeviceOnce smem_attr;
    if (!smem_attr.ensure([] { return cudaFuncSetAttribute(paged_attn_simt_kernel<T, DH, GM>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    launch_pdl(paged_attn_simt_kernel<T, DH, GM>, dim3(runs), dim3((S::kWarps + 1) * 32), (size_t)S::kBytes, stream, a);
    return BEAGLE_OK;
}

template <typename T, int DH>
beagle_status launch_simt(const PagedArgs& a, int runs, cudaStream_t stream) {
    beagle_status st;
    if (a.G == 1) st = launch_simt_heads<T, DH, 1>(a, runs, stream);
    else if (a.G <= 2) st = launch_simt_heads<T, DH, 2>(a, runs, stream);
    else if (a.G <= 4) st = launch_simt_heads<T, DH, 4>(a, runs, stream);
    else if constexpr (DH < 256) st = launch_simt_heads<T, DH, 8>(a, runs, stream);
    else return BEAGLE_ERR_SHAPE;
    if (st != BEAGLE_OK) return st;
    if (!a.whole) launch_pdl(paged_attn_join_kernel<T, DH>, dim3(runs, a.G), dim3(kJoinWarps * 32), 0, stream, a);
    return BEAGLE_OK;
}

beagle_status check_heads(const beagle_pages* p, int Hq) {
    if (Hq <= 0) return BEAGLE_ERR_INVALID_ARG;
    if (Hq % p->n_kv_heads || Hq / p->n_kv_heads > 8) return BEAGLE_ERR_SHAPE;
    // the widest rows with more than four grouped heads: as for the decode step of the draft head, no kernel has that shape
    if (p->dtype == BEAGLE_BF16 && p->head_dim == 256 && Hq / p->n_kv_heads > 4) return BEAGLE_ERR_SHAPE;
    return BEAGLE_OK;
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
    if (batch < 0 || (batch > 0 && slot_host == nullptr)) return BEAGLE_ERR_INVALID_ARG;
    if (batch > kMaxCallBatch) return BEAGLE_ERR_CAPACITY;
    for (int i = 0; i < batch; ++i) {                   // a slot may be read by several rows of the call
        if (slot_host[i] < 0 || slot_host[i] >= p->max_slots) return BEAGLE_ERR_INVALID_ARG;
        a.slots.slot[i] = slot_host[i];
    }
    st = check_heads(p, n_q_heads);
    if (st != BEAGLE_OK) return st;
    if (window < 0 || sinks < 0) return BEAGLE_ERR_INVALID_ARG;
    if (batch == 0) return BEAGLE_OK;
    const int e = p->dtype == BEAGLE_BF16 ? 2 : 4;
    size_t need = 0;
    beagle_paged_attn_workspace_bytes(p, n_q_heads, window, sinks, &need);
    if (q_dev == nullptr || out_dev == nullptr || (need > 0 && ws_dev == nullptr) || q_stride < (int64_t)n_q_heads * p->head_dim) return BEAGLE_ERR_INVALID_ARG;
    if ((((uintptr_t)q_dev | (uintptr_t)out_dev | (uintptr_t)ws_dev) & 15) || (q_stride * e) % 16 || ((uintptr_t)lse_dev & 3)) return BEAGLE_ERR_INVALID_ARG;
    if (ws_bytes < need) return BEAGLE_ERR_CAPACITY;
    if (!paged_attn_fits(p, batch)) return BEAGLE_ERR_CAPACITY;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    a.table = p->table; a.length = p->length; a.k = p->k; a.v = p->v; a.q = q_dev; a.o = out_dev; a.lse = lse_dev;
    a.q_stride = q_stride;
    a.batch = batch; a.n_pages = p->n_pages; a.max_pages = p->max_pages;
    a.page_shift = 0;
    while ((1 << a.page_shift) < p->page_size) ++a.page_shift;
    a.Hq = n_q_heads; a.Hkv = p->n_kv_heads; a.G = n_q_heads / p->n_kv_heads;
    a.window = window; a.sinks = sinks;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)p->head_dim);
    // no more runs than the cache's capacity has tiles
    const long long most = (long long)batch * p->n_kv_heads * most_tiles(p, window, sinks);
    const bool mma = uses_mma(p);
    a.whole = whole_pairs(p, n_q_heads, window, sinks) ? 1 : 0;
    long long runs = (long long)device_sm_count() * (mma ? kCtasPerSm : kSimtCtasPerSm);
    if (runs > kMaxRuns) runs = kMaxRuns;
    if (runs > most) runs = most;
    if (a.whole) runs = (long long)batch * p->n_kv_heads;
    a.join = static_cast<JoinItem*>(ws_dev);
    a.part = a.whole ? nullptr : reinterpret_cast<float*>(a.join + runs);
    if (mma) st = p->head_dim == 128 ? launch_mma<128>(p, a, (int)runs, stream) : launch_mma<64>(p, a, (int)runs, stream);
    else if (p->dtype == BEAGLE_BF16) st = p->head_dim == 256 ? launch_simt<bf16, 256>(a, (int)runs, stream) : launch_simt<bf16, 32>(a, (int)runs, stream);
    else if (p->head_dim == 128) st = launch_simt<float, 128>(a, (int)runs, stream);
    else if (p->head_dim == 64) st = launch_simt<float, 64>(a, (int)runs, stream);
    else if (p->head_dim == 32) st = launch_simt<float, 32>(a, (int)runs, stream);
    else st = launch_simt<float, 16>(a, (int)runs, stream);
    if (st != BEAGLE_OK) return st;
    return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

}  // extern "C"
