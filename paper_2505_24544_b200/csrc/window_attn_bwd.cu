// Backward of the windowed attention, bf16, head_dim 64 / 128 (tcgen05).
//
// With P = softmax over the visible keys (recomputed from the forward's log-sum-exp), dP = dO V^T, delta = rowsum(dO * O) and
// dS = P * (dP - delta):      dQ = dS K / sqrt(dh),   dK = dS^T Q / sqrt(dh),   dV = P^T dO.
//
// Two kernels and no atomics, so every sum has one order: a single kernel over keys would have to add dQ across CTAs, which costs
// either that order or an fp32 copy of dQ per key tile.  Recomputing S and dP costs 7 products instead of 5.
//   query side  one CTA = 128 queries of one (sequence, query head), 128 keys at a time:  S = Q K^T, dP = dO V^T -> dS in bf16
//               over S in tensor memory -> dQ += dS K.  S is double-buffered, so the next tile's S runs under this tile's
//               element-wise work, and dQ and the next dP under the next tile's exponentials.  It also forms delta and leaves
//               it, with the log-sum-exp, side by side for the key side.
//   key side    one CTA = 128 keys of one (sequence, K/V head), 128 queries at a time for every query head of the group:
//               S^T = K Q^T -> P^T over S^T -> dV += P^T dO, and dP^T = V dO^T -> dS^T over dP^T -> dK += dS^T Q.  The two
//               halves take turns: while the threads form P of the next tile, dK and the next dP^T run, while they form dS,
//               dV and the next S^T run.
// Both use all 512 columns of tensor memory and about 200 KB of shared memory: one CTA per SM, two threads per tile row.  The
// query side's grid is one CTA per SM and walks the items, the pipeline running on across them: the copies and the first products
// of an item start under the last products and the epilogue of the one before it (as CTAs of their own, items of five tiles spent 7 us
// of 16 on starting up and draining).  So is the key side's where a band has few jobs; longer items are CTAs of their own (launch_bwd).
// P and dS are the tensor-memory operands of their products (rows = lanes), so the accumulating products read one operand
// from shared memory, and Q, dO, K tiles serve both as K-major and as MN-major operands: nothing is copied or transposed.
// They are rounded to bf16 for that, the operand type that V, dO, K and Q have.  delta is summed in fp32 from the forward's output as it is
// stored, in bf16: sum_j P dP, which needs no O, is known only when all of a row's keys have been seen, and then dS would take a
// second pass over them; an fp32 O from the forward would be twice the bytes.  With short windows this rounding costs dQ more than
// that of dS (relative error of dQ in a model on the CPU, 512 rows, head_dim 128, with nothing but the result rounded, with dS, with O
// and with both: window 2: 1.7, 2.4, 4.0, 5.3e-3; window 8: 1.7, 2.3, 2.4, 3.3e-3; window 512: 1.7, 2.4, 1.9, 2.7e-3).
//
// The sinks' keys are read by every later query.  What lies past the band of a key tile is therefore cut into segments of
// similar length, each a CTA of its own that leaves fp32 partials of the (few) sink rows; a last small launch adds them to the
// band's partial in the order of the queries.  Where the key tiles are too few for the GPU, several CTAs share the jobs of one and
// leave fp32 partials that a launch adds in order (splits).
//
// Rows behind a sequence (the next one's) are zeroed in shared memory where they would be multiplied by a weight of 0.
// Every wait is bounded; a CTA that gives up leaves NaN in its rows.
//
// Measured (head_dim 128, 32 heads): 8 x 2048, window 512: query side 319 us, key side 408 (tensor pipe 0.39 and 0.44 of its cycles,
// nothing else above 0.3 but issue slots); two sequences up to 8191, window 2048, 4 heads a group: 650 and 700.  A key-side job takes
// 3050 cycles there, of which its four products are 2048: the threads form P for 1450 (special-function unit 1024), then dS for 730, and
// wait some 500 for the next scores, whose place P holds until dV has read it.
#include <cstring>

#include "tc_ptx.cuh"
#include "tensor_map.h"
#include "win_ptx.cuh"
#include "window_attn.h"

namespace beagle {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;


__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fffffff); }

__device__ __forceinline__ int stat_row0(const WinSeqs& s, int b) {      // first row of sequence b in WinArgs::stats
    int at = 0;
    for (int i = 0; i < b; ++i) at += (s.q_len[i] + kStatPad - 1) / kStatPad * kStatPad;
    return at;
}

// A warp's 32 rows x DH / 2 columns of an accumulator (columns from taddr; not read when `zero`), scaled, as bf16 to global
// memory: through a slab of shared memory and one TMA store when all 32 rows are this CTA's to write (rows of 64 to 128 bytes at
// once instead of 16 a lane), else row by row.  (c0, c1): the store's coordinates; dst: this lane's row.
template <int DH>
__device__ __forceinline__ void store_rows(uint32_t taddr, float scale, bool zero, const CUtensorMap* tm, uint8_t* slab, int c0, int c1, bf16* dst, bool write,
                                           int lane) {
    const bool whole = __all_sync(0xffffffffu, write);
    if (whole) {
        if (lane == 0) store_done();                             // the slab's last store has read it
        __syncwarp();
    }
#pragma unroll 1
    for (int c = 0; c < DH / 2; c += 16) {
        uint32_t o[16], y[8];
        if (!zero) { tmem_ld16(taddr + c, o); tmem_ld_wait(); }
#pragma unroll
        for (int z = 0; z < 8; ++z) y[z] = zero ? 0u : pack_bf16(__uint_as_float(o[2 * z]) * scale, __uint_as_float(o[2 * z + 1]) * scale);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int chunk = c / 8 + i, place = DH == 128 ? chunk ^ (lane & 7) : chunk ^ ((lane >> 1) & 3);
            const uint4 v = make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
            if (whole) *reinterpret_cast<uint4*>(slab + lane * DH + place * 16) = v;
            else if (write) *reinterpret_cast<uint4*>(dst + 8 * chunk) = v;
        }
    }
    if (whole) {
        fence_async_smem();
        __syncwarp();
        if (lane == 0) tma_store_2d(tm, smem_u32(slab), c0, c1);
    }
}

// The element-wise parts are written once, for whole tiles: masked scores become -inf beforehand, so their P is exactly 0, and
// the rows behind a sequence are zeroed in shared memory, so that dP is finite wherever P is 0 and dS = 0 follows.  (A second,
// masked copy of the unrolled code cost more in instruction fetches than its absence does in selects.)
__device__ __forceinline__ void mask32(uint32_t* r, uint32_t vis) {
#pragma unroll
    for (int x = 0; x < 32; ++x) r[x] = (vis >> x & 1u) ? r[x] : 0xff800000u;
}
// 32 columns of a tile: P = exp2(S * scale - lse), kept as fp32 in r.  nl(x) gives the negated log-sum-exp of columns x, x + 1.
template <typename NegLse>
__device__ __forceinline__ void chunk_p(uint32_t* r, uint64_t scale2, NegLse nl) {
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
        float e0, e1;
        un2(fma2(pk2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), scale2, nl(x)), e0, e1);
        r[x] = __float_as_uint(exp2f(e0));
        r[x + 1] = __float_as_uint(exp2f(e1));
    }
}
// dS = P * (dP - delta) of 32 columns as bf16 pairs.
template <typename NegDelta>
__device__ __forceinline__ void chunk_ds(const uint32_t* p, const uint32_t* d, NegDelta nd, uint32_t* y) {
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
        float d0, d1;
        un2(mul2(pk2(__uint_as_float(p[x]), __uint_as_float(p[x + 1])), add2(pk2(__uint_as_float(d[x]), __uint_as_float(d[x + 1])), nd(x))), d0, d1);
        y[x >> 1] = pack_bf16(d0, d1);
    }
}

// ---------------------------------------------------------------------------------------------------------------- query side
// warp 0: TMA producer, warp 1: MMA issuer, warps 2-9: two threads per tile row, 64 columns each; query side: warps 10, 11 form delta
constexpr int kThreads = 320, kQThreads = 384;

template <int DH>
struct BwdQSmem {
    static constexpr int kT = kQTile * DH * 2;           // Q, dO, and a K or V tile (three stages of K, one of V)
    static constexpr int kSlab = 32 * DH;                // a warp's rows on their way out
    static constexpr int kBytes = 6 * kT + 8 * kSlab + 4 * kQTile * 4 + 256;
};

// The key tiles of one query tile: sinks [0, sink_end) first, then the band [lo, hi).
struct KeyWalk {
    int lo, hi, sink_end, n_sink, n;
    __device__ __forceinline__ void init(int q0, int q_len, int shift, int window, int sinks) {
        hi = min(q0 + kQTile, q_len) + shift;
        lo = max(0, q0 + shift - window + 1);
        sink_end = min(sinks, lo);
        n_sink = (sink_end + kKTile - 1) / kKTile;
        n = hi > 0 ? n_sink + (hi - lo + kKTile - 1) / kKTile : 0;
    }
    __device__ __forceinline__ void tile(int j, int& start, int& end) const {
        if (j < n_sink) { start = j * kKTile; end = min(start + kKTile, sink_end); }
        else { start = lo + (j - n_sink) * kKTile; end = min(start + kKTile, hi); }
    }
};

// The items of a persistent grid: round after round, every other one backwards, so that neighbours in cost spread over the CTAs.
__device__ __forceinline__ int item_at(int round) {
    const int c = (round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    return round * gridDim.x + c;
}

struct QItem {                           // 128 queries of one (sequence, query head)
    int b, h, q0, q_len, kv_len, shift, q_row, k_row;
    KeyWalk w;
    __device__ __forceinline__ void load(int at, const WinArgs& a, const WinSeqs& s) {
        int tile;
        const int unit = at / a.Hq;
        h = at - unit * a.Hq;
        b = win_find(s.item, a.batch, unit, tile);
        q_len = s.q_len[b];
        kv_len = s.kv_len[b];
        shift = kv_len - q_len - a.strict;
        q0 = ((q_len + kQTile - 1) / kQTile - 1 - tile) * kQTile;            // the latest (longest) tiles first
        q_row = s.q_start[b] + q0;
        k_row = s.k_start[b];
        w.init(q0, q_len, shift, a.window, a.sinks);
    }
};

template <int DH>
__global__ void __launch_bounds__(kQThreads, 1) window_bwd_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                 const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                 const __grid_constant__ CUtensorMap tmdQ, const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    using SM = BwdQSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 512, kDP = 256, kDQ = 384;    // S / dS at columns 0 and 128, dP at 256, dQ at 384
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sQ = smem_u32(smem), sdO = sQ + SM::kT, sV = sdO + SM::kT, sK = sV + SM::kT;     // stage s of K at sK + s kT
    float* s_stat = reinterpret_cast<float*>(smem + 6 * SM::kT + 8 * SM::kSlab);                     // [2][2][128]: -lse (log2 units) and -delta, two items
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 6 * SM::kT + 8 * SM::kSlab + 4 * kQTile * 4);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, dp_full = bar0 + 8, ds_full = bar0 + 16, q_empty = bar0 + 24, v_full = bar0 + 32, v_empty = bar0 + 40, v_fixed = bar0 + 48;
    const uint32_t s_full = bar0 + 56, stat_full = bar0 + 72, stat_empty = bar0 + 88;          // two each
    const uint32_t k_full = bar0 + 104, k_empty = bar0 + 128, k_fixed = bar0 + 152;            // one per stage of K
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 24);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 25);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int items = seqs.item[a.batch] * a.Hq;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(dp_full, 1); mbar_init(ds_full, 8);
        mbar_init(v_full, 1); mbar_init(v_empty, 1); mbar_init(v_fixed, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(stat_full + 8 * i, 2); mbar_init(stat_empty + 8 * i, 8); }
        for (int i = 0; i < 3; ++i) { mbar_init(k_full + 8 * i, 1); mbar_init(k_empty + 8 * i, 1); mbar_init(k_fixed + 8 * i, 1); }
        *s_abort = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc<kTmem>(smem_u32(&s_tmem));
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);

    if (warp == 0) {
        bool ok = true;
        int n = 0, st = 0, ph = 0, k_issued = 0, v_issued = 0, loaded = 0;       // tiles walked, K's stage and round, copies, items with tiles
        for (int r = 0, at; ok && (at = item_at(r)) < items; ++r) {
            QItem x;
            x.load(at, a, seqs);
            if (x.w.n == 0) continue;
            ok = warp_wait(q_empty, (loaded & 1) ^ 1, s_abort);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(q_full, 2 * SM::kT);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    tma_load_2d(sQ + hf * (kQTile * 128), &tmQ, q_full, x.h * DH + hf * 64, x.q_row);
                    tma_load_2d(sdO + hf * (kQTile * 128), &tmdO, q_full, x.h * DH + hf * 64, x.q_row);
                }
            }
            __syncwarp();
            ++loaded;
            const int col = x.h / a.G * DH;
#pragma unroll 1
            for (int j = 0; j < x.w.n; ++j, ++n) {
                int start, end;
                x.w.tile(j, start, end);
                const int boxes = (end - start + 63) / 64;       // of 64 keys
                auto load = [&](const CUtensorMap* tm, uint32_t dst, uint32_t bar) {
                    if (lane == 0) {
                        mbar_expect_tx(bar, boxes * kHalves * 64 * 128);
                        for (int y = 0; y < boxes; ++y)
#pragma unroll
                            for (int hf = 0; hf < kHalves; ++hf)
                                tma_load_2d(dst + hf * (kKTile * 128) + y * (64 * 128), tm, bar, col + hf * 64, x.k_row + start + 64 * y);
                    }
                    __syncwarp();
                };
                ok = warp_wait(k_empty + 8 * st, ph ^ 1, s_abort);
                if (!ok) break;
                load(&tmK, sK + st * SM::kT, k_full + 8 * st);
                ++k_issued;
                ok = warp_wait(v_empty, (n & 1) ^ 1, s_abort);
                if (!ok) break;
                load(&tmV, sV, v_full);
                ++v_issued;
                const int cols = (end - start + 31) & ~31;
                if (start + cols > x.kv_len) {                   // rows behind the sequence: zero
                    ok = warp_wait2(k_full + 8 * st, ph, v_full, n & 1, s_abort);
                    if (!ok) break;
                    zero_rows<DH>(smem + 3 * SM::kT + st * SM::kT, kKTile, x.kv_len - start, cols, lane);
                    zero_rows<DH>(smem + 2 * SM::kT, kKTile, x.kv_len - start, cols, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(k_fixed + 8 * st); mbar_arrive(v_fixed); }
                }
                if (++st == 3) { st = 0; ph ^= 1; }
            }
        }
        if (!ok) {                                               // copies already requested still land (bounded)
            for (uint32_t i = 0; loaded > 0 && i < kSpinLimit && !mbar_try_wait(q_full, (loaded - 1) & 1); ++i) {}
            for (uint32_t i = 0; v_issued > 0 && i < kSpinLimit && !mbar_try_wait(v_full, (v_issued - 1) & 1); ++i) {}
            for (int c = max(0, k_issued - 3); c < k_issued; ++c)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(k_full + 8 * (c % 3), (c / 3) & 1); ++i) {}
        }
    } else if (warp == 1) {
        const bool leader = elect_one();
        constexpr uint32_t idesc_q = make_idesc_major(kQTile, DH, false, true);
        bool ok = true;
        uint32_t fixed = 0;                                      // phases of the repair barriers (V's in bit 3)
        // The walk of S and dP runs one tile ahead of the walk of dQ, across items.
        QItem x;
        int r = -1, j = 0, n = -1, loaded = -1;                  // x's round, its tile, tiles before this one, items with tiles before x
        int st = 2, ph = 1;                                      // K's stage and round of tile n
        bool more = true;
        int cols = 0, start = 0;
        auto advance = [&]() {
            ++n;
            if (++st == 3) { st = 0; ph ^= 1; }
            if (r >= 0 && ++j < x.w.n) {
            } else {
                j = 0;
                for (;;) {
                    const int at = item_at(++r);
                    more = at < items;
                    if (!more) return;
                    x.load(at, a, seqs);
                    if (x.w.n > 0) break;
                }
                ++loaded;
            }
            int end;
            x.w.tile(j, start, end);
            cols = (end - start + 31) & ~31;
        };
        auto product = [&](uint32_t dst, uint32_t A, uint32_t B) {       // [128 x DH] x [cols x DH]^T, both K-major
            const uint32_t idesc = make_idesc(kQTile, cols);
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) {
                const uint64_t da = umma_desc(A + hf * (kQTile * 128)), db = umma_desc(B + hf * (kKTile * 128));
#pragma unroll
                for (int k = 0; k < BK / UMMA_K; ++k) {
                    const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                    umma_ss(leader, dst, da + off, db + off, idesc, (hf > 0 || k > 0) ? 1u : 0u);
                }
            }
        };
        auto issue_s = [&]() {
            if (j == 0) ok = warp_wait(q_full, loaded & 1, s_abort);
            if (ok) ok = warp_wait(k_full + 8 * st, ph, s_abort);
            if (ok && start + cols > x.kv_len) { ok = warp_wait(k_fixed + 8 * st, fixed >> st & 1u, s_abort); fixed ^= 1u << st; }
            if (!ok) return;                                     // (dQ has read dS of tile n - 2: the walk of dQ waits for it before tile n)
            fence_after();
            product(tmem + 128 * (n & 1), sQ, sK + st * SM::kT);
            commit_el(leader, s_full + 8 * (n & 1));
        };
        auto issue_dp = [&]() {
            if (ok) ok = warp_wait(v_full, n & 1, s_abort);
            if (ok && start + cols > x.kv_len) { ok = warp_wait(v_fixed, fixed >> 3 & 1u, s_abort); fixed ^= 8u; }
            if (!ok) return;
            fence_after();
            product(tmem + kDP, sdO, sV);
            commit_el(leader, v_empty);
            commit_el(leader, dp_full);
            if (j + 1 == x.w.n) commit_el(leader, q_empty);      // the item's last products with Q and dO
        };
        advance();
#pragma unroll 1
        for (int t = -1; ok; ++t) {                              // tile t's dQ, tile t + 1's S and dP; x is at tile max(t, 0) here
            const int t_st = st, t_ph = ph, t_cols = cols;
            const bool first = j == 0;
            if (t >= 0) {
                if (!more) break;
                // dS of tile t - 1 lies where S of tile t + 1 goes
                if (t > 0) ok = warp_wait(k_empty + 8 * (t_st == 0 ? 2 : t_st - 1), t_st == 0 ? t_ph ^ 1 : t_ph, s_abort);
                advance();
            }
            if (more) issue_s();
            if (t >= 0) {
                if (ok) ok = warp_wait(ds_full, t & 1, s_abort); // dS is written, dP has been read (and the last item's dQ, if this is a first tile)
                if (!ok) break;
                fence_after();
                const uint64_t dk = umma_desc_mn(sK + t_st * SM::kT, kKTile * 128);
#pragma unroll 1
                for (int k = 0; k < t_cols / UMMA_K; ++k)
                    umma_ts(leader, tmem + kDQ, tmem + 128 * (t & 1) + (k >> 2) * 64 + (k & 3) * 8, dk + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_q,
                            (!first || k > 0) ? 1u : 0u);
                commit_el(leader, k_empty + 8 * t_st);
            }
            if (more) issue_dp();
        }
    } else if (warp >= 10) {
        // ---- delta = dO . O of every query, an item ahead of the others; 16 bytes a lane, so DH / 8 lanes to a row
        // (a small rolled loop, eight rows of both operands in flight: what it has to hide is memory latency and instruction fetches)
        constexpr int kLanes = DH / 8, kRows = 32 / kLanes, kUnroll = 8;
        const int sub = lane % kLanes, in = lane / kLanes;
        bool ok = true;
        for (int r = 0, at; ok && (at = item_at(r)) < items; ++r) {
            QItem x;
            x.load(at, a, seqs);
            ok = warp_wait(stat_empty + 8 * (r & 1), ((r >> 1) & 1) ^ 1, s_abort);
            if (!ok) break;
            float* part = s_stat + (r & 1) * 2 * kQTile;
            float* stat = a.stats + (size_t)x.h * 2 * a.stat_rows + stat_row0(seqs, x.b) + x.q0;
            const uint4* dout = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.dout) + (size_t)x.q_row * a.dout_stride + (size_t)x.h * DH) + sub;
            const uint4* out = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.out) + ((size_t)x.q_row * a.Hq + x.h) * DH) + sub;
            const float* lse = a.lse + (size_t)x.q_row * a.Hq + x.h;
            const int rows = min(kQTile, x.q_len - x.q0), blind = -x.shift - x.q0;       // rows of the tile; those below `blind` see nothing
#pragma unroll 1
            for (int r0 = (warp - 10) * 64 + in; r0 < (warp - 9) * 64; r0 += kRows * kUnroll) {
                uint4 g[kUnroll], o[kUnroll];
                float l[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const int row = min(r0 + u * kRows, rows - 1);
                    g[u] = __ldg(dout + row * (a.dout_stride / 8));
                    o[u] = __ldg(out + row * (a.Hq * DH / 8));
                    l[u] = __ldg(lse + row * a.Hq);
                }
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    float e[8], f[8], delta = 0.f;
                    unpack16<bf16>(g[u], e);
                    unpack16<bf16>(o[u], f);
#pragma unroll
                    for (int z = 0; z < 8; ++z) delta = fmaf(e[z], f[z], delta);
#pragma unroll
                    for (int d = 1; d < kLanes; d <<= 1) delta += __shfl_xor_sync(0xffffffffu, delta, d);
                    const int row = r0 + u * kRows;
                    const bool sees = row >= blind;
                    const float nls = sees ? -l[u] * kLog2e : 0.f, nds = sees ? -delta : 0.f;
                    if (sub == 0) {
                        part[row] = nls;
                        part[kQTile + row] = nds;
                        if (row < rows) {                        // for the key side, each in a row of its own
                            stat[row] = nls;
                            stat[a.stat_rows + row] = nds;
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(stat_full + 8 * (r & 1));
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;          // tensor-memory lane quarter; which 64 columns of a tile
        const int row = q * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const uint64_t scale2 = pk2(a.scale_log2, a.scale_log2);
        bool ok = true;
        int n = 0;
        for (int r = 0, at; (at = item_at(r)) < items; ++r) {
            QItem x;
            x.load(at, a, seqs);
            const int i = x.q0 + row;
            const bool valid = i < x.q_len;
            const int last = i + x.shift, oldest = last - a.window + 1;
            const int full_lo = min(x.q0 + kQTile, x.q_len) - 1 + x.shift - a.window + 1, full_hi = x.q0 + x.shift + 1;
            if (ok) ok = warp_wait(stat_full + 8 * (r & 1), (r >> 1) & 1, s_abort);
            const float nls = s_stat[(r & 1) * 2 * kQTile + row], nds = s_stat[((r & 1) * 2 + 1) * kQTile + row];
            __syncwarp();
            if (lane == 0) mbar_arrive(stat_empty + 8 * (r & 1));
            const uint64_t nl2 = pk2(nls, nls), nd2 = pk2(nds, nds);
            auto nl = [&](int) { return nl2; };
            auto nd = [&](int) { return nd2; };
            for (int j = 0; j < x.w.n; ++j, ++n) {
                const int st = n & 1;
                int start, end;
                x.w.tile(j, start, end);
                start += 64 * half;                              // this thread's columns
                const bool one = start < end, two = start + 32 < end;
                const bool full = start + 64 <= min(end, full_hi) && (start >= full_lo || start + 64 <= a.sinks);
                if (ok) ok = warp_wait(s_full + 8 * st, (n >> 1) & 1, s_abort);
                const uint32_t ts = tmem + 128 * st + 64 * half + lanes;
                uint32_t s[2][32], d[2][32], y[2][16];
                if (ok && one) {
                    fence_after();
                    tmem_ld32(ts, s[0]);
                    if (two) tmem_ld32(ts + 32, s[1]);
                    tmem_ld_wait();
                    if (!full) {
                        const int top = valid ? min(last + 1, end) - start : 0, sink_top = min(a.sinks - start, top);
                        mask32(s[0], bit_range(oldest - start, top) | bit_range(0, sink_top));
                        mask32(s[1], bit_range(oldest - start - 32, top - 32) | bit_range(0, sink_top - 32));
                    }
                    chunk_p(s[0], scale2, nl);
                    if (two) chunk_p(s[1], scale2, nl);
                }
                if (ok) ok = warp_wait(dp_full, n & 1, s_abort);
                if (!ok) continue;
                fence_after();
                if (one) {
                    tmem_ld32(tmem + kDP + 64 * half + lanes, d[0]);
                    if (two) tmem_ld32(tmem + kDP + 64 * half + 32 + lanes, d[1]);
                    tmem_ld_wait();
                    chunk_ds(s[0], d[0], nd, y[0]);
                    tmem_st16(ts, y[0]);                         // dS of this half over its own S columns
                    if (two) {
                        chunk_ds(s[1], d[1], nd, y[1]);
                        tmem_st16(ts + 16, y[1]);
                    }
                    tmem_st_wait();
                }
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(ds_full);
            }
            if (x.w.n > 0 && ok) ok = warp_wait(k_empty + 8 * ((n - 1) % 3), ((n - 1) / 3) & 1, s_abort);       // the item's last dQ
            fence_after();
            bf16* dst = static_cast<bf16*>(a.dq) + (size_t)(x.q_row + row) * a.dq_stride + (size_t)x.h * DH + half * (DH / 2);
            store_rows<DH>(tmem + kDQ + half * (DH / 2) + lanes, ok ? a.scale : nan_f(), x.w.n == 0, &tmdQ, smem + 6 * SM::kT + (warp - 2) * SM::kSlab,
                           x.h * DH + half * (DH / 2), x.q_row + q * 32, dst, valid, lane);
        }
    }
    if (lane == 0) store_done();                                 // this warp's last stores have read their slab
    fence_before();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        tmem_dealloc<kTmem>(tmem);
    }
}

// ------------------------------------------------------------------------------------------------------------------ key side
template <int DH>
struct BwdKSmem {
    static constexpr int kT = kKTile * DH * 2;           // K, V, and a tile of Q or dO (two stages)
    static constexpr int kStat = kQTile * 4;             // -lse, and -delta, of a query tile (two stages of each)
    static constexpr int kSlab = 32 * DH;                // a warp's rows on their way out
    static constexpr int kBytes = 6 * kT + 8 * kSlab + 4 * kStat + 256;
};

// The query tiles that a CTA of the key side reads: of every head of the group, from `from` in steps of 128 up to `to`.
struct QueryWalk {
    int from, to, n;                     // n tiles per head
    __device__ __forceinline__ void init(int f, int t) {
        from = max(f, 0) & ~3;           // (a multiple of four: the statistics are copied in 16-byte pieces)
        to = t;
        n = to > from ? (to - from + kQTile - 1) / kQTile : 0;
    }
};
// First query past the band of the key tile at k0: none of its keys is inside the window of a later query.
__device__ __forceinline__ int band_end(int k0, int kv_len, int q_len, int shift, int window) {
    const int last_key = min(k0 + kKTile, kv_len) - 1;
    return max(0, min(q_len, last_key - shift + window));
}

// One item: 128 keys of one (sequence, K/V head) and the queries of its band, or a segment of the queries past the band.
// Per sequence the grid's list has first the segments of each of its sinks' key tiles, then its key tiles (bands).
struct KItem {
    int b, kvh, k0, q_len, kv_len, shift, k_row, seg, band, n;      // seg: -1 = band; band: first query past it; n: jobs
    int j0, split;                       // first job; which of the tile's splits
    QueryWalk w;
    template <bool SPLIT>                // the jobs of a tile are shared
    __device__ __forceinline__ void load(int at, const WinArgs& a, const WinSeqs& s) {
        int item;
        const int splits = SPLIT ? a.splits : 1;
        const int unit = at / a.Hkv;                             // the heads of a tile side by side: the cheap tiles, the last ones, stay for the end
        kvh = at - unit * a.Hkv;
        b = win_find(s.item, a.batch, unit, item);
        q_len = s.q_len[b];
        kv_len = s.kv_len[b];
        shift = kv_len - q_len - a.strict;
        const int segs = s.segs[b], parts = (min(a.sinks, kv_len) + kKTile - 1) / kKTile * segs;
        const bool sink_part = item < parts;
        seg = sink_part ? item % segs : -1;
        const int tile = sink_part ? item / segs : (item - parts) / splits;
        split = SPLIT && !sink_part ? item - parts - tile * splits : 0;
        k0 = tile * kKTile;
        k_row = s.k_start[b] + k0;
        band = band_end(k0, kv_len, q_len, shift, a.window);
        j0 = 0;
        n = 0;
        if (!sink_part) {
            w.init(k0 - shift, band);
            const int total = w.n * a.G;
            j0 = total * split / splits;
            n = total * (split + 1) / splits - j0;
        } else {
            w.init(band, q_len);
            const int total = w.n * a.G;
            j0 = (int)((long long)total * seg / segs);
            n = (int)((long long)total * (seg + 1) / segs) - j0;
        }
    }
};
// Place of a key tile and K/V head in WinArgs::split_part.
__device__ __forceinline__ int key_unit(int b, int tile, int kvh, const WinArgs& a, const WinSeqs& s) {
    int at = tile;
    for (int i = 0; i < b; ++i) at += (s.kv_len[i] + kKTile - 1) / kKTile;
    return at * a.Hkv + kvh;
}
// Jobs of an item in order: the tiles of one head after the other.
struct Job {
    int h, qb, left;                     // query head, first query, tiles left of this head
    __device__ __forceinline__ void first(const KItem& x, int G) {
        const int skip = x.j0 > 0 ? x.j0 / x.w.n : 0, in = x.j0 - skip * x.w.n;
        h = x.kvh * G + skip;
        qb = x.w.from + in * kQTile;
        left = x.w.n - in;
    }
    __device__ __forceinline__ void next(const KItem& x) {
        qb += kQTile;
        if (--left == 0) { ++h; qb = x.w.from; left = x.w.n; }
    }
};

template <int DH, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1) window_bwd_kv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                  const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                  const __grid_constant__ CUtensorMap tmdK, const __grid_constant__ CUtensorMap tmdV,
                                                                  const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    using SM = BwdKSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 512, kY = 128, kDV = 256, kDK = 256 + DH;     // S^T / P^T at column 0, dP^T / dS^T at 128
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sK = smem_u32(smem), sV = sK + SM::kT, sQ = sV + SM::kT;      // stage s: Q at sQ + 2 s kT, dO behind it
    constexpr int kStatAt = 6 * SM::kT + 8 * SM::kSlab;
    const uint32_t sStat = sK + kStatAt;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStatAt + 4 * SM::kStat);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t kv_full = bar0, s_full = bar0 + 8, dp_full = bar0 + 16, ds_full = bar0 + 24, kv_empty = bar0 + 32;
    // one per stage; Q is free when dK has read it (so is dS^T's place), dO when dV has (so is P^T's place)
    const uint32_t q_full = bar0 + 40, do_full = bar0 + 56, y_free = bar0 + 72, x_free = bar0 + 88, stat_empty = bar0 + 104, q_fixed = bar0 + 120,
                   do_fixed = bar0 + 136;
    const uint32_t p_full = bar0 + 152;                  // P^T in two parts: the first 32 queries of each half of the tile, then the others
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 24);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 25);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int items = seqs.item[a.batch] * a.Hkv;

    if (threadIdx.x == 0) {
        mbar_init(kv_full, 1); mbar_init(kv_empty, 1); mbar_init(s_full, 1); mbar_init(p_full, 8); mbar_init(p_full + 8, 8); mbar_init(dp_full, 1); mbar_init(ds_full, 8);
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + 8 * i, 1); mbar_init(do_full + 8 * i, 1); mbar_init(y_free + 8 * i, 1); mbar_init(x_free + 8 * i, 1);
            mbar_init(stat_empty + 8 * i, 8); mbar_init(q_fixed + 8 * i, 1); mbar_init(do_fixed + 8 * i, 1);
        }
        *s_abort = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc<kTmem>(smem_u32(&s_tmem));
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);

    if (warp == 0) {
        bool ok = true;
        int n = 0, issued = 0, loaded = 0;                       // jobs walked, copies of Q and dO, items with jobs
        for (int r = 0, at; ok && (at = item_at(r)) < items; ++r) {
            KItem x;
            x.load<SPLIT>(at, a, seqs);
            if (x.n == 0) continue;
            ok = warp_wait(kv_empty, (loaded & 1) ^ 1, s_abort);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(kv_full, 2 * SM::kT);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    tma_load_2d(sK + hf * (kKTile * 128), &tmK, kv_full, x.kvh * DH + hf * 64, x.k_row);
                    tma_load_2d(sV + hf * (kKTile * 128), &tmV, kv_full, x.kvh * DH + hf * 64, x.k_row);
                }
            }
            __syncwarp();
            ++loaded;
            const int stat0 = stat_row0(seqs, x.b), q_start = seqs.q_start[x.b];
            Job job;
            job.first(x, a.G);
            for (int j = 0; j < x.n; ++j, ++n, job.next(x)) {
                const int st = n & 1, ph = (n >> 1) & 1, h = job.h, qb = job.qb;
                const uint32_t dst = sQ + st * 2 * SM::kT;
                uint8_t* tile = smem + (2 + 2 * st) * SM::kT;
                ok = warp_wait(x_free + 8 * st, ph ^ 1, s_abort);        // dO is free first
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(do_full + 8 * st, SM::kT);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
                        tma_load_2d(dst + SM::kT + hf * (kQTile * 128), &tmdO, do_full + 8 * st, h * DH + hf * 64, q_start + qb);
                }
                __syncwarp();
                ++issued;
                ok = warp_wait2(y_free + 8 * st, ph ^ 1, stat_empty + 8 * st, ph ^ 1, s_abort);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(q_full + 8 * st, SM::kT + 2 * SM::kStat);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(dst + hf * (kQTile * 128), &tmQ, q_full + 8 * st, h * DH + hf * 64, q_start + qb);
                    const float* stat = a.stats + (size_t)h * 2 * a.stat_rows + stat0 + qb;
                    bulk_load(sStat + st * 2 * SM::kStat, stat, SM::kStat, q_full + 8 * st);
                    bulk_load(sStat + st * 2 * SM::kStat + SM::kStat, stat + a.stat_rows, SM::kStat, q_full + 8 * st);
                }
                __syncwarp();
                ++issued;
                if (qb + kQTile > x.q_len) {
                    // rows behind the sequence: zero, and their statistics
                    ok = warp_wait2(q_full + 8 * st, ph, do_full + 8 * st, ph, s_abort);
                    if (!ok) break;
                    zero_rows<DH>(tile, kQTile, x.q_len - qb, kQTile, lane);
                    zero_rows<DH>(tile + SM::kT, kQTile, x.q_len - qb, kQTile, lane);
                    float* stat = reinterpret_cast<float*>(smem + kStatAt + st * 2 * SM::kStat);
                    for (int i = x.q_len - qb + lane; i < kQTile; i += 32) stat[i] = stat[kQTile + i] = 0.f;
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(q_fixed + 8 * st); mbar_arrive(do_fixed + 8 * st); }
                }
            }
        }
        if (!ok) {                                               // copies already requested still land (bounded)
            for (uint32_t i = 0; loaded > 0 && i < kSpinLimit && !mbar_try_wait(kv_full, (loaded - 1) & 1); ++i) {}
            for (int c = max(0, issued - 4); c < issued; ++c)    // copy c: dO of tile c / 2 if even, Q if odd
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait((c & 1 ? q_full : do_full) + 8 * ((c >> 1) & 1), (c >> 2) & 1); ++i) {}
        }
    } else if (warp == 1) {
        const bool leader = elect_one();
        constexpr uint32_t idesc_s = make_idesc(kKTile, kQTile), idesc_o = make_idesc_major(kKTile, DH, false, true);
        bool ok = true;
        uint32_t fixed = 0;                                      // phases of the repair barriers
        // The walk of S^T and dP^T runs one job ahead of the walk of dV and dK, across items.
        KItem x;
        Job job;
        int r = -1, j = 0, n = -1, loaded = -1;
        bool more = true;
        auto advance = [&]() {
            ++n;
            if (r >= 0 && ++j < x.n) { job.next(x); return; }
            j = 0;
            for (;;) {
                const int at = item_at(++r);
                more = at < items;
                if (!more) return;
                x.load<SPLIT>(at, a, seqs);
                if (x.n > 0) break;
            }
            job.first(x, a.G);
            ++loaded;
        };
        auto product = [&](uint32_t dst, uint32_t A, uint32_t B) {       // [128 x DH] x [128 x DH]^T, both K-major
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) {
                const uint64_t da = umma_desc(A + hf * (kKTile * 128)), db = umma_desc(B + hf * (kQTile * 128));
#pragma unroll
                for (int k = 0; k < BK / UMMA_K; ++k) {
                    const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                    umma_ss(leader, dst, da + off, db + off, idesc_s, (hf > 0 || k > 0) ? 1u : 0u);
                }
            }
        };
        // acc += (operand of tile rows x 128 queries, at `src` in two halves of 64 queries) x (B tile [query][DH]), the products of
        // 16 queries from `k0` to `k1` of each half
        auto accumulate = [&](uint32_t acc, uint32_t src, uint32_t B, int k0, int k1, bool first) {
            const uint64_t db = umma_desc_mn(B, kQTile * 128);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k = k0; k < k1; ++k)
                    umma_ts(leader, tmem + acc, tmem + src + h * 64 + k * 8, db + static_cast<uint64_t>(((4 * h + k) * UMMA_K * 128) >> 4), idesc_o,
                            (!first || h > 0 || k > k0) ? 1u : 0u);
        };
        // Q or dO of job n is there (and repaired) and, from the second job on, the place of its product is free again.
        auto wait_tile = [&](uint32_t full, uint32_t repaired, uint32_t place) {
            const int st = n & 1;
            if (!ok) return;
            if (n > 0) ok = warp_wait2(full + 8 * st, (n >> 1) & 1, place + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, s_abort);
            else ok = warp_wait(full + 8 * st, 0, s_abort);
            if (ok && job.qb + kQTile > x.q_len) {
                const uint32_t bit = repaired == q_fixed ? st : 2 + st;
                ok = warp_wait(repaired + 8 * st, fixed >> bit & 1u, s_abort);
                fixed ^= 1u << bit;
            }
        };
        auto issue_s = [&]() {                                   // S^T = K Q^T
            if (j == 0) ok = warp_wait(kv_full, loaded & 1, s_abort);
            wait_tile(q_full, q_fixed, x_free);
            if (!ok) return;
            fence_after();
            product(tmem, sK, sQ + (n & 1) * 2 * SM::kT);
            commit_el(leader, s_full);
        };
        auto issue_dp = [&]() {                                  // dP^T = V dO^T
            wait_tile(do_full, do_fixed, y_free);
            if (!ok) return;
            fence_after();
            product(tmem + kY, sV, sQ + (n & 1) * 2 * SM::kT + SM::kT);
            commit_el(leader, dp_full);
            if (j + 1 == x.n) commit_el(leader, kv_empty);       // the item's last products with K and V
        };
        advance();
#pragma unroll 1
        for (int t = -1; ok; ++t) {                              // job t's dV and dK, job t + 1's S^T and dP^T; x is at job max(t, 0) here
            const int st = t & 1;
            const uint32_t Q = sQ + st * 2 * SM::kT;
            const bool first = j == 0;
            if (t >= 0) {
                if (!more) break;
                ok = warp_wait(p_full, t & 1, s_abort);          // (and, if this is a first job, the last item's dV and dK have been read)
                if (!ok) break;
                fence_after();
                accumulate(kDV, 0, Q + SM::kT, 0, 2, first);     // dV += P^T dO
                ok = warp_wait(p_full + 8, t & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDV, 0, Q + SM::kT, 2, 4, false);
                commit_el(leader, x_free + 8 * st);
                advance();
            }
            if (more) issue_s();
            if (t >= 0) {
                if (ok) ok = warp_wait(ds_full, t & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDK, kY, Q, 0, 4, first);             // dK += dS^T Q
                commit_el(leader, y_free + 8 * st);
            }
            if (more) issue_dp();
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;          // tensor-memory lane quarter; which 64 of the tile's queries
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16, at64 = lanes + 64 * half;
        const uint64_t scale2 = pk2(a.scale_log2, a.scale_log2);
        bool ok = true;
        int n = 0;
        for (int r = 0, at; (at = item_at(r)) < items; ++r) {
            KItem x;
            x.load<SPLIT>(at, a, seqs);
            const bool sink_part = x.seg >= 0;
            if (sink_part && x.n == 0) continue;                 // the join knows
            const int key = x.k0 + q * 32 + lane;
            const bool valid = key < x.kv_len, is_sink = key < a.sinks;
            // queries that see this key and belong to this item: [first, stop)
            const int first = sink_part ? x.band : key - x.shift;
            const int stop = !valid ? 0 : sink_part ? (is_sink ? x.q_len : 0) : is_sink ? x.band : min(x.q_len, key - x.shift + a.window);
            // every key of the tile is seen by queries [full_lo, full_hi)
            const int full_lo = sink_part ? x.band : min(x.k0 + kKTile, x.kv_len) - 1 - x.shift;
            const int full_hi = x.k0 + kKTile > x.kv_len ? 0 : x.k0 + kKTile <= a.sinks ? (sink_part ? x.q_len : x.band)
                                                           : sink_part ? 0 : min(x.q_len, x.k0 - x.shift + a.window);
            Job job;
            if (x.n > 0) job.first(x, a.G);
            for (int j = 0; j < x.n; ++j, ++n, job.next(x)) {
                const int st = n & 1, c0 = job.qb + 64 * half;   // first query of this thread's columns
                const float* stat = reinterpret_cast<const float*>(smem + kStatAt + st * 2 * SM::kStat) + 64 * half;      // -lse; -delta one kStat on
                if (ok) ok = warp_wait2(q_full + 8 * st, (n >> 1) & 1, s_full, n & 1, s_abort);      // (q_full: the statistics; their repair precedes S^T)
                if (!ok) continue;
                fence_after();
                const bool full = c0 >= full_lo && c0 + 64 <= full_hi;
                uint32_t s[2][32], d[32], y[16];
                tmem_ld32(tmem + at64, s[0]);
                tmem_ld32(tmem + at64 + 32, s[1]);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    // two columns' words as one 64-bit load, the same for every lane
                    auto nl = [&](int e) { return *reinterpret_cast<const uint64_t*>(stat + 32 * c + e); };
                    if (!full) mask32(s[c], bit_range(first - c0 - 32 * c, stop - c0 - 32 * c));
                    chunk_p(s[c], scale2, nl);
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = pack_bf16(__uint_as_float(s[c][2 * e]), __uint_as_float(s[c][2 * e + 1]));
                    tmem_st16(tmem + at64 + 16 * c, y);          // P^T of this half over its own S^T columns
                    tmem_st_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 8 * c);
                }
                ok = warp_wait(dp_full, n & 1, s_abort);
                if (!ok) continue;
                fence_after();
#pragma unroll
                for (int c = 0; c < 2; ++c) {                    // (a part at a time: registers are short)
                    auto nd = [&](int e) { return *reinterpret_cast<const uint64_t*>(stat + kQTile + 32 * c + e); };
                    tmem_ld32(tmem + kY + at64 + 32 * c, d);
                    tmem_ld_wait();
                    chunk_ds(s[c], d, nd, y);
                    tmem_st16(tmem + kY + at64 + 16 * c, y);     // dS^T over this half's dP^T columns that have been read
                }
                tmem_st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(ds_full); mbar_arrive(stat_empty + 8 * st); }
            }
            if (x.n > 0 && ok) ok = warp_wait2(y_free + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, x_free + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, s_abort);
            // The item is read again rather than held over the loop above, whose registers are short.
            asm volatile("" : "+r"(at));
            x.load<SPLIT>(at, a, seqs);
            fence_after();
            const float sv = ok ? 1.f : nan_f(), sk = ok ? a.scale : nan_f();
            const int my_key = x.k0 + q * 32 + lane;
            // rows that several items share go to the joins, in fp32
            const bool sink_item = x.seg >= 0, in_splits = SPLIT && !sink_item;
            const bool to_part = in_splits ? my_key < x.kv_len : seqs.segs[x.b] > 0 && my_key < min(a.sinks, x.kv_len);
            const size_t row = (size_t)(x.k_row + q * 32 + lane);
            const int col = half * (DH / 2);                     // this thread's half of the columns
            const bool write = my_key < x.kv_len && !sink_item && !to_part;
#pragma unroll 1
            for (int m = 0; m < 2; ++m) {                        // dV, dK
                const uint32_t acc = tmem + (m == 0 ? kDV : kDK) + col + lanes;
                const float f = m == 0 ? sv : sk;
                if (__any_sync(0xffffffffu, to_part)) {
                    float* part = in_splits ? a.split_part + (((size_t)key_unit(x.b, x.k0 / kKTile, x.kvh, a, seqs) * a.splits + x.split) * kKTile + (my_key - x.k0)) * 2 * DH
                                            : a.sink_part + sink_row(a, seqs, x.b, x.kvh, 1 + x.seg, my_key) * 2 * DH;
                    part += m * DH + col;
#pragma unroll 1
                    for (int c = 0; c < DH / 2; c += 16) {
                        uint32_t u[16];
                        if (x.n > 0) { tmem_ld16(acc + c, u); tmem_ld_wait(); }
                        if (to_part)
#pragma unroll
                            for (int i = 0; i < 16; i += 4)
                                *reinterpret_cast<float4*>(part + c + i) = x.n > 0 ? make_float4(__uint_as_float(u[i]) * f, __uint_as_float(u[i + 1]) * f, __uint_as_float(u[i + 2]) * f, __uint_as_float(u[i + 3]) * f)
                                                                                   : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                }
                if (__any_sync(0xffffffffu, write)) {
                    bf16* dst = m == 0 ? static_cast<bf16*>(a.dv) + row * a.dv_stride : static_cast<bf16*>(a.dk) + row * a.dk_stride;
                    store_rows<DH>(acc, f, x.n == 0, m == 0 ? &tmdV : &tmdK, smem + 6 * SM::kT + (warp - 2) * SM::kSlab, x.kvh * DH + col, x.k_row + q * 32,
                                   dst + x.kvh * DH + col, write, lane);
                }
            }
            fence_before();                                      // the accumulators have been read before the next item's P^T is announced
        }
    }
    if (lane == 0) store_done();                                 // this warp's last stores have read their slab
    fence_before();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        tmem_dealloc<kTmem>(tmem);
    }
}

// Adds the splits of a key tile, in order: to dV and dK, or (rows of sinks that segments share) to the band's place of the sinks'
// partials.  blockIdx = (sixteen rows of a tile, K/V head, tile of all sequences).
template <int DH>
__global__ void __launch_bounds__(256) window_split_join_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    constexpr int kVecs = 2 * DH / 4;                            // float4 of a row
    const int kvh = blockIdx.y;
    int b = 0, tile = blockIdx.z;
    for (int n; tile >= (n = (seqs.kv_len[b] + kKTile - 1) / kKTile); ++b) tile -= n;
    const int kv_len = seqs.kv_len[b];
    const float4* p = reinterpret_cast<const float4*>(a.split_part) + ((size_t)blockIdx.z * a.Hkv + kvh) * a.splits * kKTile * kVecs;
    for (int i = threadIdx.x; i < 16 * kVecs; i += 256) {
        const int r = blockIdx.x * 16 + i / kVecs, c = i % kVecs * 4, key = tile * kKTile + r;
        if (key >= kv_len) break;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < a.splits; ++s) {
            const float4 y = p[((size_t)s * kKTile + r) * kVecs + c / 4];
            x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        }
        if (seqs.segs[b] > 0 && key < a.sinks) {
            *reinterpret_cast<float4*>(a.sink_part + sink_row(a, seqs, b, kvh, 0, key) * 2 * DH + c) = x;
        } else {
            const size_t row = (size_t)(seqs.k_start[b] + key);
            bf16* dst = c < DH ? static_cast<bf16*>(a.dv) + row * a.dv_stride + c : static_cast<bf16*>(a.dk) + row * a.dk_stride + c - DH;
            *reinterpret_cast<uint2*>(dst + (size_t)kvh * DH) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
        }
    }
}

// Adds the band's and the segments' partials of the sink rows, in that order.  blockIdx = (sink row, K/V head, sequence).
template <int DH>
__global__ void __launch_bounds__(2 * DH) window_sink_join_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    const int key = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int segs = seqs.segs[b], rows = min(a.sinks, kv_len);
    if (segs == 0 || key >= rows) return;
    const int k0 = key / kKTile * kKTile;
    QueryWalk w;
    w.init(band_end(k0, kv_len, q_len, shift, a.window), q_len);
    const int total = w.n * a.G;
    const size_t step = (size_t)rows * 2 * DH;
    const float* p = a.sink_part + sink_row(a, seqs, b, kvh, 0, key) * 2 * DH + threadIdx.x;
    float x = *p;
    for (int s = 0; s < segs; ++s)
        if ((int)((long long)total * (s + 1) / segs) > (int)((long long)total * s / segs)) x += p[(1 + s) * step];
    const int c = threadIdx.x % DH;
    const size_t row = (size_t)(seqs.k_start[b] + key);
    bf16* dst = threadIdx.x < DH ? static_cast<bf16*>(a.dv) + row * a.dv_stride : static_cast<bf16*>(a.dk) + row * a.dk_stride;
    dst[(size_t)kvh * DH + c] = __float2bfloat16_rn(x);
}

template <int DH>
int launch_bwd(const WinArgs& a, const WinSeqs& s, long long q_rows, long long k_rows, cudaStream_t stream) {
    using SQ = BwdQSmem<DH>;
    using SK = BwdKSmem<DH>;
    const long long qc = (long long)a.Hq * DH, kc = (long long)a.Hkv * DH;
    // where one side has no rows its maps are never used, any valid one does
    const bool hq = q_rows > 0, hk = k_rows > 0;
    CUtensorMap mq, mdo, mk64, mv64, mk, mv, mdq, mdk, mdv;
    const void* any = hq ? a.q : a.k;
    const long long any_rows = hq ? q_rows : k_rows, any_cols = hq ? qc : kc, any_ld = hq ? a.q_stride : a.k_stride;
    if (!win_map(&mq, hq ? a.q : any, hq ? q_rows : any_rows, hq ? qc : any_cols, hq ? a.q_stride : any_ld, kQTile)) return -1;
    if (!win_map(&mdo, hq ? a.dout : any, hq ? q_rows : any_rows, hq ? qc : any_cols, hq ? a.dout_stride : any_ld, kQTile)) return -1;
    if (!win_map(&mk64, hk ? a.k : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.k_stride : any_ld, 64)) return -1;
    if (!win_map(&mv64, hk ? a.v : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.v_stride : any_ld, 64)) return -1;
    if (!win_map(&mk, hk ? a.k : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.k_stride : any_ld, kKTile)) return -1;
    if (!win_map(&mv, hk ? a.v : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.v_stride : any_ld, kKTile)) return -1;
    if (hq && !win_map(&mdq, a.dq, q_rows, qc, a.dq_stride, 32, DH / 2)) return -1;
    if (hk && (!win_map(&mdk, a.dk, k_rows, kc, a.dk_stride, 32, DH / 2) || !win_map(&mdv, a.dv, k_rows, kc, a.dv_stride, 32, DH / 2))) return -1;
    static PerDeviceOnce attr;
    if (!attr.ensure([] {
            return cudaFuncSetAttribute(window_bwd_q_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, SQ::kBytes) == cudaSuccess &&
                   cudaFuncSetAttribute(window_bwd_kv_kernel<DH, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SK::kBytes) == cudaSuccess &&
                   cudaFuncSetAttribute(window_bwd_kv_kernel<DH, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SK::kBytes) == cudaSuccess;
        }))
        return -1;
    const int sms = device_sm_count();
    int launched = 0;
    if (hq) {
        const long long items = (long long)s.item[a.batch] * a.Hq;
        if (items > 0x3fffffff) return -1;
        window_bwd_q_kernel<DH><<<(unsigned)(items < sms ? items : sms), kQThreads, SQ::kBytes, stream>>>(mq, mdo, mk64, mv64, mdq, a, s);
        ++launched;
    }
    if (hk) {
        WinSeqs t = s;                   // items of the key side: band tiles and sink segments
        t.item[0] = 0;
        int tiles = 0;
        for (int b = 0; b < a.batch; ++b) {
            const int n = (s.kv_len[b] + kKTile - 1) / kKTile, sinks = ((a.sinks < s.kv_len[b] ? a.sinks : s.kv_len[b]) + kKTile - 1) / kKTile;
            tiles += n;
            t.item[b + 1] = t.item[b] + n * a.splits + sinks * s.segs[b];
        }
        if (t.item[a.batch] > 0) {
            const long long items = (long long)t.item[a.batch] * a.Hkv;
            if (items > 0x3fffffff) return -1;
            // Items of many jobs run as CTAs of their own (their start-up is small beside them and the hardware balances them), short ones
            // share a pipeline.  Backward, head_dim 128, shared against unshared, us, by jobs of a band (whole tiles of the window + 256):
            //   one head a K/V head   6: 708 / 738   10: 854 / 899   18: 1420 / 1458   25: 1760 / 1772
            //   two                   8: 557 / 577   12: 649 / 631   16: 762 / 722     20: 871 / 822    24: 991 / 883
            //   four                  16: 580 / 561  20: 616 / 591   24: 694 / 622     40: 903 / 803    72: 1200 / 1202
            // (8 x 2048; 18 and 25: 4 x 4096; 72: two sequences up to 8191).  With grouped heads, whose items are fewer and longer, the
            // turn comes at ten jobs already: up to 7 % are left there between ten and 24.
            const long long jobs = ((long long)(a.window < 1 << 24 ? a.window : 1 << 24) + 2 * kKTile) / kQTile * a.G;
            const bool share = jobs < 24 && items > sms;
            (a.splits > 1 ? window_bwd_kv_kernel<DH, true> : window_bwd_kv_kernel<DH, false>)
                <<<(unsigned)(share ? sms : items), kThreads, SK::kBytes, stream>>>(mq, mdo, mk, mv, mdk, mdv, a, t);
            ++launched;
            if (a.splits > 1) {
                window_split_join_kernel<DH><<<dim3(kKTile / 16, a.Hkv, tiles), 256, 0, stream>>>(a, t);
                ++launched;
            }
            if (a.sink_rows > 0) {
                window_sink_join_kernel<DH><<<dim3(a.sink_rows, a.Hkv, a.batch), 2 * DH, 0, stream>>>(a, t);
                ++launched;
            }
        }
    }
    return launched;
}

}  // namespace

int window_bwd_bf16(const WinArgs& a, const WinSeqs& s, int dh, long long q_rows, long long k_rows, cudaStream_t stream) {
    return dh == 128 ? launch_bwd<128>(a, s, q_rows, k_rows, stream) : launch_bwd<64>(a, s, q_rows, k_rows, stream);
}

}  // namespace beagle
