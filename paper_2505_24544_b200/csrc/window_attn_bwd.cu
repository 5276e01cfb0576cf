// Backward of the windowed attention, bf16, head_dim 64 / 128 (tcgen05).
//
// With P = softmax over the visible keys (recomputed from the forward's log-sum-exp), dP = dO V^T, delta = rowsum(dO * O) and
// dS = P * (dP - delta):      dQ = dS K / sqrt(dh),   dK = dS^T Q / sqrt(dh),   dV = P^T dO.
//
// Two kernels and no atomics, so every sum has one order: a single kernel over keys would have to add dQ across CTAs, which costs
// either that order or an fp32 copy of dQ per key tile.  Recomputing S and dP costs 7 products instead of 5.
//   query side  one CTA = 128 queries of one (sequence, query head), 64 keys at a time:  S = Q K^T, dP = dO V^T -> dS in bf16
//               over S in tensor memory -> dQ += dS K.  256 tensor-memory columns and 112 KB: two CTAs share an SM, each one's
//               element-wise part runs under the other's products.  It also forms delta and leaves it, with the log-sum-exp,
//               side by side for the key side.
//   key side    one CTA = 128 keys of one (sequence, K/V head), 128 queries at a time for every query head of the group:
//               S^T = K Q^T -> P^T over S^T -> dV += P^T dO, and dP^T = V dO^T -> dS^T over dP^T -> dK += dS^T Q.  The two
//               halves take turns: while the threads form P of the next tile, dK and the next dP^T run, while they form dS,
//               dV and the next S^T run.
// P and dS are the tensor-memory operands of their products (rows = lanes), so the accumulating products read one operand
// from shared memory, and Q, dO, K tiles serve both as K-major and as MN-major operands: nothing is copied or transposed.
//
// The sinks' keys are read by every later query.  What lies past the band of a key tile is therefore cut into segments of
// similar length, each a CTA of its own that leaves fp32 partials of the (few) sink rows; a last small launch adds them to the
// band's partial in the order of the queries.
//
// Rows behind a sequence (the next one's) are zeroed in shared memory where they would be multiplied by a weight of 0.
// Every wait is bounded; a CTA that gives up leaves NaN in its rows.
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

// One thread's row of an accumulator (n columns from taddr), scaled, as bf16.
__device__ __forceinline__ void store_row32(uint32_t taddr, float scale, bf16* dst, bool write, bool zero) {
    uint32_t o[32];
    if (!zero) { tmem_ld32(taddr, o); tmem_ld_wait(); }
    if (!write) return;
#pragma unroll
    for (int x = 0; x < 32; x += 8) {
        uint32_t y[4];
#pragma unroll
        for (int z = 0; z < 4; ++z)
            y[z] = zero ? 0u : pack_bf16(__uint_as_float(o[x + 2 * z]) * scale, __uint_as_float(o[x + 2 * z + 1]) * scale);
        *reinterpret_cast<uint4*>(dst + x) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

// ---------------------------------------------------------------------------------------------------------------- query side
constexpr int kQThreads = 192;           // warp 0: TMA producer, warp 1: MMA issuer, warps 2-5: one thread per query
constexpr int kQCols = 64;               // keys of a tile

template <int DH>
struct BwdQSmem {
    static constexpr int kRes = kQTile * DH * 2;         // Q, and dO
    static constexpr int kT = kQCols * DH * 2;           // a K or V tile: two of K, one of V
    static constexpr int kBytes = 2 * kRes + 3 * kT + 256;
};

struct KeyWalk64 {
    int lo, hi, sink_end, n_sink, n;
    __device__ __forceinline__ void init(int q0, int q_len, int shift, int window, int sinks) {
        hi = min(q0 + kQTile, q_len) + shift;
        lo = max(0, q0 + shift - window + 1);
        sink_end = min(sinks, lo);
        n_sink = (sink_end + kQCols - 1) / kQCols;
        n = hi > 0 ? n_sink + (hi - lo + kQCols - 1) / kQCols : 0;
    }
    __device__ __forceinline__ void tile(int j, int& start, int& end) const {
        if (j < n_sink) { start = j * kQCols; end = min(start + kQCols, sink_end); }
        else { start = lo + (j - n_sink) * kQCols; end = min(start + kQCols, hi); }
    }
};

template <int DH>
__global__ void __launch_bounds__(kQThreads, 2) window_bwd_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                  const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                  const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    using SM = BwdQSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 256, kDP = 64, kDQ = 128;     // S / dS at column 0, dP at 64, dQ at 128
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sQ = smem_u32(smem), sdO = sQ + SM::kRes, sK = sdO + SM::kRes, sV = sK + 2 * SM::kT;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 2 * SM::kRes + 3 * SM::kT);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, k_full = bar0 + 8, k_empty = bar0 + 24, k_fixed = bar0 + 40, v_full = bar0 + 48, v_empty = bar0 + 56,
                   s_full = bar0 + 64, dp_full = bar0 + 72, ds_full = bar0 + 80, dq_done = bar0 + 88;
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 16);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 17);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int tile;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int q0 = ((q_len + kQTile - 1) / kQTile - 1 - tile) * kQTile;
    const int h = blockIdx.y, kvh = h / a.G;
    const int q_row = seqs.q_start[b] + q0, k_row = seqs.k_start[b];
    KeyWalk64 w;
    w.init(q0, q_len, shift, a.window, a.sinks);
    const int J = w.n;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(k_full + 8 * i, 1); mbar_init(k_empty + 8 * i, 1); }
        mbar_init(k_fixed, 1); mbar_init(v_full, 1); mbar_init(v_empty, 1);
        mbar_init(s_full, 1); mbar_init(dp_full, 1); mbar_init(ds_full, 4); mbar_init(dq_done, 1);
        *s_abort = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc<kTmem>(smem_u32(&s_tmem));
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;

    if (warp == 0) {
        if (J > 0) {
            if (lane == 0) {
                mbar_expect_tx(q_full, 2 * SM::kRes);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    tma_load_2d(sQ + hf * (kQTile * 128), &tmQ, q_full, h * DH + hf * 64, q_row);
                    tma_load_2d(sdO + hf * (kQTile * 128), &tmdO, q_full, h * DH + hf * 64, q_row);
                }
            }
            bool ok = true;
            int k_issued = 0, v_issued = 0;
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1;
                int start, end;
                w.tile(j, start, end);
                ok = __all_sync(0xffffffffu, mbar_wait(k_empty + 8 * st, ((j >> 1) & 1) ^ 1, s_abort));
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(k_full + 8 * st, SM::kT);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(sK + st * SM::kT + hf * (kQCols * 128), &tmK, k_full + 8 * st, kvh * DH + hf * 64, k_row + start);
                }
                __syncwarp();
                ++k_issued;
                const int cols = (end - start + 31) & ~31;
                if (start + cols > kv_len) {                     // rows behind the sequence: zero
                    ok = __all_sync(0xffffffffu, mbar_wait(k_full + 8 * st, (j >> 1) & 1, s_abort));
                    if (!ok) break;
                    zero_rows<DH>(smem + 2 * SM::kRes + st * SM::kT, kQCols, kv_len - start, cols, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(k_fixed);
                }
                ok = __all_sync(0xffffffffu, mbar_wait(v_empty, (j & 1) ^ 1, s_abort));
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(v_full, SM::kT);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(sV + hf * (kQCols * 128), &tmV, v_full, kvh * DH + hf * 64, k_row + start);
                }
                __syncwarp();
                ++v_issued;
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(q_full, 0); ++i) {}
                for (int n = max(0, k_issued - 2); n < k_issued; ++n)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(k_full + 8 * (n & 1), (n >> 1) & 1); ++i) {}
                for (uint32_t i = 0; v_issued > 0 && i < kSpinLimit && !mbar_try_wait(v_full, (v_issued - 1) & 1); ++i) {}
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && J > 0) {
            constexpr uint32_t idesc_q = make_idesc_major(kQTile, DH, false, true);
            bool ok = mbar_wait(q_full, 0, s_abort);
            int fixes = 0;
            auto cols_of = [&](int j, int& start) {
                int end;
                w.tile(j, start, end);
                return (end - start + 31) & ~31;
            };
            auto product = [&](uint32_t dst, uint32_t A, uint32_t B, int cols) {      // [128 x DH] x [cols x DH]^T, both K-major
                const uint32_t idesc = make_idesc(kQTile, cols);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    const uint64_t da = umma_desc(A + hf * (kQTile * 128)), db = umma_desc(B + hf * (kQCols * 128));
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k) {
                        const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                        umma_bf16(dst, da + off, db + off, idesc, (hf > 0 || k > 0) ? 1u : 0u);
                    }
                }
            };
            auto issue_s = [&](int j) {
                const int st = j & 1;
                int start;
                const int cols = cols_of(j, start);
                if (ok) ok = mbar_wait(k_full + 8 * st, (j >> 1) & 1, s_abort);
                if (ok && start + cols > kv_len) ok = mbar_wait(k_fixed, fixes++ & 1, s_abort);
                if (ok && j > 0) ok = mbar_wait(dq_done, (j - 1) & 1, s_abort);       // dS of the last tile lies where S goes now
                if (!ok) return;
                fence_after();
                product(tmem, sQ, sK + st * SM::kT, cols);
                umma_commit(s_full);
            };
            auto issue_dp = [&](int j) {
                int start;
                const int cols = cols_of(j, start);
                if (ok) ok = mbar_wait(v_full, j & 1, s_abort);
                if (!ok) return;
                fence_after();
                product(tmem + kDP, sdO, sV, cols);
                umma_commit(v_empty);
                umma_commit(dp_full);
            };
            issue_s(0);
            issue_dp(0);
            for (int j = 0; j < J && ok; ++j) {
                int start;
                const int cols = cols_of(j, start);
                ok = mbar_wait(ds_full, j & 1, s_abort);         // dS is written, dP has been read
                if (!ok) break;
                fence_after();
                const uint64_t dk = umma_desc_mn(sK + (j & 1) * SM::kT, kQCols * 128);
                for (int k = 0; k < cols / UMMA_K; ++k)
                    umma_bf16_ts(tmem + kDQ, tmem + 8 * k, dk + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_q, (j > 0 || k > 0) ? 1u : 0u);
                umma_commit(k_empty + 8 * (j & 1));
                umma_commit(dq_done);
                if (j + 1 < J) {
                    issue_dp(j + 1);
                    issue_s(j + 1);
                }
            }
        }
    } else {
        const int q = warp & 3;
        const int i = q0 + q * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const bool valid = i < q_len;
        const int last = i + shift, oldest = last - a.window + 1;
        const int full_lo = min(q0 + kQTile, q_len) - 1 + shift - a.window + 1, full_hi = q0 + shift + 1;
        // delta = dO . O of this query, and its log-sum-exp in log2 units
        float delta = 0.f, lse2 = 0.f;
        if (valid) {
            const size_t row = (size_t)(q_row + q * 32 + lane);
            const uint4* x = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.dout) + row * a.dout_stride + (size_t)h * DH);
            const uint4* y = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.out) + (row * a.Hq + h) * DH);
#pragma unroll 4
            for (int c = 0; c < DH / 8; ++c) {
                float f[8], g[8];
                unpack16<bf16>(__ldg(x + c), f);
                unpack16<bf16>(__ldg(y + c), g);
#pragma unroll
                for (int z = 0; z < 8; ++z) delta = fmaf(f[z], g[z], delta);
            }
            lse2 = __ldg(a.lse + row * a.Hq + h) * kLog2e;
            if (last < 0) { delta = 0.f; lse2 = 0.f; }           // a query that sees nothing
            a.stats[(size_t)h * a.stat_rows + stat_row0(seqs, b) + i] = make_float2(lse2, delta);
        }
        bool ok = true;
        for (int j = 0; j < J; ++j) {
            int start, end;
            w.tile(j, start, end);
            const int cols = (end - start + 31) & ~31;
            if (ok) ok = mbar_wait(s_full, j & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            uint32_t s[2][32], d[2][32];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (32 * c < cols) tmem_ld32(tmem + 32 * c + lanes, s[c]);
            tmem_ld_wait();
            const bool full = start + cols <= min(end, full_hi) && (start >= full_lo || end <= a.sinks);
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (32 * c < cols) {
                    const int k0 = start + 32 * c, top = valid ? min(last + 1, end) - k0 : 0;
                    const uint32_t vis = full ? 0xffffffffu : bit_range(oldest - k0, top) | bit_range(0, min(a.sinks - k0, top));
#pragma unroll
                    for (int x = 0; x < 32; ++x) {
                        const float p = exp2f(fmaf(__uint_as_float(s[c][x]), a.scale_log2, -lse2));
                        s[c][x] = (vis >> x & 1u) ? __float_as_uint(p) : 0u;
                    }
                }
            ok = mbar_wait(dp_full, j & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (32 * c < cols) tmem_ld32(tmem + kDP + 32 * c + lanes, d[c]);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (32 * c < cols) {
                    uint32_t y[16];
#pragma unroll
                    for (int x = 0; x < 32; x += 2) {
                        const float p0 = __uint_as_float(s[c][x]), p1 = __uint_as_float(s[c][x + 1]);
                        // a masked pair's dP may hold anything: its dS is 0, not 0 * dP
                        const float d0 = p0 == 0.f ? 0.f : p0 * (__uint_as_float(d[c][x]) - delta);
                        const float d1 = p1 == 0.f ? 0.f : p1 * (__uint_as_float(d[c][x + 1]) - delta);
                        y[x >> 1] = pack_bf16(d0, d1);
                    }
                    tmem_st16(tmem + 16 * c + lanes, y);
                }
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (J > 0) {
            if (ok) ok = mbar_wait(dq_done, (J - 1) & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
        }
        fence_after();
        bf16* dst = static_cast<bf16*>(a.dq) + (size_t)(q_row + q * 32 + lane) * a.dq_stride + (size_t)h * DH;
#pragma unroll
        for (int c = 0; c < DH; c += 32) store_row32(tmem + kDQ + c + lanes, ok ? a.scale : nan_f(), dst + c, valid, J == 0);
    }
    fence_before();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        tmem_dealloc<kTmem>(tmem);
    }
}

// ------------------------------------------------------------------------------------------------------------------ key side
constexpr int kKThreads = 320;           // warp 0: TMA producer, warp 1: MMA issuer, warps 2-9: two threads per key, 64 queries each

template <int DH>
struct BwdKSmem {
    static constexpr int kT = kKTile * DH * 2;           // K, V, and a tile of Q or dO (two stages)
    static constexpr int kStat = kQTile * 8;             // log-sum-exp and delta of a query tile (two stages)
    static constexpr int kBytes = 6 * kT + 2 * kStat + 256;
};

// The query tiles that a CTA of the key side reads: of every head of the group, from `from` in steps of 128 up to `to`.
struct QueryWalk {
    int from, to, n;                     // n tiles per head
    __device__ __forceinline__ void init(int f, int t) {
        from = max(f, 0) & ~1;           // (even: the statistics are copied in 16-byte pieces)
        to = t;
        n = to > from ? (to - from + kQTile - 1) / kQTile : 0;
    }
};
// First query past the band of the key tile at k0: none of its keys is inside the window of a later query.
__device__ __forceinline__ int band_end(int k0, int kv_len, int q_len, int shift, int window) {
    const int last_key = min(k0 + kKTile, kv_len) - 1;
    return max(0, min(q_len, last_key - shift + window));
}

// Items of the grid, per sequence: first its key tiles (band), then, for each of the sink_tiles, sink_segs segments.
template <int DH>
__global__ void __launch_bounds__(kKThreads, 1) window_bwd_kv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                   const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                   const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    using SM = BwdKSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 512, kY = 128, kDV = 256, kDK = 256 + DH;     // S^T / P^T at column 0, dP^T / dS^T at 128
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sK = smem_u32(smem), sV = sK + SM::kT, sQ = sV + SM::kT;      // stage s: Q at sQ + 2 s kT, dO behind it
    const uint32_t sStat = sQ + 4 * SM::kT;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 6 * SM::kT + 2 * SM::kStat);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t kv_full = bar0, qd_full = bar0 + 8, qd_empty = bar0 + 24, qd_fixed = bar0 + 40, s_full = bar0 + 48, p_full = bar0 + 56, x_free = bar0 + 64,
                   dp_full = bar0 + 72, ds_full = bar0 + 80, y_free = bar0 + 88, stat_empty = bar0 + 96;
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 20);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 21);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int item;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, item);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int kvh = blockIdx.y;
    const int tiles = (kv_len + kKTile - 1) / kKTile;
    const bool sink_part = item >= tiles;
    const int sink_tile = sink_part ? (item - tiles) / a.sink_segs : item;
    const int seg = sink_part ? (item - tiles) % a.sink_segs : -1;
    const int k0 = sink_tile * kKTile;
    QueryWalk w;
    int j0 = 0, J;
    {
        const int end = band_end(k0, kv_len, q_len, shift, a.window);
        if (!sink_part) {
            w.init(k0 - shift, end);
            J = w.n * a.G;
        } else {                                             // segment `seg` of the queries past the band, of all heads
            if (k0 >= min(a.sinks, kv_len)) return;          // (uniform over the CTA; nothing allocated yet)
            w.init(end, q_len);
            const int total = w.n * a.G;
            j0 = (int)((long long)total * seg / a.sink_segs);
            J = (int)((long long)total * (seg + 1) / a.sink_segs) - j0;
            if (J <= 0) return;                              // the join knows
        }
    }
    const int k_row = seqs.k_start[b] + k0;
    const int from_query = sink_part ? band_end(k0, kv_len, q_len, shift, a.window) : 0;
    auto job = [&](int j, int& h, int& qb) {                 // head and first query of job j
        const int x = j0 + j;
        h = kvh * a.G + x / w.n;
        qb = w.from + (x % w.n) * kQTile;
    };

    if (threadIdx.x == 0) {
        mbar_init(kv_full, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(qd_full + 8 * i, 1); mbar_init(qd_empty + 8 * i, 1); mbar_init(stat_empty + 8 * i, 8); }
        mbar_init(qd_fixed, 1);
        mbar_init(s_full, 1); mbar_init(p_full, 8); mbar_init(x_free, 1);
        mbar_init(dp_full, 1); mbar_init(ds_full, 8); mbar_init(y_free, 1);
        *s_abort = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc<kTmem>(smem_u32(&s_tmem));
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;

    if (warp == 0) {
        if (J > 0) {
            if (lane == 0) {
                mbar_expect_tx(kv_full, 2 * SM::kT);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    tma_load_2d(sK + hf * (kKTile * 128), &tmK, kv_full, kvh * DH + hf * 64, k_row);
                    tma_load_2d(sV + hf * (kKTile * 128), &tmV, kv_full, kvh * DH + hf * 64, k_row);
                }
            }
            const int stat0 = stat_row0(seqs, b);
            bool ok = true;
            int issued = 0;
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1;
                int h, qb;
                job(j, h, qb);
                ok = mbar_wait(qd_empty + 8 * st, ((j >> 1) & 1) ^ 1, s_abort);
                if (ok) ok = mbar_wait(stat_empty + 8 * st, ((j >> 1) & 1) ^ 1, s_abort);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = qd_full + 8 * st, dq = sQ + st * 2 * SM::kT;
                    mbar_expect_tx(bar, 2 * SM::kT + SM::kStat);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) {
                        tma_load_2d(dq + hf * (kQTile * 128), &tmQ, bar, h * DH + hf * 64, seqs.q_start[b] + qb);
                        tma_load_2d(dq + SM::kT + hf * (kQTile * 128), &tmdO, bar, h * DH + hf * 64, seqs.q_start[b] + qb);
                    }
                    bulk_load(sStat + st * SM::kStat, a.stats + (size_t)h * a.stat_rows + stat0 + qb, SM::kStat, bar);
                }
                __syncwarp();
                ++issued;
                if (qb + kQTile > q_len) {                       // rows behind the sequence: zero
                    ok = __all_sync(0xffffffffu, mbar_wait(qd_full + 8 * st, (j >> 1) & 1, s_abort));
                    if (!ok) break;
                    uint8_t* at = smem + 2 * SM::kT + st * 2 * SM::kT;
                    zero_rows<DH>(at, kQTile, q_len - qb, kQTile, lane);
                    zero_rows<DH>(at + SM::kT, kQTile, q_len - qb, kQTile, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(qd_fixed);
                }
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(kv_full, 0); ++i) {}
                for (int n = max(0, issued - 2); n < issued; ++n)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(qd_full + 8 * (n & 1), (n >> 1) & 1); ++i) {}
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && J > 0) {
            constexpr uint32_t idesc_s = make_idesc(kKTile, kQTile), idesc_o = make_idesc_major(kKTile, DH, false, true);
            bool ok = mbar_wait(kv_full, 0, s_abort);
            int fixes = 0;
            auto product = [&](uint32_t dst, uint32_t A, uint32_t B) {       // [128 x DH] x [128 x DH]^T, both K-major
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    const uint64_t da = umma_desc(A + hf * (kKTile * 128)), db = umma_desc(B + hf * (kQTile * 128));
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k) {
                        const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                        umma_bf16(dst, da + off, db + off, idesc_s, (hf > 0 || k > 0) ? 1u : 0u);
                    }
                }
            };
            // acc += (operand of tile rows x 128 queries, at `src` in two halves of 64 queries) x (B tile [query][DH])
            auto accumulate = [&](uint32_t acc, uint32_t src, uint32_t B, bool first) {
                const uint64_t db = umma_desc_mn(B, kQTile * 128);
#pragma unroll
                for (int k = 0; k < kQTile / UMMA_K; ++k)
                    umma_bf16_ts(tmem + acc, tmem + src + (k >> 2) * 64 + (k & 3) * 8, db + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_o,
                                 (!first || k > 0) ? 1u : 0u);
            };
            auto wait_tile = [&](int j) {                        // Q and dO of job j are there (and repaired)
                int h, qb;
                job(j, h, qb);
                if (ok) ok = mbar_wait(qd_full + 8 * (j & 1), (j >> 1) & 1, s_abort);
                if (ok && qb + kQTile > q_len) ok = mbar_wait(qd_fixed, fixes++ & 1, s_abort);
            };
            wait_tile(0);
            if (ok) {
                fence_after();
                product(tmem, sK, sQ);
                umma_commit(s_full);
                product(tmem + kY, sV, sQ + SM::kT);
                umma_commit(dp_full);
            }
            for (int j = 0; j < J && ok; ++j) {
                const uint32_t Q = sQ + (j & 1) * 2 * SM::kT, nextQ = sQ + ((j + 1) & 1) * 2 * SM::kT;
                ok = mbar_wait(p_full, j & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDV, 0, Q + SM::kT, j == 0);              // dV += P^T dO
                umma_commit(x_free);
                if (j + 1 < J) {
                    wait_tile(j + 1);
                    if (ok) ok = mbar_wait(x_free, j & 1, s_abort);  // P lies where the next S^T goes
                    if (!ok) break;
                    fence_after();
                    product(tmem, sK, nextQ);
                    umma_commit(s_full);
                }
                ok = mbar_wait(ds_full, j & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDK, kY, Q, j == 0);                      // dK += dS^T Q
                umma_commit(qd_empty + 8 * (j & 1));
                umma_commit(y_free);
                if (j + 1 < J) {
                    ok = mbar_wait(y_free, j & 1, s_abort);
                    if (!ok) break;
                    fence_after();
                    product(tmem + kY, sV, nextQ + SM::kT);
                    umma_commit(dp_full);
                }
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;          // tensor-memory lane quarter; which 64 of the tile's queries
        const int key = k0 + q * 32 + lane;
        const uint32_t at = (static_cast<uint32_t>(q * 32) << 16) + 64 * half;
        const bool valid = key < kv_len;
        const bool is_sink = key < a.sinks;
        // queries that see this key: [first, stop)
        const int first = max(key - shift, from_query);
        const int stop = !valid ? 0 : is_sink ? q_len : sink_part ? 0 : min(q_len, key - shift + a.window);
        const int stop_band = sink_part ? q_len : band_end(k0, kv_len, q_len, shift, a.window);      // a band CTA leaves the rest to the segments
        const int stop_all = min(stop, stop_band);
        // every key of the tile is seen by queries [full_lo, full_hi)
        const int full_lo = max(min(k0 + kKTile, kv_len) - 1 - shift, from_query);
        const int full_hi = k0 + kKTile > kv_len ? 0 : k0 + kKTile <= a.sinks ? stop_band : sink_part ? 0 : min(q_len, k0 - shift + a.window);
        bool ok = true;
        for (int j = 0; j < J; ++j) {
            int h, qb;
            job(j, h, qb);
            const int st = j & 1, c0 = qb + 64 * half;           // first query of this thread's columns
            const float4* stat = reinterpret_cast<const float4*>(smem + 6 * SM::kT + st * SM::kStat + 64 * half * 8);     // (lse, delta) pairs
            if (ok) ok = mbar_wait(qd_full + 8 * st, (j >> 1) & 1, s_abort);     // the statistics
            if (ok) ok = mbar_wait(s_full, j & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            const bool full = c0 >= full_lo && c0 + 64 <= full_hi;
            uint32_t s[2][32], d[32];
            tmem_ld32(tmem + at, s[0]);
            tmem_ld32(tmem + at + 32, s[1]);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t vis = full ? 0xffffffffu : bit_range(first - c0 - 32 * c, stop_all - c0 - 32 * c);
                uint32_t y[16];
#pragma unroll
                for (int x = 0; x < 32; x += 2) {
                    const float4 t = stat[16 * c + (x >> 1)];    // two queries' (lse, delta), the same words for every lane
                    float p0 = exp2f(fmaf(__uint_as_float(s[c][x]), a.scale_log2, -t.x));
                    float p1 = exp2f(fmaf(__uint_as_float(s[c][x + 1]), a.scale_log2, -t.z));
                    if (!full) {
                        p0 = (vis >> x & 1u) ? p0 : 0.f;
                        p1 = (vis >> (x + 1) & 1u) ? p1 : 0.f;
                    }
                    s[c][x] = __float_as_uint(p0);
                    s[c][x + 1] = __float_as_uint(p1);
                    y[x >> 1] = pack_bf16(p0, p1);
                }
                tmem_st16(tmem + at + 16 * c, y);                // P^T of this half over its own S^T columns
            }
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full);

            ok = mbar_wait(dp_full, j & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            uint32_t z[2][16];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                tmem_ld32(tmem + kY + at + 32 * c, d);
                tmem_ld_wait();
#pragma unroll
                for (int x = 0; x < 32; x += 2) {
                    const float4 t = stat[16 * c + (x >> 1)];
                    const float p0 = __uint_as_float(s[c][x]), p1 = __uint_as_float(s[c][x + 1]);
                    float d0 = p0 * (__uint_as_float(d[x]) - t.y), d1 = p1 * (__uint_as_float(d[x + 1]) - t.w);
                    if (!full) {                                 // a masked pair's dP and delta may hold anything
                        d0 = p0 == 0.f ? 0.f : d0;
                        d1 = p1 == 0.f ? 0.f : d1;
                    }
                    z[c][x >> 1] = pack_bf16(d0, d1);
                }
            }
            tmem_st16(tmem + kY + at, z[0]);                     // dS^T over this half's own dP^T columns, which are in registers
            tmem_st16(tmem + kY + at + 16, z[1]);
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) { mbar_arrive(ds_full); mbar_arrive(stat_empty + 8 * st); }
        }
        if (J > 0) {
            if (ok) ok = mbar_wait(y_free, (J - 1) & 1, s_abort);
            if (ok) ok = mbar_wait(x_free, (J - 1) & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
        }
        fence_after();
        const float sv = ok ? 1.f : nan_f(), sk = ok ? a.scale : nan_f();
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const bool to_part = a.sink_segs > 0 && is_sink && valid;        // rows that several CTAs share go to the join, in fp32
        // every thread reads its half of the columns; a warp may hold rows of both kinds
        const size_t row = (size_t)(k_row + q * 32 + lane);
        bf16* dk = static_cast<bf16*>(a.dk) + row * a.dk_stride + (size_t)kvh * DH;
        bf16* dv = static_cast<bf16*>(a.dv) + row * a.dv_stride + (size_t)kvh * DH;
        float* part = nullptr;
        if (to_part)
            part = a.sink_part + ((((size_t)b * a.Hkv + kvh) * (1 + a.sink_segs) + (sink_part ? 1 + seg : 0)) * a.sink_rows + key) * 2 * DH;
#pragma unroll
        for (int c = 0; c < DH / 2; c += 32) {
            const int col = half * (DH / 2) + c;
            uint32_t x[32], y[32];
            if (J > 0) { tmem_ld32(tmem + kDV + col + lanes, x); tmem_ld32(tmem + kDK + col + lanes, y); tmem_ld_wait(); }
            else {
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = y[i] = 0u;
            }
            if (to_part) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    *reinterpret_cast<float4*>(part + col + i) = make_float4(__uint_as_float(x[i]) * sv, __uint_as_float(x[i + 1]) * sv, __uint_as_float(x[i + 2]) * sv, __uint_as_float(x[i + 3]) * sv);
                    *reinterpret_cast<float4*>(part + DH + col + i) = make_float4(__uint_as_float(y[i]) * sk, __uint_as_float(y[i + 1]) * sk, __uint_as_float(y[i + 2]) * sk, __uint_as_float(y[i + 3]) * sk);
                }
            } else if (valid && !sink_part) {
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    uint32_t u[4], v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        u[e] = pack_bf16(__uint_as_float(x[i + 2 * e]) * sv, __uint_as_float(x[i + 2 * e + 1]) * sv);
                        v[e] = pack_bf16(__uint_as_float(y[i + 2 * e]) * sk, __uint_as_float(y[i + 2 * e + 1]) * sk);
                    }
                    *reinterpret_cast<uint4*>(dv + col + i) = make_uint4(u[0], u[1], u[2], u[3]);
                    *reinterpret_cast<uint4*>(dk + col + i) = make_uint4(v[0], v[1], v[2], v[3]);
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        tmem_dealloc<kTmem>(tmem);
    }
}

// Adds the band's and the segments' partials of the sink rows, in that order.  blockIdx = (sink row, K/V head, sequence).
template <int DH>
__global__ void __launch_bounds__(2 * DH) window_sink_join_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    const int key = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    if (key >= kv_len) return;
    const int k0 = key / kKTile * kKTile;
    QueryWalk w;
    w.init(band_end(k0, kv_len, q_len, shift, a.window), q_len);
    const int total = w.n * a.G;
    const size_t step = (size_t)a.sink_rows * 2 * DH;
    const float* p = a.sink_part + (((size_t)b * a.Hkv + kvh) * (1 + a.sink_segs) * a.sink_rows + key) * 2 * DH + threadIdx.x;
    float x = *p;
    for (int s = 0; s < a.sink_segs; ++s)
        if ((int)((long long)total * (s + 1) / a.sink_segs) > (int)((long long)total * s / a.sink_segs)) x += p[(1 + s) * step];
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
    CUtensorMap mq, mdo, mk64, mv64, mk, mv;
    const void* any = hq ? a.q : a.k;
    const long long any_rows = hq ? q_rows : k_rows, any_cols = hq ? qc : kc, any_ld = hq ? a.q_stride : a.k_stride;
    if (!win_map(&mq, hq ? a.q : any, hq ? q_rows : any_rows, hq ? qc : any_cols, hq ? a.q_stride : any_ld, kQTile)) return -1;
    if (!win_map(&mdo, hq ? a.dout : any, hq ? q_rows : any_rows, hq ? qc : any_cols, hq ? a.dout_stride : any_ld, kQTile)) return -1;
    if (!win_map(&mk64, hk ? a.k : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.k_stride : any_ld, kQCols)) return -1;
    if (!win_map(&mv64, hk ? a.v : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.v_stride : any_ld, kQCols)) return -1;
    if (!win_map(&mk, hk ? a.k : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.k_stride : any_ld, kKTile)) return -1;
    if (!win_map(&mv, hk ? a.v : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.v_stride : any_ld, kKTile)) return -1;
    static PerDeviceOnce attr;
    if (!attr.ensure([] {
            return cudaFuncSetAttribute(window_bwd_q_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, SQ::kBytes) == cudaSuccess &&
                   cudaFuncSetAttribute(window_bwd_kv_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, SK::kBytes) == cudaSuccess;
        }))
        return -1;
    int launched = 0;
    if (hq) {
        window_bwd_q_kernel<DH><<<dim3(s.item[a.batch], a.Hq), kQThreads, SQ::kBytes, stream>>>(mq, mdo, mk64, mv64, a, s);
        ++launched;
    }
    if (hk) {
        WinSeqs t = s;                   // items of the key side: band tiles and sink segments
        t.item[0] = 0;
        for (int b = 0; b < a.batch; ++b) t.item[b + 1] = t.item[b] + (s.kv_len[b] + kKTile - 1) / kKTile + a.sink_tiles * a.sink_segs;
        if (t.item[a.batch] > 0) {
            window_bwd_kv_kernel<DH><<<dim3(t.item[a.batch], a.Hkv), kKThreads, SK::kBytes, stream>>>(mq, mdo, mk, mv, a, t);
            ++launched;
            if (a.sink_segs > 0) {
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
