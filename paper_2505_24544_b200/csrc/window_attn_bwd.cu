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
// Both use all 512 columns of tensor memory and about 200 KB of shared memory (one CTA per SM, two threads per tile row).
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
constexpr int kPoly = 3;                 // of every eight pairs of exponentials, those on the multiply-add pipe


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

// 32 columns of a tile: P = exp2(S * scale - lse), kept as fp32 in r (masked: 0 where `vis` has no bit).  nl(x) gives the negated
// log-sum-exp of columns x, x + 1.
template <bool MASK, typename NegLse>
__device__ __forceinline__ void chunk_p(uint32_t* r, uint32_t vis, uint64_t scale2, NegLse nl) {
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
        float e0, e1;
        const uint64_t z = fma2(pk2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), scale2, nl(x));
        if (!MASK && poly_pair<kPoly>(x)) {
            exp2_poly2(z, e0, e1);
        } else {
            un2(z, e0, e1);
            e0 = exp2f(e0);
            e1 = exp2f(e1);
        }
        if (MASK) {
            e0 = (vis >> x & 1u) ? e0 : 0.f;
            e1 = (vis >> (x + 1) & 1u) ? e1 : 0.f;
        }
        r[x] = __float_as_uint(e0);
        r[x + 1] = __float_as_uint(e1);
    }
}
// dS = P * (dP - delta) of 32 columns as bf16 pairs; a masked pair's dP and delta may hold anything: its dS is 0.
template <bool MASK, typename NegDelta>
__device__ __forceinline__ void chunk_ds(const uint32_t* p, const uint32_t* d, NegDelta nd, uint32_t* y) {
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
        const float p0 = __uint_as_float(p[x]), p1 = __uint_as_float(p[x + 1]);
        float d0, d1;
        un2(mul2(pk2(p0, p1), add2(pk2(__uint_as_float(d[x]), __uint_as_float(d[x + 1])), nd(x))), d0, d1);
        if (MASK) {
            d0 = p0 == 0.f ? 0.f : d0;
            d1 = p1 == 0.f ? 0.f : d1;
        }
        y[x >> 1] = pack_bf16(d0, d1);
    }
}

// ---------------------------------------------------------------------------------------------------------------- query side
constexpr int kThreads = 320;            // warp 0: TMA producer, warp 1: MMA issuer, warps 2-9: two threads per tile row, 64 columns each

template <int DH>
struct BwdQSmem {
    static constexpr int kT = kQTile * DH * 2;           // Q, dO, and a K or V tile (two stages of each)
    static constexpr int kBytes = 6 * kT + 2 * kQTile * 4 + 256;
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

template <int DH>
__global__ void __launch_bounds__(kThreads, 1) window_bwd_q_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                 const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                 const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    using SM = BwdQSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 512, kDP = 256, kDQ = 384;    // S / dS at columns 0 and 128, dP at 256, dQ at 384
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sQ = smem_u32(smem), sdO = sQ + SM::kT, sKV = sdO + SM::kT;       // stage s: K at sKV + 2 s kT, V behind it
    float* s_delta = reinterpret_cast<float*>(smem + 6 * SM::kT);                    // [2][128]: the two halves of dO . O
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 6 * SM::kT + 2 * kQTile * 4);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, dp_full = bar0 + 8, ds_full = bar0 + 16, dq_done = bar0 + 24, k_full = bar0 + 32, k_empty = bar0 + 48, k_fixed = bar0 + 64,
                   s_full = bar0 + 80, v_full = bar0 + 96, v_empty = bar0 + 112;         // the last six: one per stage
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 20);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 21);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    int tile;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int q0 = ((q_len + kQTile - 1) / kQTile - 1 - tile) * kQTile;
    const int h = blockIdx.y, kvh = h / a.G;
    const int q_row = seqs.q_start[b] + q0, k_row = seqs.k_start[b];
    KeyWalk w;
    w.init(q0, q_len, shift, a.window, a.sinks);
    const int J = w.n;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1); mbar_init(dp_full, 1); mbar_init(ds_full, 8); mbar_init(dq_done, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, 1); mbar_init(k_empty + 8 * i, 1); mbar_init(k_fixed + 8 * i, 1);
            mbar_init(v_full + 8 * i, 1); mbar_init(v_empty + 8 * i, 1); mbar_init(s_full + 8 * i, 1);
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
        if (J > 0) {
            if (lane == 0) {
                mbar_expect_tx(q_full, 2 * SM::kT);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    tma_load_2d(sQ + hf * (kQTile * 128), &tmQ, q_full, h * DH + hf * 64, q_row);
                    tma_load_2d(sdO + hf * (kQTile * 128), &tmdO, q_full, h * DH + hf * 64, q_row);
                }
            }
            bool ok = true;
            int issued = 0;
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1, ph = (j >> 1) & 1;
                int start, end;
                w.tile(j, start, end);
                const int boxes = (end - start + 63) / 64;       // of 64 keys
                auto load = [&](const CUtensorMap* tm, uint32_t at, uint32_t bar) {
                    if (lane == 0) {
                        mbar_expect_tx(bar, boxes * kHalves * 64 * 128);
                        for (int x = 0; x < boxes; ++x)
#pragma unroll
                            for (int hf = 0; hf < kHalves; ++hf)
                                tma_load_2d(at + hf * (kKTile * 128) + x * (64 * 128), tm, bar, kvh * DH + hf * 64, k_row + start + 64 * x);
                    }
                    __syncwarp();
                };
                ok = warp_wait(v_empty + 8 * st, ph ^ 1, s_abort);      // (free before the K tile of the same stage)
                if (!ok) break;
                load(&tmV, sKV + (2 * st + 1) * SM::kT, v_full + 8 * st);
                ++issued;
                ok = warp_wait(k_empty + 8 * st, ph ^ 1, s_abort);
                if (!ok) break;
                load(&tmK, sKV + 2 * st * SM::kT, k_full + 8 * st);
                ++issued;
                const int cols = (end - start + 31) & ~31;
                if (start + cols > kv_len) {                     // rows of K behind the sequence: zero
                    ok = warp_wait(k_full + 8 * st, ph, s_abort);
                    if (!ok) break;
                    zero_rows<DH>(smem + (2 + 2 * st) * SM::kT, kKTile, kv_len - start, cols, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(k_fixed + 8 * st);
                }
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(q_full, 0); ++i) {}
                for (int n = max(0, issued - 4); n < issued; ++n)        // copy n: V of tile n / 2 if even, K if odd
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait((n & 1 ? k_full : v_full) + 8 * ((n >> 1) & 1), (n >> 2) & 1); ++i) {}
            }
        }
    } else if (warp == 1) {
        if (J > 0) {
            const bool leader = elect_one();
            constexpr uint32_t idesc_q = make_idesc_major(kQTile, DH, false, true);
            bool ok = warp_wait(q_full, 0, s_abort);
            uint32_t fixed = 0;                                  // phase of every stage's repair barrier
            auto cols_of = [&](int j, int& start) {
                int end;
                w.tile(j, start, end);
                return (end - start + 31) & ~31;
            };
            auto product = [&](uint32_t dst, uint32_t A, uint32_t B, int cols) {      // [128 x DH] x [cols x DH]^T, both K-major
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
            auto issue_s = [&](int j) {
                const int st = j & 1;
                int start;
                const int cols = cols_of(j, start);
                if (ok) ok = warp_wait(k_full + 8 * st, (j >> 1) & 1, s_abort);
                if (ok && start + cols > kv_len) { ok = warp_wait(k_fixed + 8 * st, fixed >> st & 1u, s_abort); fixed ^= 1u << st; }
                if (!ok) return;                                 // (dS of tile j - 2 has been read: k_full follows k_empty)
                fence_after();
                product(tmem + 128 * st, sQ, sKV + st * 2 * SM::kT, cols);
                commit_el(leader, s_full + 8 * st);
            };
            auto issue_dp = [&](int j) {
                int start;
                const int cols = cols_of(j, start);
                if (ok) ok = warp_wait(v_full + 8 * (j & 1), (j >> 1) & 1, s_abort);
                if (!ok) return;
                fence_after();
                product(tmem + kDP, sdO, sKV + (j & 1) * 2 * SM::kT + SM::kT, cols);
                commit_el(leader, v_empty + 8 * (j & 1));
                commit_el(leader, dp_full);
            };
            issue_s(0);
            issue_dp(0);
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1;
                if (j + 1 < J) issue_s(j + 1);
                if (ok) ok = warp_wait(ds_full, j & 1, s_abort);         // dS is written, dP has been read
                if (!ok) break;
                fence_after();
                int start;
                const int cols = cols_of(j, start);
                const uint64_t dk = umma_desc_mn(sKV + st * 2 * SM::kT, kKTile * 128);
                for (int k = 0; k < cols / UMMA_K; ++k)
                    umma_ts(leader, tmem + kDQ, tmem + 128 * st + (k >> 2) * 64 + (k & 3) * 8, dk + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_q,
                                 (j > 0 || k > 0) ? 1u : 0u);
                commit_el(leader, k_empty + 8 * st);
                if (j + 1 == J) commit_el(leader, dq_done);
                else issue_dp(j + 1);
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;          // tensor-memory lane quarter; which 64 columns of a tile
        const int row = q * 32 + lane, i = q0 + row;
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const bool valid = i < q_len;
        const int last = i + shift, oldest = last - a.window + 1;
        const int full_lo = min(q0 + kQTile, q_len) - 1 + shift - a.window + 1, full_hi = q0 + shift + 1;
        // delta = dO . O of this query (each thread of the row half of it), and its log-sum-exp in log2 units
        float delta = 0.f, lse2 = 0.f;
        if (valid) {
            const size_t at = (size_t)(q_row + row);
            const uint4* x = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.dout) + at * a.dout_stride + (size_t)h * DH + half * (DH / 2));
            const uint4* y = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.out) + (at * a.Hq + h) * DH + half * (DH / 2));
#pragma unroll
            for (int c = 0; c < DH / 16; ++c) {
                float f[8], g[8];
                unpack16<bf16>(__ldg(x + c), f);
                unpack16<bf16>(__ldg(y + c), g);
#pragma unroll
                for (int z = 0; z < 8; ++z) delta = fmaf(f[z], g[z], delta);
            }
            lse2 = __ldg(a.lse + at * a.Hq + h) * kLog2e;
        }
        s_delta[half * kQTile + row] = delta;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        delta = s_delta[row] + s_delta[kQTile + row];
        if (last < 0) { delta = 0.f; lse2 = 0.f; }               // a query that sees nothing
        if (valid) {                                             // for the key side: -lse and -delta, each in a row of its own
            float* stat = a.stats + (size_t)h * 2 * a.stat_rows + stat_row0(seqs, b) + i;
            if (half == 0) stat[0] = -lse2;
            else stat[a.stat_rows] = -delta;
        }
        const uint64_t scale2 = pk2(a.scale_log2, a.scale_log2), nl2 = pk2(-lse2, -lse2), nd2 = pk2(-delta, -delta);
        auto nl = [&](int) { return nl2; };
        auto nd = [&](int) { return nd2; };
        bool ok = true;
        for (int j = 0; j < J; ++j) {
            const int st = j & 1;
            int start, end;
            w.tile(j, start, end);
            start += 64 * half;                                  // this thread's columns
            const bool one = start < end, two = start + 32 < end;
            const bool full = start + 64 <= min(end, full_hi) && (start >= full_lo || start + 64 <= a.sinks);
            if (ok) ok = warp_wait(s_full + 8 * st, (j >> 1) & 1, s_abort);
            if (!ok) break;
            fence_after();
            const uint32_t ts = tmem + 128 * st + 64 * half + lanes;
            uint32_t s[2][32], d[2][32], y[2][16];
            if (one) {
                tmem_ld32(ts, s[0]);
                if (two) tmem_ld32(ts + 32, s[1]);
                tmem_ld_wait();
                if (full) {
                    chunk_p<false>(s[0], 0u, scale2, nl);
                    chunk_p<false>(s[1], 0u, scale2, nl);
                } else {
                    const int top = valid ? min(last + 1, end) - start : 0;
                    chunk_p<true>(s[0], bit_range(oldest - start, top) | bit_range(0, min(a.sinks - start, top)), scale2, nl);
                    if (two) chunk_p<true>(s[1], bit_range(oldest - start - 32, top - 32) | bit_range(0, min(a.sinks - start, top) - 32), scale2, nl);
                }
            }
            ok = warp_wait(dp_full, j & 1, s_abort);
            if (!ok) break;
            fence_after();
            if (one) {
                tmem_ld32(tmem + kDP + 64 * half + lanes, d[0]);
                if (two) tmem_ld32(tmem + kDP + 64 * half + 32 + lanes, d[1]);
                tmem_ld_wait();
                if (full) {
                    chunk_ds<false>(s[0], d[0], nd, y[0]);
                    chunk_ds<false>(s[1], d[1], nd, y[1]);
                } else {
                    chunk_ds<true>(s[0], d[0], nd, y[0]);
                    if (two) chunk_ds<true>(s[1], d[1], nd, y[1]);
                }
                tmem_st16(ts, y[0]);                             // dS of this half over its own S columns
                if (two) tmem_st16(ts + 16, y[1]);
                tmem_st_wait();
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (J > 0) {
            if (ok) ok = warp_wait(dq_done, 0, s_abort);
        }
        fence_after();
        bf16* dst = static_cast<bf16*>(a.dq) + (size_t)(q_row + row) * a.dq_stride + (size_t)h * DH;
#pragma unroll
        for (int c = 0; c < DH / 2; c += 32) {
            const int col = half * (DH / 2) + c;
            store_row32(tmem + kDQ + col + lanes, ok ? a.scale : nan_f(), dst + col, valid, J == 0);
        }
    }
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
    static constexpr int kBytes = 6 * kT + 4 * kStat + 256;
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

// Items of the grid, per sequence: first its key tiles (band), then, for each of the sink_tiles, sink_segs segments.
template <int DH>
__global__ void __launch_bounds__(kThreads, 1) window_bwd_kv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmdO,
                                                                   const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                   const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    using SM = BwdKSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 512, kY = 128, kDV = 256, kDK = 256 + DH;     // S^T / P^T at column 0, dP^T / dS^T at 128
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sK = smem_u32(smem), sV = sK + SM::kT, sQ = sV + SM::kT;      // stage s: Q at sQ + 2 s kT, dO behind it
    const uint32_t sStat = sQ + 4 * SM::kT;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + 6 * SM::kT + 4 * SM::kStat);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t kv_full = bar0, s_full = bar0 + 8, dp_full = bar0 + 16, ds_full = bar0 + 24;
    // one per stage; Q is free when dK has read it (so is dS^T's place), dO when dV has (so is P^T's place)
    const uint32_t p_full = bar0 + 152;                  // P^T in two parts: the first 32 queries of each half of the tile, then the others
    const uint32_t q_full = bar0 + 40, do_full = bar0 + 56, y_free = bar0 + 72, x_free = bar0 + 88, stat_empty = bar0 + 104, q_fixed = bar0 + 120,
                   do_fixed = bar0 + 136;
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 24);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 25);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
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
    // Jobs in order: the tiles of one head after the other.
    struct Job {
        int h, qb, left;                 // query head, first query, tiles left of this head
    } const job0 = {kvh * a.G + (w.n > 0 ? j0 / w.n : 0), w.from + (w.n > 0 ? j0 % w.n : 0) * kQTile, w.n - (w.n > 0 ? j0 % w.n : 0)};
    auto next_job = [&](Job& x) {
        x.qb += kQTile;
        if (--x.left == 0) { ++x.h; x.qb = w.from; x.left = w.n; }
    };

    if (threadIdx.x == 0) {
        mbar_init(kv_full, 1); mbar_init(s_full, 1); mbar_init(p_full, 8); mbar_init(p_full + 8, 8); mbar_init(dp_full, 1); mbar_init(ds_full, 8);
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
            Job job = job0;
            for (int j = 0; j < J && ok; ++j, next_job(job)) {
                const int st = j & 1, ph = (j >> 1) & 1, h = job.h, qb = job.qb;
                const uint32_t at = sQ + st * 2 * SM::kT;
                uint8_t* tile = smem + (2 + 2 * st) * SM::kT;
                const bool edge = qb + kQTile > q_len;           // rows behind the sequence: zero
                auto repair = [&](uint32_t full, uint32_t fixed, uint8_t* t) {
                    ok = warp_wait(full, ph, s_abort);
                    if (!ok) return;
                    zero_rows<DH>(t, kQTile, q_len - qb, kQTile, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(fixed);
                };
                ok = warp_wait(x_free + 8 * st, ph ^ 1, s_abort);        // dO is needed last and free first
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(do_full + 8 * st, SM::kT);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
                        tma_load_2d(at + SM::kT + hf * (kQTile * 128), &tmdO, do_full + 8 * st, h * DH + hf * 64, seqs.q_start[b] + qb);
                }
                __syncwarp();
                ++issued;
                ok = warp_wait(y_free + 8 * st, ph ^ 1, s_abort);
                if (ok) ok = warp_wait(stat_empty + 8 * st, ph ^ 1, s_abort);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(q_full + 8 * st, SM::kT + 2 * SM::kStat);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(at + hf * (kQTile * 128), &tmQ, q_full + 8 * st, h * DH + hf * 64, seqs.q_start[b] + qb);
                    const float* stat = a.stats + (size_t)h * 2 * a.stat_rows + stat0 + qb;
                    bulk_load(sStat + st * 2 * SM::kStat, stat, SM::kStat, q_full + 8 * st);
                    bulk_load(sStat + st * 2 * SM::kStat + SM::kStat, stat + a.stat_rows, SM::kStat, q_full + 8 * st);
                }
                __syncwarp();
                ++issued;
                if (edge) {
                    repair(q_full + 8 * st, q_fixed + 8 * st, tile);
                    if (ok) repair(do_full + 8 * st, do_fixed + 8 * st, tile + SM::kT);
                }
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(kv_full, 0); ++i) {}
                for (int n = max(0, issued - 4); n < issued; ++n)        // copy n: dO of tile n / 2 if even, Q if odd
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait((n & 1 ? q_full : do_full) + 8 * ((n >> 1) & 1), (n >> 2) & 1); ++i) {}
            }
        }
    } else if (warp == 1) {
        if (J > 0) {
            const bool leader = elect_one();
            constexpr uint32_t idesc_s = make_idesc(kKTile, kQTile), idesc_o = make_idesc_major(kKTile, DH, false, true);
            bool ok = warp_wait(kv_full, 0, s_abort);
            uint32_t fixed = 0;                                  // phase of every stage's repair barrier
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
            Job job = job0;                                      // of the next S^T (and, right after it, the next dP^T)
            auto wait_tile = [&](int j, uint32_t full, uint32_t repaired, int qb) {      // Q or dO of job j is there (and repaired)
                const int st = j & 1;
                if (ok) ok = warp_wait(full + 8 * st, (j >> 1) & 1, s_abort);
                if (ok && qb + kQTile > q_len) {
                    const uint32_t bit = repaired == q_fixed ? st : 2 + st;
                    ok = warp_wait(repaired + 8 * st, fixed >> bit & 1u, s_abort);
                    fixed ^= 1u << bit;
                }
            };
            auto issue_s = [&](int j) {                          // S^T = K Q^T
                wait_tile(j, q_full, q_fixed, job.qb);
                if (ok && j > 0) ok = warp_wait(x_free + 8 * ((j - 1) & 1), ((j - 1) >> 1) & 1, s_abort);    // P^T of the last job lies there
                if (!ok) return;
                fence_after();
                product(tmem, sK, sQ + (j & 1) * 2 * SM::kT);
                commit_el(leader, s_full);
            };
            auto issue_dp = [&](int j) {                         // dP^T = V dO^T
                wait_tile(j, do_full, do_fixed, job.qb);
                next_job(job);
                if (ok && j > 0) ok = warp_wait(y_free + 8 * ((j - 1) & 1), ((j - 1) >> 1) & 1, s_abort);    // dS^T of the last job lies there
                if (!ok) return;
                fence_after();
                product(tmem + kY, sV, sQ + (j & 1) * 2 * SM::kT + SM::kT);
                commit_el(leader, dp_full);
            };
            issue_s(0);
            issue_dp(0);
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1;
                const uint32_t Q = sQ + st * 2 * SM::kT;
                ok = warp_wait(p_full, j & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDV, 0, Q + SM::kT, 0, 2, j == 0);    // dV += P^T dO
                ok = warp_wait(p_full + 8, j & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDV, 0, Q + SM::kT, 2, 4, false);
                commit_el(leader, x_free + 8 * st);
                if (j + 1 < J) issue_s(j + 1);
                if (ok) ok = warp_wait(ds_full, j & 1, s_abort);
                if (!ok) break;
                fence_after();
                accumulate(kDK, kY, Q, 0, 4, j == 0);            // dK += dS^T Q
                commit_el(leader, y_free + 8 * st);
                if (j + 1 < J) issue_dp(j + 1);
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
        const uint64_t scale2 = pk2(a.scale_log2, a.scale_log2);
        bool ok = true;
        Job job = job0;
        for (int j = 0; j < J; ++j, next_job(job)) {
            const int st = j & 1, c0 = job.qb + 64 * half;           // first query of this thread's columns
            const float* stat = reinterpret_cast<const float*>(smem + 6 * SM::kT + st * 2 * SM::kStat) + 64 * half;      // -lse; -delta one kStat on
            if (ok) ok = warp_wait(q_full + 8 * st, (j >> 1) & 1, s_abort);      // the statistics
            if (ok) ok = warp_wait(s_full, j & 1, s_abort);
            if (!ok) break;
            fence_after();
            const bool full = c0 >= full_lo && c0 + 64 <= full_hi;
            uint32_t s[2][32], d[2][32], y[2][16];
            tmem_ld32(tmem + at, s[0]);
            tmem_ld32(tmem + at + 32, s[1]);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                // two columns' words as one 64-bit load, the same for every lane
                auto nl = [&](int x) { return *reinterpret_cast<const uint64_t*>(stat + 32 * c + x); };
                if (full) chunk_p<false>(s[c], 0u, scale2, nl);
                else chunk_p<true>(s[c], bit_range(first - c0 - 32 * c, stop_all - c0 - 32 * c), scale2, nl);
#pragma unroll
                for (int x = 0; x < 16; ++x) y[c][x] = pack_bf16(__uint_as_float(s[c][2 * x]), __uint_as_float(s[c][2 * x + 1]));
                tmem_st16(tmem + at + 16 * c, y[c]);             // P^T of this half over its own S^T columns
                tmem_st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * c);
            }

            ok = warp_wait(dp_full, j & 1, s_abort);
            if (!ok) break;
            fence_after();
            tmem_ld32(tmem + kY + at, d[0]);
            tmem_ld32(tmem + kY + at + 32, d[1]);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                auto nd = [&](int x) { return *reinterpret_cast<const uint64_t*>(stat + kQTile + 32 * c + x); };
                if (full) chunk_ds<false>(s[c], d[c], nd, y[c]);
                else chunk_ds<true>(s[c], d[c], nd, y[c]);
                tmem_st16(tmem + kY + at + 16 * c, y[c]);        // dS^T over this half's own dP^T columns, which are in registers
            }
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) { mbar_arrive(ds_full); mbar_arrive(stat_empty + 8 * st); }
        }
        if (J > 0) {
            if (ok) ok = warp_wait(y_free + 8 * ((J - 1) & 1), ((J - 1) >> 1) & 1, s_abort);
            if (ok) ok = warp_wait(x_free + 8 * ((J - 1) & 1), ((J - 1) >> 1) & 1, s_abort);
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
    if (!win_map(&mk64, hk ? a.k : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.k_stride : any_ld, 64)) return -1;
    if (!win_map(&mv64, hk ? a.v : any, hk ? k_rows : any_rows, hk ? kc : any_cols, hk ? a.v_stride : any_ld, 64)) return -1;
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
        window_bwd_q_kernel<DH><<<dim3(s.item[a.batch], a.Hq), kThreads, SQ::kBytes, stream>>>(mq, mdo, mk64, mv64, a, s);
        ++launched;
    }
    if (hk) {
        WinSeqs t = s;                   // items of the key side: band tiles and sink segments
        t.item[0] = 0;
        for (int b = 0; b < a.batch; ++b) t.item[b + 1] = t.item[b] + (s.kv_len[b] + kKTile - 1) / kKTile + a.sink_tiles * a.sink_segs;
        if (t.item[a.batch] > 0) {
            window_bwd_kv_kernel<DH><<<dim3(t.item[a.batch], a.Hkv), kThreads, SK::kBytes, stream>>>(mq, mdo, mk, mv, a, t);
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
