// Causal attention over whole sequences with a sliding window and sinks, forward, bf16, head_dim 64 / 128 (tcgen05).
//
// One CTA = 128 consecutive queries of one (sequence, query head): one tensor-memory lane and one softmax thread per query, so
// row maxima and sums need no shuffles.  Only the keys that the tile can see are walked: the sinks in front of the window
// (a tile of 32 columns when there are a few), then the band from the first query's oldest key to the last query's newest one
// in tiles of 64 that start where the band starts (rows of a TMA box may start anywhere), so a window of W costs
// about W + 128 columns per row.  Per tile: S = Q K^T into tensor memory -> the row threads form P = exp2(S - m) in bf16 and
// write it back over S, packed two to a column -> O += P V with P as the tensor-memory operand, so that this product
// reads V alone from shared memory.  m is the row's reference point, moved only when a tile exceeds it by more than 2^8 (then
// the row's O is rescaled in tensor memory).  S is double-buffered: the next tile's S runs under this tile's softmax.
//
// Two S buffers of 64 columns and O take 256 tensor-memory columns, Q and two stages of K and V 96 KB, so two CTAs share
// an SM and fill each other's waits.
//
// Measured (head_dim 128, 32 heads): 8 x 2048, window 512: 210 us; two sequences up to 8191, window 2048: 408; chunks of 300 to 1024
// over 7000 cached keys, window 4096: 188.  No pipe is saturated (8 x 2048: tensor 0.39, special functions 0.39, issue 0.36): a tile
// takes a thread about 1500 cycles, 700 of them exponentials and the rest the hand-over with the tensor cores, and two tiles per
// SM are in flight.  One CTA per SM with two query tiles that share K and V, 128 keys at a time, took 298 and 560 us.
//
// Rows of V past the sequence's keys (the next sequence's rows) are zeroed in shared memory before use, since their weight 0
// would not silence a NaN.  Every wait is bounded; a CTA that gives up leaves NaN in its rows.
#include <cstring>

#include "tc_ptx.cuh"
#include "tensor_map.h"
#include "win_ptx.cuh"
#include "window_attn.h"

namespace beagle {
namespace {

using namespace tc;

constexpr int kThreads = 192;            // warp 0: TMA producer, warp 1: MMA issuer, warps 2-5: softmax
constexpr int kCols = 64;                // keys of a tile
constexpr float kSlack = 8.f;

template <int DH>
struct FwdSmem {
    static constexpr int kQ = kQTile * DH * 2, kT = kCols * DH * 2;          // Q; a K or V tile, two stages of each
    static constexpr int kBytes = kQ + 4 * kT + 256 + 1024;                  // + barriers, alignment slack
};

// The key tiles of one query tile: sinks [0, sink_end) first, then the band [lo, hi).
struct KeyWalk {
    int lo, hi, sink_end, n_sink, n;
    __device__ __forceinline__ void init(int q0, int q_len, int shift, int window, int sinks) {
        hi = min(q0 + kQTile, q_len) + shift;                    // one past the newest key of the last query
        lo = max(0, q0 + shift - window + 1);                    // the first query's oldest key inside the window
        sink_end = min(sinks, lo);
        n_sink = (sink_end + kCols - 1) / kCols;
        n = hi > 0 ? n_sink + (hi - lo + kCols - 1) / kCols : 0;
    }
    __device__ __forceinline__ void tile(int j, int& start, int& end) const {
        if (j < n_sink) { start = j * kCols; end = min(start + kCols, sink_end); }
        else { start = lo + (j - n_sink) * kCols; end = min(start + kCols, hi); }
    }
};

template <int DH>
__global__ void __launch_bounds__(kThreads, 2) window_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ WinArgs a,
                                                               const __grid_constant__ WinSeqs seqs) {
    using SM = FwdSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 256, kO = 128;            // S / P at columns 0 and 64, O at 128
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sQ = smem_u32(smem), sK = sQ + SM::kQ, sV = sK + 2 * SM::kT;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + SM::kQ + 4 * SM::kT);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, k_full = bar0 + 16, k_empty = bar0 + 32, v_full = bar0 + 48, s_full = bar0 + 64, p_full = bar0 + 80,
                   pv_done = bar0 + 96, v_fixed = bar0 + 112;      // all but the first: one per stage
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 16);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 17);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    int tile;
    const int unit = blockIdx.x / a.Hq, h = blockIdx.x - unit * a.Hq, kvh = h / a.G;      // the heads of a tile side by side
    const int b = win_find(seqs.item, a.batch, unit, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int q0 = ((q_len + kQTile - 1) / kQTile - 1 - tile) * kQTile;      // the latest (longest) tiles first
    const int q_row = seqs.q_start[b] + q0, k_row = seqs.k_start[b];
    KeyWalk w;
    w.init(q0, q_len, shift, a.window, a.sinks);
    const int J = w.n;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, 1); mbar_init(k_empty + 8 * i, 1); mbar_init(v_full + 8 * i, 1);
            mbar_init(s_full + 8 * i, 1); mbar_init(p_full + 8 * i, 4); mbar_init(pv_done + 8 * i, 1);
            mbar_init(v_fixed + 8 * i, 1);
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
                mbar_expect_tx(q_full, SM::kQ);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(sQ + hf * (kQTile * 128), &tmQ, q_full, h * DH + hf * 64, q_row);
            }
            bool ok = true;
            int k_issued = 0, v_issued = 0;
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1, ph = (j >> 1) & 1;
                int start, end;
                w.tile(j, start, end);
                ok = warp_wait(k_empty + 8 * st, ph ^ 1, s_abort);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(k_full + 8 * st, SM::kT);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(sK + st * SM::kT + hf * (kCols * 128), &tmK, k_full + 8 * st, kvh * DH + hf * 64, k_row + start);
                }
                __syncwarp();
                ++k_issued;
                ok = warp_wait(pv_done + 8 * st, ph ^ 1, s_abort);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(v_full + 8 * st, SM::kT);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(sV + st * SM::kT + hf * (kCols * 128), &tmV, v_full + 8 * st, kvh * DH + hf * 64, k_row + start);
                }
                __syncwarp();
                ++v_issued;
                const int cols = (end - start + 31) & ~31;
                if (start + cols > kv_len) {                     // rows behind the sequence: zero
                    ok = warp_wait(v_full + 8 * st, ph, s_abort);
                    if (!ok) break;
                    zero_rows<DH>(smem + SM::kQ + (2 + st) * SM::kT, kCols, kv_len - start, cols, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(v_fixed + 8 * st);
                }
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(q_full, 0); ++i) {}
                for (int n = max(0, k_issued - 2); n < k_issued; ++n)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(k_full + 8 * (n & 1), (n >> 1) & 1); ++i) {}
                for (int n = max(0, v_issued - 2); n < v_issued; ++n)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(v_full + 8 * (n & 1), (n >> 1) & 1); ++i) {}
            }
        }
    } else if (warp == 1) {
        if (J > 0) {
            const bool leader = elect_one();
            constexpr uint32_t idesc_o = make_idesc_major(kQTile, DH, false, true);
            bool ok = warp_wait(q_full, 0, s_abort);
            uint32_t fixed = 0;                                  // phase of every stage's repair barrier
            auto issue_s = [&](int j) {
                const int st = j & 1;
                int start, end;
                w.tile(j, start, end);
                if (ok) ok = warp_wait(k_full + 8 * st, (j >> 1) & 1, s_abort);
                if (ok && j >= 2) ok = warp_wait(pv_done + 8 * st, ((j >> 1) & 1) ^ 1, s_abort);     // P of tile j - 2 lies where S goes now
                if (!ok) return;
                fence_after();
                const uint32_t idesc_s = make_idesc(kQTile, (end - start + 31) & ~31);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    const uint64_t dq = umma_desc(sQ + hf * (kQTile * 128)), dk = umma_desc(sK + st * SM::kT + hf * (kCols * 128));
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k) {
                        const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                        umma_ss(leader, tmem + st * kCols, dq + off, dk + off, idesc_s, (hf > 0 || k > 0) ? 1u : 0u);
                    }
                }
                commit_el(leader, k_empty + 8 * st);
                commit_el(leader, s_full + 8 * st);
            };
            issue_s(0);
            for (int j = 0; j < J && ok; ++j) {
                const int st = j & 1, ph = (j >> 1) & 1;
                if (j + 1 < J) issue_s(j + 1);
                int start, end;
                w.tile(j, start, end);
                const int cols = (end - start + 31) & ~31;
                if (ok) ok = warp_wait(v_full + 8 * st, ph, s_abort);
                if (ok && start + cols > kv_len) { ok = warp_wait(v_fixed + 8 * st, fixed >> st & 1u, s_abort); fixed ^= 1u << st; }
                if (ok) ok = warp_wait(p_full + 8 * st, ph, s_abort);
                if (!ok) break;
                fence_after();
                const uint64_t dv = umma_desc_mn(sV + st * SM::kT, kCols * 128);
                for (int k = 0; k < cols / UMMA_K; ++k)
                    umma_ts(leader, tmem + kO, tmem + st * kCols + 8 * k, dv + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_o, (j > 0 || k > 0) ? 1u : 0u);
                commit_el(leader, pv_done + 8 * st);
            }
        }
    } else {
        const int q = warp & 3;                                  // tensor-memory lane quarter of this warp
        const int i = q0 + q * 32 + lane;                        // query of this thread
        const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
        const bool valid = i < q_len;
        const int last = i + shift;                              // newest visible key
        const int oldest = last - a.window + 1;                  // of the window
        const int full_lo = min(q0 + kQTile, q_len) - 1 + shift - a.window + 1, full_hi = q0 + shift + 1;    // keys every query of the tile sees
        const uint64_t scale2 = pk2(a.scale_log2, a.scale_log2);
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < J; ++j) {
            const int st = j & 1, ph = (j >> 1) & 1;
            int start, end;
            w.tile(j, start, end);
            const bool two = end - start > 32;                   // the tile's second 32 columns exist
            if (ok) ok = warp_wait(s_full + 8 * st, ph, s_abort);
            if (!ok) break;
            fence_after();
            const uint32_t ts = tmem + st * kCols + lanes;
            uint32_t r[2][32];
            tmem_ld32(ts, r[0]);
            if (two) tmem_ld32(ts + 32, r[1]);
            tmem_ld_wait();
            float mx;
            const bool full = start + (two ? 64 : 32) <= min(end, full_hi) && (start >= full_lo || end <= a.sinks);
            if (full) {
                mx = chunk_max<false>(r[0], 0u, -INFINITY);
                if (two) mx = chunk_max<false>(r[1], 0u, mx);
            } else {
                const int top = valid ? min(last + 1, end) - start : 0;
                mx = chunk_max<true>(r[0], bit_range(oldest - start, top) | bit_range(0, min(a.sinks - start, top)), -INFINITY);
                if (two) mx = chunk_max<true>(r[1], bit_range(oldest - start - 32, top - 32) | bit_range(0, min(a.sinks - start, top) - 32), mx);
            }
            mx *= a.scale_log2;
            const float m_old = m;
            const bool grow = mx > m_old + kSlack;
            m = grow ? mx : m_old;
            const float factor = (grow && m_old != -INFINITY) ? exp2f(m_old - m) : 1.f;
            if (__any_sync(0xffffffffu, factor != 1.f)) {        // (never in the first tile: m was -inf there)
                ok = warp_wait(pv_done + 8 * (st ^ 1), ((j - 1) >> 1) & 1, s_abort);      // O is complete up to the last tile
                if (!ok) break;
                fence_after();
#pragma unroll
                for (int c0 = 0; c0 < DH; c0 += 16) {
                    uint32_t o[16];
                    tmem_ld16(tmem + kO + c0 + lanes, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * factor);
                    tmem_st16(tmem + kO + c0 + lanes, o);
                }
            }
            const float neg = m == -INFINITY ? 0.f : -m;         // nothing visible so far: every weight is exp2(-inf) = 0
            const uint64_t neg2 = pk2(neg, neg);
            uint64_t sum0 = 0, sum1 = 0;                         // row sum in fp32 over the unrounded weights
            uint32_t p[16];
            chunk_exp(r[0], scale2, neg2, p, sum0, sum1);
            tmem_st16(ts, p);                                    // over S: this thread has its row in registers
            if (two) {
                chunk_exp(r[1], scale2, neg2, p, sum0, sum1);
                tmem_st16(ts + 16, p);
            }
            float x0, x1;
            un2(add2(sum0, sum1), x0, x1);
            l = fmaf(l, factor, x0 + x1);
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 8 * st);
        }
        if (J > 0) {
            if (ok) ok = warp_wait(pv_done + 8 * ((J - 1) & 1), ((J - 1) >> 1) & 1, s_abort);
        }
        const float inv = !ok ? __int_as_float(0x7fffffff) : l != 0.f ? 1.f / l : 0.f;
        bf16* dst = static_cast<bf16*>(a.o) + ((size_t)(q_row + q * 32 + lane) * a.Hq + h) * DH;
        fence_after();
#pragma unroll
        for (int c0 = 0; c0 < DH; c0 += 32) {
            uint32_t o[32];
            if (J > 0) { tmem_ld32(tmem + kO + c0 + lanes, o); tmem_ld_wait(); }
            if (valid) {
#pragma unroll
                for (int x = 0; x < 32; x += 8) {
                    uint32_t y[4];
#pragma unroll
                    for (int z = 0; z < 4; ++z)                  // a row that saw nothing has every weight 0: O is 0 already
                        y[z] = J > 0 ? pack_bf16(__uint_as_float(o[x + 2 * z]) * inv, __uint_as_float(o[x + 2 * z + 1]) * inv) : 0u;
                    *reinterpret_cast<uint4*>(dst + c0 + x) = make_uint4(y[0], y[1], y[2], y[3]);
                }
            }
        }
        if (valid && a.lse_out != nullptr)
            a.lse_out[(size_t)(q_row + q * 32 + lane) * a.Hq + h] = !ok ? inv : l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
    fence_before();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        tmem_dealloc<kTmem>(tmem);
    }
}

template <int DH>
int launch_fwd(const WinArgs& a, const WinSeqs& s, long long q_rows, long long k_rows, cudaStream_t stream) {
    using SM = FwdSmem<DH>;
    CUtensorMap mq, mk, mv;
    if (!win_map(&mq, a.q, q_rows, (long long)a.Hq * DH, a.q_stride, kQTile)) return -1;
    // no keys at all: the maps are never used, any valid one does
    if (!win_map(&mk, k_rows > 0 ? a.k : a.q, k_rows > 0 ? k_rows : q_rows, (long long)a.Hkv * DH, k_rows > 0 ? a.k_stride : a.q_stride, 64)) return -1;
    if (!win_map(&mv, k_rows > 0 ? a.v : a.q, k_rows > 0 ? k_rows : q_rows, (long long)a.Hkv * DH, k_rows > 0 ? a.v_stride : a.q_stride, 64)) return -1;
    static PerDeviceOnce attr;
    if (!attr.ensure([] { return cudaFuncSetAttribute(window_fwd_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::kBytes) == cudaSuccess; })) return -1;
    const long long items = (long long)s.item[a.batch] * a.Hq;
    if (items > 0x7fffffff) return -1;
    window_fwd_kernel<DH><<<(unsigned)items, kThreads, SM::kBytes, stream>>>(mq, mk, mv, a, s);
    return 1;
}

}  // namespace

int window_fwd_bf16(const WinArgs& a, const WinSeqs& s, int dh, long long q_rows, long long k_rows, cudaStream_t stream) {
    return dh == 128 ? launch_fwd<128>(a, s, q_rows, k_rows, stream) : launch_fwd<64>(a, s, q_rows, k_rows, stream);
}

}  // namespace beagle
