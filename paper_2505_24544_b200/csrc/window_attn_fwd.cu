// Causal attention over whole sequences with a sliding window and sinks, forward, bf16, head_dim 64 / 128 (tcgen05).
//
// One CTA = 128 consecutive queries of one (sequence, query head): one tensor-memory lane and one softmax thread per query, so
// row maxima and sums need no shuffles.  Only the keys that the tile can see are walked: the sinks in front of the window
// (a tile of 32 columns when there are a few), then the band from the first query's oldest key to the last query's newest one
// in tiles of 128 that start where the band starts (rows of a TMA box may start anywhere), so a window of W costs
// about W + 128 columns per row.  Per tile: S = Q K^T into tensor memory -> the row threads form P = exp2(S - m) in bf16 and
// write it back over S, packed two to a column -> O += P V with P as the tensor-memory operand.  From shared memory such a
// product reads V alone: both operands there, at 128 rows, would need the full shared-memory bandwidth.  m is the
// row's reference point, moved only when a tile exceeds it by more than 2^8 (then the row's O is rescaled in tensor memory).
//
// S, P and O take 256 tensor-memory columns and K, V one tile each (96 KB with Q), so two CTAs share an SM and each one's
// softmax runs under the other's products; a second stage would buy nothing: K is free once S is complete and V is not
// needed before the softmax is through.
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
constexpr int kCols = 128;               // keys of a tile
constexpr float kSlack = 8.f;

template <int DH>
struct FwdSmem {
    static constexpr int kQ = kQTile * DH * 2, kK = kCols * DH * 2;
    static constexpr int kBytes = kQ + 2 * kK + 256 + 1024;      // barriers, alignment slack
};

// The key tiles of one query tile: sinks [0, sink_end) first, then the band [lo, hi).
struct KeyWalk {
    int lo, hi, sink_end, n_sink, n;
    __device__ __forceinline__ void init(int q0, int q_len, int shift, int window, int sinks, int step) {
        hi = min(q0 + kQTile, q_len) - 1 + shift + 1;            // one past the newest key of the last query
        lo = max(0, q0 + shift - window + 1);                    // the first query's oldest key inside the window
        sink_end = min(sinks, lo);
        n_sink = (sink_end + step - 1) / step;
        n = hi > 0 ? n_sink + (hi - lo + step - 1) / step : 0;
    }
    __device__ __forceinline__ void tile(int j, int step, int& start, int& end) const {
        if (j < n_sink) { start = j * step; end = min(start + step, sink_end); }
        else { start = lo + (j - n_sink) * step; end = min(start + step, hi); }
    }
};

template <int DH>
__global__ void __launch_bounds__(kThreads, 2) window_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ WinArgs a,
                                                               const __grid_constant__ WinSeqs seqs) {
    using SM = FwdSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kTmem = 256, kO = 128;            // S / P at column 0, O at 128
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sQ = smem_u32(smem), sK = sQ + SM::kQ, sV = sK + SM::kK;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + SM::kQ + 2 * SM::kK);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, k_full = bar0 + 8, k_empty = bar0 + 16, v_full = bar0 + 24, v_fixed = bar0 + 32, s_full = bar0 + 40,
                   p_full = bar0 + 48, pv_done = bar0 + 56;
    uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(bars + 16);
    volatile int* s_abort = reinterpret_cast<int*>(bars + 17);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int tile;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int q0 = ((q_len + kQTile - 1) / kQTile - 1 - tile) * kQTile;      // the latest (longest) tiles first
    const int h = blockIdx.y, kvh = h / a.G;
    const int q_row = seqs.q_start[b] + q0, k_row = seqs.k_start[b];
    KeyWalk w;
    w.init(q0, q_len, shift, a.window, a.sinks, kCols);
    const int J = w.n;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1); mbar_init(k_full, 1); mbar_init(k_empty, 1); mbar_init(v_full, 1); mbar_init(v_fixed, 1);
        mbar_init(s_full, 1); mbar_init(p_full, 4); mbar_init(pv_done, 1);
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
                mbar_expect_tx(q_full, SM::kQ);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(sQ + hf * (kQTile * 128), &tmQ, q_full, h * DH + hf * 64, q_row);
            }
            bool ok = true;
            int k_issued = 0, v_issued = 0;
            for (int j = 0; j < J && ok; ++j) {
                int start, end;
                w.tile(j, kCols, start, end);
                const int boxes = (end - start + 63) / 64;       // of 64 keys
                auto load = [&](uint32_t dst, const CUtensorMap* tm, uint32_t bar) {
                    if (lane == 0) {
                        mbar_expect_tx(bar, boxes * kHalves * 64 * 128);
                        for (int x = 0; x < boxes; ++x)
#pragma unroll
                            for (int hf = 0; hf < kHalves; ++hf)
                                tma_load_2d(dst + hf * (kCols * 128) + x * (64 * 128), tm, bar, kvh * DH + hf * 64, k_row + start + x * 64);
                    }
                    __syncwarp();
                };
                ok = __all_sync(0xffffffffu, mbar_wait(k_empty, (j & 1) ^ 1, s_abort));
                if (!ok) break;
                load(sK, &tmK, k_full);
                ++k_issued;
                ok = __all_sync(0xffffffffu, mbar_wait(pv_done, (j & 1) ^ 1, s_abort));
                if (!ok) break;
                load(sV, &tmV, v_full);
                ++v_issued;
                const int cols = (end - start + 31) & ~31;
                if (start + cols > kv_len) {                     // rows behind the sequence: zero
                    ok = __all_sync(0xffffffffu, mbar_wait(v_full, j & 1, s_abort));
                    if (!ok) break;
                    zero_rows<DH>(smem + SM::kQ + SM::kK, kCols, kv_len - start, cols, lane);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(v_fixed);
                }
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(q_full, 0); ++i) {}
                for (uint32_t i = 0; k_issued > 0 && i < kSpinLimit && !mbar_try_wait(k_full, (k_issued - 1) & 1); ++i) {}
                for (uint32_t i = 0; v_issued > 0 && i < kSpinLimit && !mbar_try_wait(v_full, (v_issued - 1) & 1); ++i) {}
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && J > 0) {
            constexpr uint32_t idesc_o = make_idesc_major(kQTile, DH, false, true);
            bool ok = mbar_wait(q_full, 0, s_abort);
            int fixes = 0;
            for (int j = 0; j < J && ok; ++j) {
                int start, end;
                w.tile(j, kCols, start, end);
                const int cols = (end - start + 31) & ~31;
                ok = mbar_wait(k_full, j & 1, s_abort);
                if (ok && j > 0) ok = mbar_wait(pv_done, (j - 1) & 1, s_abort);      // P of the last tile lies where S goes now
                if (!ok) break;
                fence_after();
                const uint32_t idesc_s = make_idesc(kQTile, cols);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    const uint64_t dq = umma_desc(sQ + hf * (kQTile * 128)), dk = umma_desc(sK + hf * (kCols * 128));
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k) {
                        const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                        umma_bf16(tmem, dq + off, dk + off, idesc_s, (hf > 0 || k > 0) ? 1u : 0u);
                    }
                }
                umma_commit(k_empty);
                umma_commit(s_full);
                ok = mbar_wait(p_full, j & 1, s_abort);
                if (ok) ok = mbar_wait(v_full, j & 1, s_abort);
                if (ok && start + cols > kv_len) ok = mbar_wait(v_fixed, fixes++ & 1, s_abort);
                if (!ok) break;
                fence_after();
                const uint64_t dv = umma_desc_mn(sV, kCols * 128);
                for (int k = 0; k < cols / UMMA_K; ++k)
                    umma_bf16_ts(tmem + kO, tmem + 8 * k, dv + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_o, (j > 0 || k > 0) ? 1u : 0u);
                umma_commit(pv_done);
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
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < J; ++j) {
            int start, end;
            w.tile(j, kCols, start, end);
            const int cols = (end - start + 31) & ~31;
            if (ok) ok = mbar_wait(s_full, j & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            uint32_t r[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (32 * c < cols) tmem_ld32(tmem + 32 * c + lanes, r[c]);
            tmem_ld_wait();
            const bool full = start + cols <= min(end, full_hi) && (start >= full_lo || end <= a.sinks);
            float mx = -INFINITY;
            if (!full) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (32 * c < cols) {
                        const int k0 = start + 32 * c;
                        const int top = valid ? min(last + 1, end) - k0 : 0;
                        const uint32_t vis = bit_range(oldest - k0, top) | bit_range(0, min(a.sinks - k0, top));
#pragma unroll
                        for (int x = 0; x < 32; ++x) r[c][x] = (vis >> x & 1u) ? r[c][x] : 0xff800000u;      // -inf
                    }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (32 * c < cols) {
                    float y = -INFINITY;                                 // two chains
#pragma unroll
                    for (int x = 0; x < 32; x += 2) {
                        mx = fmaxf(mx, __uint_as_float(r[c][x]));
                        y = fmaxf(y, __uint_as_float(r[c][x + 1]));
                    }
                    mx = fmaxf(mx, y);
                }
            mx *= a.scale_log2;
            const float m_old = m;
            const bool grow = mx > m_old + kSlack;
            m = grow ? mx : m_old;
            const float factor = (grow && m_old != -INFINITY) ? exp2f(m_old - m) : 1.f;
            if (__any_sync(0xffffffffu, factor != 1.f)) {                // (never in the first tile: m was -inf there)
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
            const float neg = m == -INFINITY ? 0.f : -m;                 // nothing visible so far: every weight is exp2(-inf) = 0
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (32 * c < cols) {
                    uint32_t p[16];
#pragma unroll
                    for (int x = 0; x < 32; x += 2) {
                        const float p0 = exp2f(fmaf(__uint_as_float(r[c][x]), a.scale_log2, neg));
                        const float p1 = exp2f(fmaf(__uint_as_float(r[c][x + 1]), a.scale_log2, neg));
                        l0 += p0;                                        // row sum in fp32 over the unrounded weights
                        l1 += p1;
                        p[x >> 1] = pack_bf16(p0, p1);
                    }
                    tmem_st16(tmem + 16 * c + lanes, p);                 // over S: this thread has all of its row in registers
                }
            l = fmaf(l, factor, l0 + l1);
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full);
        }
        if (J > 0) {
            if (ok) ok = mbar_wait(pv_done, (J - 1) & 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
        }
        const float inv = !ok ? __int_as_float(0x7fffffff) : l > 0.f ? 1.f / l : 0.f;
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
                    for (int z = 0; z < 4; ++z)
                        y[z] = J > 0 ? pack_bf16(__uint_as_float(o[x + 2 * z]) * inv, __uint_as_float(o[x + 2 * z + 1]) * inv) : 0u;
                    // a row that saw nothing has every weight 0: O is 0 already
                    *reinterpret_cast<uint4*>(dst + c0 + x) = make_uint4(y[0], y[1], y[2], y[3]);
                }
            }
        }
        if (valid && a.lse_out != nullptr)
            a.lse_out[(size_t)(q_row + q * 32 + lane) * a.Hq + h] = !ok ? inv : l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
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
    window_fwd_kernel<DH><<<dim3(s.item[a.batch], a.Hq), kThreads, SM::kBytes, stream>>>(mq, mk, mv, a, s);
    return 1;
}

}  // namespace

int window_fwd_bf16(const WinArgs& a, const WinSeqs& s, int dh, long long q_rows, long long k_rows, cudaStream_t stream) {
    return dh == 128 ? launch_fwd<128>(a, s, q_rows, k_rows, stream) : launch_fwd<64>(a, s, q_rows, k_rows, stream);
}

}  // namespace beagle
