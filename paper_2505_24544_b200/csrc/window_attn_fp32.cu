// The windowed attention in fp32 (forward and backward), head_dim 16 | 32 | 64 | 128, on the CUDA cores: the tiny head's type,
// for which exactness counts more than rate (no tensor-core product keeps 24 bits).
//
// Tiles of R x 64 (R = 64 or 32 rows: queries, or keys on the key side; R = 32 while 64 would leave SMs without a CTA); 256
// threads as 16 x 16, each with an R/16 x 4 piece of S (operands read as 16-byte vectors from padded shared-memory rows) and
// with its R/16 rows x head_dim / 16 columns of the accumulators.  The 16 threads of a row are half a warp, so row maxima, sums
// and the hand-over of P through shared memory need no CTA barrier.  The streamed tiles come by cp.async, the next one under
// this one's work where shared memory holds two.
// Backward as in the bf16 kernels: a query side (dQ, and delta) and a key side (dK, dV), what lies past the band of the sinks in segments;
// the key side gives every query head its own CTA and, where heads share keys, leaves fp32 partials that a last launch adds in the
// order of the heads.
//
// Measured: three sequences up to 333, 4 heads of 64, window 64: forward 14 us, query side 20, key side 36, all latency (88 CTAs).
#include "tensor_map.h"
#include "window_attn.h"

namespace beagle {
namespace {

constexpr int kT = 64;                   // queries, and keys, of a tile
constexpr int kPad = 4;
constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int DH> __host__ __device__ constexpr int row_len() { return DH + kPad; }
constexpr int kPRow = kT + kPad;

__device__ __forceinline__ bool visible(int key, int last, const WinArgs& a) { return key <= last && (key > last - a.window || key < a.sinks); }

__device__ __forceinline__ void cp_async16(float* dst, const float* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows [r0, r0 + R) of a packed matrix (column offset `col`) on their way into shared memory; rows at and past `rows` as zero.
template <int DH, int R>
__device__ __forceinline__ void load_tile(float* dst, const float* src, long long stride, int r0, int rows, size_t col) {
#pragma unroll
    for (int i = threadIdx.x; i < R * (DH / 4); i += kThreads) {
        const int r = i / (DH / 4), c = i % (DH / 4);
        const bool there = r0 + r < rows;
        cp_async16(dst + r * row_len<DH>() + 4 * c, src + (size_t)(there ? r0 + r : 0) * stride + col + 4 * c, there);
    }
}
// acc[r][c] = <A row (RT ty + r), B row (tx + 16 c)>
template <int DH, int RT>
__device__ __forceinline__ void dots(const float* A, const float* B, int ty, int tx, float acc[RT][4]) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[r][c] = 0.f;
#pragma unroll 4
    for (int d = 0; d < DH; d += 4) {
        float4 x[RT], y[4];
#pragma unroll
        for (int r = 0; r < RT; ++r) x[r] = *reinterpret_cast<const float4*>(A + (RT * ty + r) * row_len<DH>() + d);
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = *reinterpret_cast<const float4*>(B + (tx + 16 * c) * row_len<DH>() + d);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                acc[r][c] = fmaf(x[r].x, y[c].x, fmaf(x[r].y, y[c].y, fmaf(x[r].z, y[c].z, fmaf(x[r].w, y[c].w, acc[r][c]))));
    }
}
// The accumulator columns of a thread: runs of up to four, so that they load and store as vectors.
template <int DH>
__device__ __forceinline__ int col(int tx, int e) { return DH >= 64 ? 64 * (e / 4) + 4 * tx + e % 4 : DH / 16 * tx + e; }
// DH / 16 values at the thread's columns of a row.
template <int DH>
__device__ __forceinline__ void get_cols(const float* row, int tx, float* x) {
    if constexpr (DH >= 64) {
#pragma unroll
        for (int e = 0; e < DH / 16; e += 4) {
            const float4 t = *reinterpret_cast<const float4*>(row + col<DH>(tx, e));
            x[e] = t.x; x[e + 1] = t.y; x[e + 2] = t.z; x[e + 3] = t.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) x[e] = row[col<DH>(tx, e)];
    }
}
template <int DH>
__device__ __forceinline__ void set_cols(float* row, int tx, const float* x, float f) {
    if constexpr (DH >= 64) {
#pragma unroll
        for (int e = 0; e < DH / 16; e += 4) *reinterpret_cast<float4*>(row + col<DH>(tx, e)) = make_float4(x[e] * f, x[e + 1] * f, x[e + 2] * f, x[e + 3] * f);
    } else {
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) row[col<DH>(tx, e)] = x[e] * f;
    }
}
// acc[r][e] += sum_k P[RT ty + r][k] X[k][col(e)]
template <int DH, int RT>
__device__ __forceinline__ void weigh(const float* P, const float* X, int ty, int tx, float acc[RT][DH / 16]) {
#pragma unroll 2
    for (int k = 0; k < kT; k += 4) {
        float p[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const float4 t = *reinterpret_cast<const float4*>(P + (RT * ty + r) * kPRow + k);
            p[r][0] = t.x; p[r][1] = t.y; p[r][2] = t.z; p[r][3] = t.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[DH / 16];
            get_cols<DH>(X + (k + i) * row_len<DH>(), tx, x);
#pragma unroll
            for (int e = 0; e < DH / 16; ++e)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[r][e] = fmaf(p[r][i], x[e], acc[r][e]);
        }
    }
}
template <int RT>
__device__ __forceinline__ void put(float* P, int ty, int tx, const float v[RT][4]) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) P[(RT * ty + r) * kPRow + tx + 16 * c] = v[r][c];
}
// Shared memory: NR resident and 2 * stages streamed tiles, NP tiles of P; two stages where they fit.
template <int DH, int R, int NR, int NP>
struct Fp32Smem {
    static constexpr int kRes = R * (DH + kPad), kStr = kT * (DH + kPad), kP = R * kPRow;
    static constexpr int kStages = (NR * kRes + 4 * kStr + NP * kP) * 4 <= 227 * 1024 ? 2 : 1;
    static constexpr int kBytes = (NR * kRes + 2 * kStages * kStr + NP * kP) * 4;
};

// The key tiles of the queries [q0, q0 + R): sinks in front of the window, then the band.
struct Keys {
    int lo, hi, sink_end, n_sink, n;
    __device__ __forceinline__ void init(int q0, int rows, int q_len, int shift, const WinArgs& a) {
        hi = min(q0 + rows, q_len) + shift;
        lo = max(0, q0 + shift - a.window + 1);
        sink_end = min(a.sinks, lo);
        n_sink = (sink_end + kT - 1) / kT;
        n = hi > 0 ? n_sink + (hi - lo + kT - 1) / kT : 0;
    }
    __device__ __forceinline__ void tile(int j, int& start, int& end) const {
        if (j < n_sink) { start = j * kT; end = min(start + kT, sink_end); }
        else { start = lo + (j - n_sink) * kT; end = min(start + kT, hi); }
    }
};

template <int DH, int R>
__global__ void __launch_bounds__(kThreads) window_fwd_fp32_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    extern __shared__ __align__(16) float sm[];
    using SM = Fp32Smem<DH, R, 1, 1>;
    constexpr int RT = R / 16;
    float *Q = sm, *KV = Q + SM::kRes, *P = KV + 2 * SM::kStages * SM::kStr;       // stage s: K at KV + 2 s kStr, V behind it
    int tile;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int q0 = ((q_len + R - 1) / R - 1 - tile) * R, h = blockIdx.y, kvh = h / a.G;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    load_tile<DH, R>(Q, static_cast<const float*>(a.q) + (size_t)seqs.q_start[b] * a.q_stride, a.q_stride, q0, q_len, (size_t)h * DH);
    cp_commit();
    Keys w;
    w.init(q0, R, q_len, shift, a);
    float o[RT][DH / 16], m[RT], l[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) o[r][e] = 0.f;
    }
    auto load_kv = [&](int j) {
        int start, end;
        w.tile(j, start, end);
        float* dst = KV + (j % SM::kStages) * 2 * SM::kStr;
        load_tile<DH, kT>(dst, static_cast<const float*>(a.k) + (size_t)seqs.k_start[b] * a.k_stride, a.k_stride, start, end, (size_t)kvh * DH);
        load_tile<DH, kT>(dst + SM::kStr, static_cast<const float*>(a.v) + (size_t)seqs.k_start[b] * a.v_stride, a.v_stride, start, end, (size_t)kvh * DH);
        cp_commit();
    };
    if (SM::kStages == 2 && w.n > 0) load_kv(0);
    for (int j = 0; j < w.n; ++j) {
        int start, end;
        w.tile(j, start, end);
        __syncthreads();                                 // the tile that the next copy overwrites has been read
        if (SM::kStages == 1) load_kv(j);
        else if (j + 1 < w.n) load_kv(j + 1);
        if (SM::kStages == 2 && j + 1 < w.n) cp_wait<1>();
        else cp_wait<0>();
        __syncthreads();
        const float *K = KV + (j % SM::kStages) * 2 * SM::kStr, *V = K + SM::kStr;
        float s[RT][4];
        dots<DH, RT>(Q, K, ty, tx, s);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int last = q0 + RT * ty + r + shift;
            float mx = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int key = start + tx + 16 * c;
                s[r][c] = (key < end && visible(key, last, a)) ? s[r][c] * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[r][c]);
            }
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            mx = fmaxf(mx, m[r]);
            const float f = m[r] == -INFINITY ? 1.f : exp2f(m[r] - mx);
            const float neg = mx == -INFINITY ? 0.f : -mx;
            m[r] = mx;
            l[r] *= f;
#pragma unroll
            for (int e = 0; e < DH / 16; ++e) o[r][e] *= f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[r][c] = exp2f(s[r][c] + neg);
                l[r] += s[r][c];
            }
        }
        put<RT>(P, ty, tx, s);
        __syncwarp();                                    // a row's 16 threads are half of one warp
        weigh<DH, RT>(P, V, ty, tx, o);
        __syncwarp();
    }
    cp_wait<0>();                                        // (a CTA without tiles: its queries have landed before it ends)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
        const int i = q0 + RT * ty + r;
        if (i >= q_len) continue;
        const size_t row = ((size_t)(seqs.q_start[b] + i) * a.Hq + h);
        const float inv = l[r] != 0.f ? __fdiv_rn(1.f, l[r]) : 0.f;
        set_cols<DH>(static_cast<float*>(a.o) + row * DH, tx, o[r], inv);
        if (tx == 0 && a.lse_out != nullptr) a.lse_out[row] = l[r] != 0.f ? (m[r] + log2f(l[r])) * kLn2 : -INFINITY;
    }
}

__device__ __forceinline__ int stat_row0(const WinSeqs& s, int b) {
    int at = 0;
    for (int i = 0; i < b; ++i) at += (s.q_len[i] + kStatPad - 1) / kStatPad * kStatPad;
    return at;
}

template <int DH, int R>
__global__ void __launch_bounds__(kThreads) window_bwd_q_fp32_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    extern __shared__ __align__(16) float sm[];
    using SM = Fp32Smem<DH, R, 2, 1>;
    constexpr int RT = R / 16;
    float *Q = sm, *dO = Q + SM::kRes, *KV = dO + SM::kRes, *P = KV + 2 * SM::kStages * SM::kStr;
    int tile;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int q0 = ((q_len + R - 1) / R - 1 - tile) * R, h = blockIdx.y, kvh = h / a.G;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    load_tile<DH, R>(Q, static_cast<const float*>(a.q) + (size_t)seqs.q_start[b] * a.q_stride, a.q_stride, q0, q_len, (size_t)h * DH);
    load_tile<DH, R>(dO, static_cast<const float*>(a.dout) + (size_t)seqs.q_start[b] * a.dout_stride, a.dout_stride, q0, q_len, (size_t)h * DH);
    cp_commit();
    cp_wait<0>();
    __syncthreads();
    float lse2[RT], delta[RT], dq[RT][DH / 16];
    const int stat0 = stat_row0(seqs, b);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int i = q0 + RT * ty + r;
        const size_t row = (size_t)(seqs.q_start[b] + min(i, q_len - 1)) * a.Hq + h;
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) {
            t = fmaf(dO[(RT * ty + r) * row_len<DH>() + tx + 16 * e], static_cast<const float*>(a.out)[row * DH + tx + 16 * e], t);      // (any order of the columns)
            dq[r][e] = 0.f;
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
        const bool sees = i + shift >= 0;
        delta[r] = sees ? t : 0.f;
        lse2[r] = sees ? a.lse[row] * kLog2e : 0.f;
        if (tx == 0 && i < q_len) {
            float* stat = a.stats + (size_t)h * 2 * a.stat_rows + stat0 + i;
            stat[0] = -lse2[r];
            stat[a.stat_rows] = -delta[r];
        }
    }
    Keys w;
    w.init(q0, R, q_len, shift, a);
    auto load_kv = [&](int j) {
        int start, end;
        w.tile(j, start, end);
        float* dst = KV + (j % SM::kStages) * 2 * SM::kStr;
        load_tile<DH, kT>(dst, static_cast<const float*>(a.k) + (size_t)seqs.k_start[b] * a.k_stride, a.k_stride, start, end, (size_t)kvh * DH);
        load_tile<DH, kT>(dst + SM::kStr, static_cast<const float*>(a.v) + (size_t)seqs.k_start[b] * a.v_stride, a.v_stride, start, end, (size_t)kvh * DH);
        cp_commit();
    };
    if (SM::kStages == 2 && w.n > 0) load_kv(0);
    for (int j = 0; j < w.n; ++j) {
        int start, end;
        w.tile(j, start, end);
        __syncthreads();                                 // the tile that the next copy overwrites has been read
        if (SM::kStages == 1) load_kv(j);
        else if (j + 1 < w.n) load_kv(j + 1);
        if (SM::kStages == 2 && j + 1 < w.n) cp_wait<1>();
        else cp_wait<0>();
        __syncthreads();
        const float *K = KV + (j % SM::kStages) * 2 * SM::kStr, *V = K + SM::kStr;
        float s[RT][4], dp[RT][4];
        dots<DH, RT>(Q, K, ty, tx, s);
        dots<DH, RT>(dO, V, ty, tx, dp);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int last = q0 + RT * ty + r + shift;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int key = start + tx + 16 * c;
                s[r][c] = (key < end && visible(key, last, a)) ? exp2f(fmaf(s[r][c], a.scale_log2, -lse2[r])) * (dp[r][c] - delta[r]) : 0.f;
            }
        }
        put<RT>(P, ty, tx, s);
        __syncwarp();
        weigh<DH, RT>(P, K, ty, tx, dq);
        __syncwarp();
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int i = q0 + RT * ty + r;
        if (i >= q_len) continue;
        set_cols<DH>(static_cast<float*>(a.dq) + (size_t)(seqs.q_start[b] + i) * a.dq_stride + (size_t)h * DH, tx, dq[r], a.scale);
    }
}

// One CTA = R keys of one (sequence, query head).  What lies past the band of a sink tile is cut into segments, CTAs of their own that
// come first; the rows of that sequence's sinks then go to a.sink_part (the band's part, then the segments').  a.group_part (where heads
// share keys): [kv rows][Hq][2][DH], dV then dK.  The last launches add both up in order.
template <int DH, int R>
__global__ void __launch_bounds__(kThreads) window_bwd_kv_fp32_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs) {
    extern __shared__ __align__(16) float sm[];
    using SM = Fp32Smem<DH, R, 2, 2>;
    constexpr int RT = R / 16;
    float *K = sm, *V = K + SM::kRes, *QD = V + SM::kRes, *P = QD + 2 * SM::kStages * SM::kStr, *dS = P + SM::kP;
    int tile;
    const int b = win_find(seqs.item, a.batch, blockIdx.x, tile);
    const int q_len = seqs.q_len[b], kv_len = seqs.kv_len[b], shift = kv_len - q_len - a.strict;
    const int segs = seqs.segs[b], parts = (min(a.sinks, kv_len) + R - 1) / R * segs;
    const int seg = tile < parts ? tile % segs : -1;
    const int k0 = (seg >= 0 ? tile / segs : tile - parts) * R, h = blockIdx.y, kvh = h / a.G;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    load_tile<DH, R>(K, static_cast<const float*>(a.k) + (size_t)seqs.k_start[b] * a.k_stride, a.k_stride, k0, kv_len, (size_t)kvh * DH);
    load_tile<DH, R>(V, static_cast<const float*>(a.v) + (size_t)seqs.k_start[b] * a.v_stride, a.v_stride, k0, kv_len, (size_t)kvh * DH);
    const int band = max(0, min(q_len, min(k0 + R, kv_len) - 1 - shift + a.window));      // the first query past the band
    int from = max(0, k0 - shift), to = k0 < a.sinks && segs == 0 ? q_len : band;
    if (seg >= 0) {
        from = max(from, band);
        const int all = from < q_len ? (q_len - from + kT - 1) / kT : 0;
        to = min(q_len, from + (int)((long long)all * (seg + 1) / segs) * kT);
        from += (int)((long long)all * seg / segs) * kT;
    }
    const float* stats = a.stats + (size_t)h * 2 * a.stat_rows + stat_row0(seqs, b);
    float dk[RT][DH / 16], dv[RT][DH / 16];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) dk[r][e] = dv[r][e] = 0.f;
    const int n = to > from ? (to - from + kT - 1) / kT : 0;
    cp_commit();
    auto load_qd = [&](int j) {
        float* dst = QD + (j % SM::kStages) * 2 * SM::kStr;
        load_tile<DH, kT>(dst, static_cast<const float*>(a.q) + (size_t)seqs.q_start[b] * a.q_stride, a.q_stride, from + j * kT, q_len, (size_t)h * DH);
        load_tile<DH, kT>(dst + SM::kStr, static_cast<const float*>(a.dout) + (size_t)seqs.q_start[b] * a.dout_stride, a.dout_stride, from + j * kT, q_len, (size_t)h * DH);
        cp_commit();
    };
    if (SM::kStages == 2 && n > 0) load_qd(0);
    for (int j = 0; j < n; ++j) {
        const int q0 = from + j * kT;
        __syncthreads();
        if (SM::kStages == 1) load_qd(j);
        else if (j + 1 < n) load_qd(j + 1);
        if (SM::kStages == 2 && j + 1 < n) cp_wait<1>();
        else cp_wait<0>();
        __syncthreads();
        const float *Q = QD + (j % SM::kStages) * 2 * SM::kStr, *dO = Q + SM::kStr;
        float s[RT][4], dp[RT][4];
        dots<DH, RT>(K, Q, ty, tx, s);
        dots<DH, RT>(V, dO, ty, tx, dp);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int i = q0 + tx + 16 * c;
            const float nl = i < q_len ? __ldg(stats + i) : 0.f, nd = i < q_len ? __ldg(stats + a.stat_rows + i) : 0.f;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bool vis = i < to && visible(k0 + RT * ty + r, i + shift, a);
                const float p = vis ? exp2f(fmaf(s[r][c], a.scale_log2, nl)) : 0.f;
                s[r][c] = p;
                dp[r][c] = vis ? p * (dp[r][c] + nd) : 0.f;
            }
        }
        put<RT>(P, ty, tx, s);
        put<RT>(dS, ty, tx, dp);
        __syncwarp();
        weigh<DH, RT>(P, dO, ty, tx, dv);
        weigh<DH, RT>(dS, Q, ty, tx, dk);
        __syncwarp();
    }
    cp_wait<0>();                                        // (a CTA without tiles: its keys and values have landed before it ends)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int key = k0 + RT * ty + r;
        if (key >= kv_len) continue;
        const size_t row = (size_t)(seqs.k_start[b] + key);
        const bool part = segs > 0 && key < a.sinks;
        if (seg >= 0 && !part) continue;
        float* to_v = part ? a.sink_part + sink_row(a, seqs, b, h, 1 + seg, key) * 2 * DH
                    : a.G > 1 ? a.group_part + (row * a.Hq + h) * 2 * DH : static_cast<float*>(a.dv) + row * a.dv_stride + (size_t)kvh * DH;
        float* to_k = part || a.G > 1 ? to_v + DH : static_cast<float*>(a.dk) + row * a.dk_stride + (size_t)kvh * DH;
        set_cols<DH>(to_v, tx, dv[r], 1.f);
        set_cols<DH>(to_k, tx, dk[r], a.scale);
    }
}

// dK, dV of one key row: the query heads of every group added in order.
__global__ void __launch_bounds__(256) window_group_join_fp32_kernel(const __grid_constant__ WinArgs a, int DH, long long rows) {
    const long long n = rows * a.Hkv * 2 * DH;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int c = (int)(i % (2 * DH));
        const long long rest = i / (2 * DH);
        const int kvh = (int)(rest % a.Hkv);
        const long long row = rest / a.Hkv;
        const float* p = a.group_part + ((size_t)row * a.Hq + (size_t)kvh * a.G) * 2 * DH + c;
        float x = 0.f;
        for (int g = 0; g < a.G; ++g) x += p[(size_t)g * 2 * DH];
        if (c < DH) static_cast<float*>(a.dv)[(size_t)row * a.dv_stride + (size_t)kvh * DH + c] = x;
        else static_cast<float*>(a.dk)[(size_t)row * a.dk_stride + (size_t)kvh * DH + c - DH] = x;
    }
}

// dK, dV of the sinks: head after head of the group, the band's part and the segments' of each.  blockIdx = (row, K/V head, sequence).
__global__ void __launch_bounds__(256) window_sink_join_fp32_kernel(const __grid_constant__ WinArgs a, const __grid_constant__ WinSeqs seqs, int DH) {
    const int key = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z, c = threadIdx.x;
    const int segs = seqs.segs[b], rows = min(a.sinks, seqs.kv_len[b]);
    if (segs == 0 || key >= rows || c >= 2 * DH) return;
    const float* p = a.sink_part + sink_row(a, seqs, b, kvh * a.G, 0, key) * 2 * DH + c;
    float x = 0.f;
    for (int i = 0; i < a.G * (1 + segs); ++i) x += p[(size_t)i * rows * 2 * DH];
    const size_t row = (size_t)(seqs.k_start[b] + key);
    if (c < DH) static_cast<float*>(a.dv)[row * a.dv_stride + (size_t)kvh * DH + c] = x;
    else static_cast<float*>(a.dk)[row * a.dk_stride + (size_t)kvh * DH + c - DH] = x;
}

int retile(WinSeqs& s, int batch, const int32_t* len, int rows) {
    s.item[0] = 0;
    for (int b = 0; b < batch; ++b) s.item[b + 1] = s.item[b] + (len[b] + rows - 1) / rows;
    return s.item[batch];
}
// 64 rows a CTA unless that leaves SMs idle (three sequences up to 333, 4 heads of 64: 48 CTAs of 64 rows, 92 of 32: forward and
// backward 35 + 88 us against 39 + 105).
bool small_rows(WinSeqs& s, int batch, const int32_t* len, int heads) { return (long long)retile(s, batch, len, 64) * heads < device_sm_count(); }

template <typename K, typename SM>
bool raise_limit(K kernel, PerDeviceOnce& once, SM) {
    return once.ensure([=] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::kBytes) == cudaSuccess; });
}

template <int DH, int R>
int fwd_rows(const WinArgs& a, WinSeqs s, cudaStream_t stream) {
    using SM = Fp32Smem<DH, R, 1, 1>;
    static PerDeviceOnce once;
    if (!raise_limit(window_fwd_fp32_kernel<DH, R>, once, SM())) return -1;
    window_fwd_fp32_kernel<DH, R><<<dim3(retile(s, a.batch, s.q_len, R), a.Hq), kThreads, SM::kBytes, stream>>>(a, s);
    return 1;
}
template <int DH, int R>
int bwd_q_rows(const WinArgs& a, WinSeqs s, cudaStream_t stream) {
    using SM = Fp32Smem<DH, R, 2, 1>;
    static PerDeviceOnce once;
    if (!raise_limit(window_bwd_q_fp32_kernel<DH, R>, once, SM())) return -1;
    window_bwd_q_fp32_kernel<DH, R><<<dim3(retile(s, a.batch, s.q_len, R), a.Hq), kThreads, SM::kBytes, stream>>>(a, s);
    return 1;
}
template <int DH, int R>
int bwd_kv_rows(const WinArgs& a, WinSeqs s, cudaStream_t stream) {
    using SM = Fp32Smem<DH, R, 2, 2>;
    static PerDeviceOnce once;
    if (!raise_limit(window_bwd_kv_fp32_kernel<DH, R>, once, SM())) return -1;
    retile(s, a.batch, s.kv_len, R);
    for (int b = 0, parts = 0; b < a.batch; ++b) {
        parts += ((a.sinks < s.kv_len[b] ? a.sinks : s.kv_len[b]) + R - 1) / R * s.segs[b];
        s.item[b + 1] += parts;
    }
    window_bwd_kv_fp32_kernel<DH, R><<<dim3(s.item[a.batch], a.Hq), kThreads, SM::kBytes, stream>>>(a, s);
    return 1;
}

template <int DH>
int fwd(const WinArgs& a, WinSeqs s, cudaStream_t stream) {
    return small_rows(s, a.batch, s.q_len, a.Hq) ? fwd_rows<DH, 32>(a, s, stream) : fwd_rows<DH, 64>(a, s, stream);
}

template <int DH>
int bwd(const WinArgs& a, WinSeqs s, cudaStream_t stream) {
    int launched = 0, rc = 0;
    if (retile(s, a.batch, s.q_len, 64) > 0) {
        rc = small_rows(s, a.batch, s.q_len, a.Hq) ? bwd_q_rows<DH, 32>(a, s, stream) : bwd_q_rows<DH, 64>(a, s, stream);
        if (rc < 0) return rc;
        launched += rc;
    }
    if (retile(s, a.batch, s.kv_len, 64) > 0) {
        rc = small_rows(s, a.batch, s.kv_len, a.Hq) ? bwd_kv_rows<DH, 32>(a, s, stream) : bwd_kv_rows<DH, 64>(a, s, stream);
        if (rc < 0) return rc;
        launched += rc;
        if (a.G > 1) {
            const long long rows = (long long)s.k_start[a.batch - 1] + s.kv_len[a.batch - 1], n = rows * a.Hkv * 2 * DH;
            const long long ctas = (n + 255) / 256, fit = device_sm_count() * 8;
            window_group_join_fp32_kernel<<<dim3((unsigned)(ctas < fit ? ctas : fit)), 256, 0, stream>>>(a, DH, rows);
            ++launched;
        }
        if (a.sink_rows > 0) {           // (over what the join of the groups left in the sinks' rows)
            window_sink_join_fp32_kernel<<<dim3(a.sink_rows, a.Hkv, a.batch), 256, 0, stream>>>(a, s, DH);
            ++launched;
        }
    }
    return launched;
}

}  // namespace

int window_fwd_fp32(const WinArgs& a, const WinSeqs& s, int dh, cudaStream_t stream) {
    return dh == 128 ? fwd<128>(a, s, stream) : dh == 64 ? fwd<64>(a, s, stream) : dh == 32 ? fwd<32>(a, s, stream) : fwd<16>(a, s, stream);
}
int window_bwd_fp32(const WinArgs& a, const WinSeqs& s, int dh, cudaStream_t stream) {
    return dh == 128 ? bwd<128>(a, s, stream) : dh == 64 ? bwd<64>(a, s, stream) : dh == 32 ? bwd<32>(a, s, stream) : bwd<16>(a, s, stream);
}

}  // namespace beagle
