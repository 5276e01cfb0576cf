// Shared pieces of the windowed attention kernels (beagle_window_attn_*).  Internal to the library.
#pragma once
#include "../../include/beagle.h"
#include "common.cuh"

namespace beagle {

// The sequences of one call, by value in the kernel parameters.  Query i of sequence b sees the keys
//     j <= last(i) = i + shift[b]   with   j > last(i) - window   or   j < sinks,     shift = kv_len - q_len - strict.
struct WinSeqs {
    int32_t q_start[kMaxCallBatch], k_start[kMaxCallBatch];      // first packed row
    int32_t q_len[kMaxCallBatch], kv_len[kMaxCallBatch];
    int32_t item[kMaxCallBatch + 1];                             // prefix sum of the launch's tiles per sequence
    int32_t segs[kMaxCallBatch];                                 // backward: segments of the queries past the band of the sinks' key tiles
    long long part[kMaxCallBatch];                               // first row (of 2 DH fp32) of the sequence in WinArgs::sink_part; 0 segments: none
};

struct WinArgs {
    int32_t batch, Hq, Hkv, G, window, sinks, strict;            // window: "none" is kNoWindow
    float scale, scale_log2;
    const void *q, *k, *v, *out, *dout;
    const float* lse;
    long long q_stride, k_stride, v_stride, dout_stride, dq_stride, dk_stride, dv_stride;
    void *o, *dq, *dk, *dv;
    float* lse_out;
    float* stats;                                                // [Hq][2][stat_rows]: -log-sum-exp (log2 units), and -delta, of every query
    float* sink_part;                                            // fp32 partials of the sinks' dK, dV: see sink_row()
    float* split_part;                                           // key side in splits: fp32 [tile][K/V head][split][128][2][DH], dV then dK
    float* group_part;                                           // fp32 kernels: dV, dK of every query head, where heads share keys
    int32_t stat_rows;                                           // sum over the sequences of q_len padded to kStatPad
    int32_t splits;                                              // CTAs that share the jobs of a key tile
    int32_t sink_rows;                                           // the most rows of sinks of a sequence with segments (0: no such sequence)
};
constexpr int kNoWindow = 0x3fffffff;
constexpr int kStatPad = 128;
constexpr int kQTile = 128;              // queries of one tile
constexpr int kKTile = 128;              // keys of one tile of the key side

// Which sequence a linear item belongs to (the item's index inside it in `in`).
__device__ __forceinline__ int win_find(const int32_t* item, int batch, int at, int& in) {
    int b = 0;
    while (b + 1 < batch && at >= item[b + 1]) ++b;
    in = at - item[b];
    return b;
}

// Row of sequence b's key `key` < min(sinks, kv_len) in WinArgs::sink_part: [head][1 + segments][min(sinks, kv_len)] a sequence, part 0 the
// band's; dV, then dK in a row.  head: K/V head (bf16), query head (fp32).
__device__ __forceinline__ size_t sink_row(const WinArgs& a, const WinSeqs& s, int b, int head, int part, int key) {
    return (size_t)s.part[b] + ((size_t)head * (1 + s.segs[b]) + part) * min(a.sinks, s.kv_len[b]) + key;
}

// 32-bit visibility of columns [0, 32) of a chunk: bits [lo, hi).
__device__ __forceinline__ uint32_t bit_range(int lo, int hi) {
    lo = max(lo, 0);
    hi = min(hi, 32);
    if (hi <= lo) return 0u;
    return (0xffffffffu >> (32 - (hi - lo))) << lo;
}

// host side
int window_fwd_bf16(const WinArgs& a, const WinSeqs& s, int dh, long long q_rows, long long k_rows, cudaStream_t stream);
int window_bwd_bf16(const WinArgs& a, const WinSeqs& s, int dh, long long q_rows, long long k_rows, cudaStream_t stream);
int window_fwd_fp32(const WinArgs& a, const WinSeqs& s, int dh, cudaStream_t stream);
int window_bwd_fp32(const WinArgs& a, const WinSeqs& s, int dh, cudaStream_t stream);

}  // namespace beagle
