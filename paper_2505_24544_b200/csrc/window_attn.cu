// Entry points of the windowed attention over whole sequences: host-side checks, workspace layout and launch choice.
#include <cstring>

#include "tensor_map.h"
#include "window_attn.h"

using namespace beagle;

namespace {

struct Layout {
    size_t stats, part, group, split, total;
    int stat_rows, sink_rows, splits;
};

constexpr int kMaxSinks = 1024;          // with a window
constexpr long long kMaxRows = 1 << 27;
constexpr int kMaxSegs = 64;             // segments of the queries past the sinks' band
constexpr size_t kSmallParts = 4 << 20;

// Everything that does not depend on device pointers.  Fills `s` and the shape part of `a`; rows of queries and keys in total.
beagle_status check(const beagle_window_attn* w, WinArgs& a, WinSeqs& s, long long& q_rows, long long& k_rows) {
    if (w == nullptr) return BEAGLE_ERR_INVALID_ARG;
    if (w->dtype != BEAGLE_FP32 && w->dtype != BEAGLE_BF16) return BEAGLE_ERR_INVALID_ARG;
    if (w->n_q_heads <= 0 || w->n_kv_heads <= 0 || w->batch < 0 || w->window < 0 || w->sinks < 0) return BEAGLE_ERR_INVALID_ARG;
    if (w->strict != 0 && w->strict != 1) return BEAGLE_ERR_INVALID_ARG;
    if (w->n_q_heads % w->n_kv_heads || w->n_q_heads > 65535) return BEAGLE_ERR_SHAPE;
    const int d = w->head_dim;
    if (!(d == 64 || d == 128 || (w->dtype == BEAGLE_FP32 && (d == 16 || d == 32)))) return BEAGLE_ERR_SHAPE;
    if (w->batch > kMaxCallBatch) return BEAGLE_ERR_CAPACITY;
    if (w->batch > 0 && (w->q_len_host == nullptr || w->kv_len_host == nullptr)) return BEAGLE_ERR_INVALID_ARG;
    if (w->window > 0 && w->sinks > kMaxSinks) return BEAGLE_ERR_CAPACITY;
    memset(&a, 0, sizeof(a));
    memset(&s, 0, sizeof(s));
    q_rows = k_rows = 0;
    for (int b = 0; b < w->batch; ++b) {
        if (w->q_len_host[b] < 0 || w->kv_len_host[b] < 0) return BEAGLE_ERR_INVALID_ARG;
        s.q_start[b] = (int)q_rows;
        s.k_start[b] = (int)k_rows;
        s.q_len[b] = w->q_len_host[b];
        s.kv_len[b] = w->kv_len_host[b];
        q_rows += s.q_len[b];
        k_rows += s.kv_len[b];
        if (q_rows > kMaxRows || k_rows > kMaxRows) return BEAGLE_ERR_CAPACITY;
        s.item[b + 1] = s.item[b] + (s.q_len[b] + kQTile - 1) / kQTile;
    }
    a.batch = w->batch;
    a.Hq = w->n_q_heads; a.Hkv = w->n_kv_heads; a.G = w->n_q_heads / w->n_kv_heads;
    a.window = w->window > 0 && w->window < kNoWindow ? w->window : kNoWindow;
    a.sinks = a.window == kNoWindow ? 0 : w->sinks;      // without a window every earlier key is visible anyway
    a.strict = w->strict;
    a.scale = 1.f / sqrtf((float)d);
    a.scale_log2 = 1.4426950408889634f * a.scale;
    return BEAGLE_OK;
}

// Also fills the sequences' segments and their places in the sinks' partials.
Layout layout(const beagle_window_attn* w, const WinArgs& a, WinSeqs& s, long long k_rows) {
    Layout L;
    memset(&L, 0, sizeof(L));
    long long rows = kStatPad;           // a tile that starts inside the last sequence may read past its padded end
    int most_kv = 0;
    for (int b = 0; b < a.batch; ++b) {
        rows += (s.q_len[b] + kStatPad - 1) / kStatPad * kStatPad;
        most_kv = s.kv_len[b] > most_kv ? s.kv_len[b] : most_kv;
    }
    L.stat_rows = (int)rows;
    size_t off = ((size_t)a.Hq * rows * 2 * sizeof(float) + 255) / 256 * 256;
    const size_t d = w->head_dim;
    const bool fp32 = w->dtype == BEAGLE_FP32;
    if (fp32 && a.G > 1) {
        L.group = off;
        off += ((size_t)k_rows * a.Hq * 2 * d * sizeof(float) + 255) / 256 * 256;
    }
    L.part = off;
    // Jobs (128 queries of one head) past the band of a sequence's first key tile, and of a key tile's band at most.
    auto past = [&](int b) -> long long {
        if (a.sinks == 0 || s.kv_len[b] == 0) return 0;
        const long long shift = s.kv_len[b] - s.q_len[b] - a.strict;
        long long end = (s.kv_len[b] < kKTile ? s.kv_len[b] : kKTile) - 1 - shift + a.window;
        end = end < 0 ? 0 : end > s.q_len[b] ? s.q_len[b] : end;
        return s.q_len[b] == end ? 0 : (s.q_len[b] - end + kQTile) / kQTile * (fp32 ? 1 : a.G);        // (the fp32 kernels: a CTA per head)
    };
    auto rows_of = [&](int b) { return a.sinks < s.kv_len[b] ? a.sinks : s.kv_len[b]; };
    long long band = ((long long)a.window + 2 * kKTile) / kQTile * (fp32 ? 1 : a.G);
    L.splits = 1;
    if (band < (fp32 ? 2 : 8)) band = fp32 ? 2 : 8;
    if (!fp32) {
        // Few key tiles with many jobs each: several CTAs share a tile's jobs, with as few jobs each (two at least) as leave every
        // CTA, those of the sinks' segments among them, an SM of its own.  (Backward, 8 heads of 128 over one K/V head, 1000 queries:
        // 127 us unshared, 52 so; 8 x 200, 16 heads over 2, window 9: 57 and 45; below eight jobs a tile the join costs what it saves.)
        long long tiles = 0, jobs = 0, late[kMaxCallBatch];
        for (int b = 0; b < a.batch; ++b) {
            const long long span = (long long)a.window + 2 * kKTile < s.q_len[b] ? (long long)a.window + 2 * kKTile : s.q_len[b];
            const long long n = (span + kQTile - 1) / kQTile * a.G;
            jobs = n > jobs ? n : jobs;
            late[b] = past(b);
            tiles += (s.kv_len[b] + kKTile - 1) / kKTile;
        }
        const long long units = tiles * a.Hkv, sms = device_sm_count();
        if (units * 2 <= sms && jobs >= 8) {
            long long each = 2;
            auto ctas = [&]() {
                long long n = units * ((jobs + each - 1) / each);
                for (int b = 0; b < a.batch; ++b) n += (late[b] + each - 1) / each * ((rows_of(b) + kKTile - 1) / kKTile) * a.Hkv;
                return n;
            };
            while (each < jobs && ctas() > sms) ++each;
            const long long n = (jobs + each - 1) / each;
            L.splits = (int)(n < 16 ? n : 16);
            if (L.splits > 1) band = each;
        }
        if (L.splits > 1) {
            L.split = off;
            off += (size_t)units * L.splits * kKTile * 2 * d * sizeof(float);
            L.part = off;
        }
    }
    // Segments of the queries past the band of the sinks' key tiles, about as long as a band CTA's work (at least eight jobs where
    // the tiles are not shared, fp32 two).  A sequence takes as many as it needs itself: one long sequence among short ones, or more sinks
    // than the others have keys, costs only its own partials.
    const long long heads = fp32 ? a.Hq : a.Hkv;
    long long parts = 0;
    int most_segs = 0, most_rows = a.sinks < most_kv ? a.sinks : most_kv;
    for (int b = 0; b < a.batch; ++b) {
        const long long need = (past(b) + band - 1) / band;
        s.segs[b] = (int)(need < kMaxSegs ? need : kMaxSegs);
        s.part[b] = parts;
        if (s.segs[b] == 0) continue;
        parts += heads * (1 + s.segs[b]) * rows_of(b);
        most_segs = s.segs[b] > most_segs ? s.segs[b] : most_segs;
        L.sink_rows = rows_of(b) > L.sink_rows ? rows_of(b) : L.sink_rows;
    }
    if (parts > 0) {
        // (Up to 4 MB every sequence is given what the largest takes: the size of small calls does not follow each length.)
        const size_t row = 2 * d * sizeof(float), even = (size_t)a.batch * heads * (1 + most_segs) * most_rows * row, own = parts * row;
        off += own > kSmallParts ? own : even < kSmallParts ? even : kSmallParts;
    }
    L.total = (off + 255) / 256 * 256;
    return L;
}

bool row_ok(const void* p, int64_t stride, int64_t width, int elt) {
    return p != nullptr && !((uintptr_t)p & 15) && stride >= width && (stride * elt) % 16 == 0;
}

}  // namespace

extern "C" {

beagle_status beagle_window_attn_forward(const beagle_window_attn* w, void* out_dev, float* lse_dev, void* stream) {
    WinArgs a;
    WinSeqs s;
    long long q_rows, k_rows;
    const beagle_status st = check(w, a, s, q_rows, k_rows);
    if (st != BEAGLE_OK || q_rows == 0) return st;
    const int e = w->dtype == BEAGLE_BF16 ? 2 : 4;
    const int64_t qw = (int64_t)w->n_q_heads * w->head_dim, kw = (int64_t)w->n_kv_heads * w->head_dim;
    if (!row_ok(w->q_dev, w->q_stride, qw, e) || !row_ok(out_dev, qw, qw, e) || ((uintptr_t)lse_dev & 3)) return BEAGLE_ERR_INVALID_ARG;
    if (k_rows > 0 && (!row_ok(w->k_dev, w->k_stride, kw, e) || !row_ok(w->v_dev, w->v_stride, kw, e))) return BEAGLE_ERR_INVALID_ARG;
    a.q = w->q_dev; a.k = w->k_dev; a.v = w->v_dev;
    a.q_stride = w->q_stride; a.k_stride = w->k_stride; a.v_stride = w->v_stride;
    a.o = out_dev;
    a.lse_out = lse_dev;
    const cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const int rc = w->dtype == BEAGLE_BF16 ? window_fwd_bf16(a, s, w->head_dim, q_rows, k_rows, cs) : window_fwd_fp32(a, s, w->head_dim, cs);
    return rc >= 0 && cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

beagle_status beagle_window_attn_workspace_bytes(const beagle_window_attn* w, size_t* bytes) {
    WinArgs a;
    WinSeqs s;
    long long q_rows, k_rows;
    if (bytes == nullptr) return BEAGLE_ERR_INVALID_ARG;
    const beagle_status st = check(w, a, s, q_rows, k_rows);
    if (st != BEAGLE_OK) return st;
    *bytes = layout(w, a, s, k_rows).total;
    return BEAGLE_OK;
}

beagle_status beagle_window_attn_backward(const beagle_window_attn* w, const void* out_dev, const float* lse_dev, const void* dout_dev, int64_t dout_stride,
                                          void* dq_dev, int64_t dq_stride, void* dk_dev, int64_t dk_stride, void* dv_dev, int64_t dv_stride,
                                          void* ws_dev, size_t ws_bytes, void* stream) {
    WinArgs a;
    WinSeqs s;
    long long q_rows, k_rows;
    const beagle_status st = check(w, a, s, q_rows, k_rows);
    if (st != BEAGLE_OK || (q_rows == 0 && k_rows == 0)) return st;
    const int e = w->dtype == BEAGLE_BF16 ? 2 : 4;
    const int64_t qw = (int64_t)w->n_q_heads * w->head_dim, kw = (int64_t)w->n_kv_heads * w->head_dim;
    if (q_rows > 0 && (!row_ok(w->q_dev, w->q_stride, qw, e) || !row_ok(out_dev, qw, qw, e) || !row_ok(dout_dev, dout_stride, qw, e) ||
                       !row_ok(dq_dev, dq_stride, qw, e) || lse_dev == nullptr || ((uintptr_t)lse_dev & 3)))
        return BEAGLE_ERR_INVALID_ARG;
    if (k_rows > 0 && (!row_ok(w->k_dev, w->k_stride, kw, e) || !row_ok(w->v_dev, w->v_stride, kw, e) || !row_ok(dk_dev, dk_stride, kw, e) ||
                       !row_ok(dv_dev, dv_stride, kw, e)))
        return BEAGLE_ERR_INVALID_ARG;
    if (ws_dev == nullptr || ((uintptr_t)ws_dev & 255)) return BEAGLE_ERR_INVALID_ARG;
    const Layout L = layout(w, a, s, k_rows);
    if (ws_bytes < L.total) return BEAGLE_ERR_CAPACITY;
    a.q = w->q_dev; a.k = w->k_dev; a.v = w->v_dev; a.out = out_dev; a.dout = dout_dev;
    a.lse = lse_dev;
    a.q_stride = w->q_stride; a.k_stride = w->k_stride; a.v_stride = w->v_stride;
    a.dout_stride = dout_stride; a.dq_stride = dq_stride; a.dk_stride = dk_stride; a.dv_stride = dv_stride;
    a.dq = dq_dev; a.dk = dk_dev; a.dv = dv_dev;
    a.stats = reinterpret_cast<float*>(static_cast<char*>(ws_dev) + L.stats);
    a.sink_part = reinterpret_cast<float*>(static_cast<char*>(ws_dev) + L.part);
    a.group_part = reinterpret_cast<float*>(static_cast<char*>(ws_dev) + L.group);
    a.split_part = reinterpret_cast<float*>(static_cast<char*>(ws_dev) + L.split);
    a.splits = L.splits;
    a.stat_rows = L.stat_rows; a.sink_rows = L.sink_rows;
    const cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const int rc = w->dtype == BEAGLE_BF16 ? window_bwd_bf16(a, s, w->head_dim, q_rows, k_rows, cs) : window_bwd_fp32(a, s, w->head_dim, cs);
    return rc >= 0 && cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

}  // extern "C"
