// Attention over a paged key/value cache: arguments, and how the visible tiles are divided among thread blocks on the device, where the
// lengths are.  Shared by the one-token kernels (paged_attn.cu) and the common part of groups of rows (paged_grouped.cu).
#pragma once
#include "pages.h"

namespace beagle {

constexpr int kTile = 64;               // cached positions per tile
constexpr float kSlack = 8.f;           // how far (log2) a score may exceed the row's reference point before it moves
constexpr float kLn2 = 0.6931471805599453f;

// What the join does for a run: the pair that begins in it and ends in a later one, if there is one.
struct JoinItem { int pair, last_run, second, total; };          // pair: b * Hkv + kvh or -1; second: it is the run's second partial; all tiles
struct PagedArgs {
    static constexpr bool kShared = false;
    static constexpr int kEntries = kMaxCallBatch;
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

// beagle_paged_attn_shared: what is walked are entries instead of the call's rows.  An entry is up to eight query rows (of the grouped
// heads and of several rows of the call) that read the same positions of the same slot: the common part of a group for eight of its rows
// times grouped heads, or what a row has behind it.
struct SharedEntry {
    uint8_t row0;                       // row of the call whose slot is read; the query rows count from its first grouped head
    uint8_t group;                      // 255: a group of one row, all of it is read as the row's own
    uint8_t prefix;                     // 1: the common part, 0: what lies behind it
    uint8_t n;                          // query rows
    uint16_t j0;                        // first one: query row j is row row0 + j / G, grouped head j % G
};
struct SharedArgs : PagedArgs {         // `batch` counts the entries
    static constexpr bool kShared = true;
    static constexpr int kEntries = 2 * kMaxCallBatch;
    const int32_t* shared;
    int2* span;                         // [n_pairs] first and last run that worked on a pair (first > last: none), in the workspace
    int rows, n_groups, n_pairs;        // rows of the call; entries * Hkv
    SharedEntry entry[kEntries];
    uint8_t group_of[kMaxCallBatch];    // of a row; 255 as above
    uint8_t prefix_entry[kMaxCallBatch];        // first entry of a group's common part (the rows' own entries have the rows' numbers)
    uint8_t group_row0[kMaxCallBatch];
    int block;                          // query rows of a common part's entry
    int split;                          // partials that a run leaves of a pair: one of each consumer warp on mma.sync, else 1
};

// How the visible tiles are divided; computed by every CTA from the lengths (64 values at most).
template <int N>
struct ScheduleOf {
    int len[N];             // positions of the sequence
    int lo[N];              // first position of the window (0: everything is visible)
    int sink_tiles[N];      // tiles in front of the window's first one
    int first[N];           // first tile of the window
    int start[N + 1];       // prefix sum of (tiles * Hkv)
};
typedef ScheduleOf<kMaxCallBatch> Schedule;

template <int N>
__device__ __forceinline__ int tiles_of(const ScheduleOf<N>& s, int b, int Hkv) { return (s.start[b + 1] - s.start[b]) / Hkv; }
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

// The same for the entries, of up to two sets over the same rows (`b` may be `a`: one set); whole CTA of at least 128 threads, barriers
// inside.  The common part of a group: shared_dev, not above its shortest length, in whole tiles.
__device__ __forceinline__ void build_schedules(const SharedArgs& a, ScheduleOf<SharedArgs::kEntries>& sa, const SharedArgs& b, ScheduleOf<SharedArgs::kEntries>& sb) {
    __shared__ int s_len[kMaxCallBatch], s_common[kMaxCallBatch], s_warp[2][4];
    const int t = threadIdx.x, lane = t & 31;
    int n = 0;
    if (t < a.rows) n = min(max(__ldcg(a.length + a.slots.slot[t]), 0), a.max_pages << a.page_shift);
    if (t < a.n_groups) s_common[t] = max(__ldcg(a.shared + t), 0);
    __syncthreads();
    if (t < a.rows) {
        s_len[t] = n;
        if (a.group_of[t] != 255) atomicMin(&s_common[a.group_of[t]], n);
    }
    __syncthreads();
    const bool two = &a != &b;
    int incl[2] = {0, 0};
    if (t < SharedArgs::kEntries) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const SharedArgs& y = x ? b : a;
            ScheduleOf<SharedArgs::kEntries>& s = x ? sb : sa;
            if (t < y.batch && (x == 0 || two)) {
                const SharedEntry e = y.entry[t];
                const int common = e.group == 255 ? 0 : s_common[e.group] / kTile * kTile;
                const int len = e.prefix ? common : s_len[e.row0], lo = e.prefix ? 0 : common;
                s.len[t] = len; s.lo[t] = lo; s.first[t] = lo / kTile; s.sink_tiles[t] = 0;
                incl[x] = ((len + kTile - 1) / kTile - lo / kTile) * y.Hkv;
            }
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int v = __shfl_up_sync(0xffffffffu, incl[x], o);
                if (lane >= o) incl[x] += v;
            }
        if (lane == 31) { s_warp[0][t >> 5] = incl[0]; s_warp[1][t >> 5] = incl[1]; }
    }
    __syncthreads();
    if (t < SharedArgs::kEntries) {
        for (int i = 0; i < t >> 5; ++i) { incl[0] += s_warp[0][i]; incl[1] += s_warp[1][i]; }
        sa.start[t + 1] = incl[0];
        if (t == 0) sa.start[0] = 0;
        if (two) {
            sb.start[t + 1] = incl[1];
            if (t == 0) sb.start[0] = 0;
        }
    }
    __syncthreads();
}
__device__ __forceinline__ void build_schedule(const SharedArgs& a, ScheduleOf<SharedArgs::kEntries>& s) { build_schedules(a, s, a, s); }
__device__ __forceinline__ void build_schedule(const PagedArgs& a, Schedule& s) {
    make_schedule(a, s);
    __syncthreads();
    finish_schedule(s);
    __syncthreads();
}

// Where query row g of pair (b, kvh) lies, in heads: row of the call * stride, head.
__device__ __forceinline__ int rows_of(const PagedArgs& a, int) { return a.G; }
__device__ __forceinline__ int rows_of(const SharedArgs& a, int b) { return a.entry[b].n; }
__device__ __forceinline__ int slot_of(const PagedArgs& a, int b) { return a.slots.slot[b]; }
__device__ __forceinline__ int slot_of(const SharedArgs& a, int b) { return a.slots.slot[a.entry[b].row0]; }
__device__ __forceinline__ size_t query_at(const PagedArgs& a, int b, int kvh, int g, int dh) { return (size_t)b * a.q_stride + (size_t)(kvh * a.G + g) * dh; }
__device__ __forceinline__ size_t query_at(const SharedArgs& a, int b, int kvh, int g, int dh) {
    const int j = a.entry[b].j0 + g, r = j / a.G;
    return (size_t)(a.entry[b].row0 + r) * a.q_stride + (size_t)(kvh * a.G + j - r * a.G) * dh;
}

// Walks the units [u, end) of one run: for every tile the pair (b, kvh), the tile's first position and whether the pair ends.
struct Walk {
    int b, kvh, i, n;                   // sequence, K/V head, tile index inside the pair, tiles of the pair
    template <int N>
    __device__ __forceinline__ void seek(const ScheduleOf<N>& s, int unit, int Hkv) {          // whole warps
        const int lane = threadIdx.x & 31;
        b = 0;
#pragma unroll
        for (int x = 1; x <= N; x += 32) b += __popc(__ballot_sync(0xffffffffu, s.start[lane + x] <= unit));
        n = tiles_of(s, b, Hkv);
        const int in = unit - s.start[b];
        kvh = in / n;
        i = in - kvh * n;
    }
    template <int N>
    __device__ __forceinline__ void next(const ScheduleOf<N>& s, int batch, int Hkv) {
        if (++i < n) return;
        i = 0;
        if (++kvh < Hkv) return;
        kvh = 0;
        do { ++b; } while (b < batch && s.start[b + 1] == s.start[b]);
        if (b < batch) n = tiles_of(s, b, Hkv);
    }
    template <int N>
    __device__ __forceinline__ int tile(const ScheduleOf<N>& s) const { return i < s.sink_tiles[b] ? i : s.first[b] + i - s.sink_tiles[b]; }
};

// The units of run `run` of `count`, never more runs than there are tiles, so that every run between two others has some.  Threads 0 <= t < n
// leave word of which runs work on which pair (shared out over the CTAs of the grid).
__device__ __forceinline__ void begin_shared(const SharedArgs& a, const ScheduleOf<SharedArgs::kEntries>& s, int run, int count, int t, int n_threads, int& u0, int& u1) {
    const int total = s.start[SharedArgs::kEntries];
    const Runs runs(total, max(1, min(total, count)));
    u0 = run >= 0 && run < runs.runs ? runs.begin(run) : 0;
    u1 = run >= 0 && run < runs.runs ? runs.begin(run + 1) : 0;
    if (t < 0) return;
    for (int p = blockIdx.x + gridDim.x * t; p < a.n_pairs; p += gridDim.x * n_threads) {
        const int e = p / a.Hkv, n = tiles_of(s, e, a.Hkv), first = s.start[e] + (p - e * a.Hkv) * n;
        a.span[p] = n > 0 ? make_int2(runs.of(first), runs.of(first + n - 1)) : make_int2(0, -1);
    }
}

// What beagle_paged_attn_shared leaves to the tensor cores: the common parts of groups with many query rows.  `entry` holds blocks of up
// to 128 query rows; part_rows is the largest of them, rounded up to 4: a partial is part_rows rows of O, then their (maximum, sum).
struct PrefixArgs : SharedArgs {
    int part_rows;
    uint8_t on[kMaxCallBatch];           // of a group: its common part is done there
};
beagle_status launch_grouped(const beagle_pages* p, const SharedArgs& rows, const PrefixArgs& prefix, int runs, cudaStream_t stream);
int prefix_block(int G);                 // query rows of a block: whole rows of the call

}  // namespace beagle
