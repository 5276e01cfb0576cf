// Bookkeeping and data movement of a paged key/value cache (beagle_pages_* of include/beagle.h).
//
// All state lies in device memory (page table, lengths, reference counts), so that every call can be captured into a graph and
// a length that only the device knows (the accepted drafts of a verification) never travels to the host.  A call is one
// bookkeeping launch and, where rows or pages move, one dependent launch that moves them: the bookkeeping is a few thousand
// integers (one CTA, one pass over the reference counts in order, so that pages are taken lowest id first), the movement is
// bound by memory bandwidth (16-byte loads and stores, four in flight per thread).
//
// Measured: prompts of up to 8192 tokens for 8 sequences (370 MB moved) 64 us, book-keeping before it 6; copy of 16 serving
// sequences 63 us (6.5 TB/s), its book-keeping 9.
//
// Every index that comes from device memory (table entries, lengths, counts) is clamped or range-checked before it is used, so
// a damaged table yields wrong contents but no access outside the caller's buffers.
#include <cstring>

#include "pages.h"
#include "tensor_map.h"

using namespace beagle;

namespace beagle {

bool pages_valid_shape(const beagle_pages* p) {
    if (p->dtype != BEAGLE_FP32 && p->dtype != BEAGLE_BF16) return false;
    const int d = p->head_dim;
    const bool dim_ok = p->dtype == BEAGLE_BF16 ? (d == 32 || d == 64 || d == 128 || d == 256) : (d == 16 || d == 32 || d == 64 || d == 128);
    const int s = p->page_size;
    return dim_ok && s >= 8 && s <= 256 && (s & (s - 1)) == 0;
}

beagle_status pages_check(const beagle_pages* p) {
    if (p == nullptr) return BEAGLE_ERR_INVALID_ARG;
    if (p->k == nullptr || p->v == nullptr || p->table == nullptr || p->length == nullptr || p->refs == nullptr || p->ws == nullptr)
        return BEAGLE_ERR_INVALID_ARG;
    if (p->n_pages <= 0 || p->n_kv_heads <= 0 || p->max_slots <= 0 || p->max_pages <= 0) return BEAGLE_ERR_INVALID_ARG;
    if (!pages_valid_shape(p)) return p->dtype != BEAGLE_FP32 && p->dtype != BEAGLE_BF16 ? BEAGLE_ERR_INVALID_ARG : BEAGLE_ERR_SHAPE;
    // rows of the pools and entries of the table are counted in 32 bits (their byte offsets are not)
    if ((long long)p->n_pages * p->n_kv_heads * p->page_size > 0x7fffffffll || (long long)p->max_slots * p->max_pages > 0x7fffffffll ||
        (long long)p->max_pages * p->page_size > 0x3fffffffll || p->n_kv_heads > 65535)
        return BEAGLE_ERR_CAPACITY;
    if (((uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->refs | (uintptr_t)p->ws) & 15) return BEAGLE_ERR_INVALID_ARG;
    if (((uintptr_t)p->table | (uintptr_t)p->length) & 3) return BEAGLE_ERR_INVALID_ARG;
    size_t need = 0;
    beagle_pages_workspace_bytes(p, &need);
    return p->ws_bytes < need ? BEAGLE_ERR_CAPACITY : BEAGLE_OK;
}

// n slots of a call: in range and distinct.
beagle_status pages_check_slots(const beagle_pages* p, int n, const int32_t* slots, PageSlots* out) {
    if (n < 0 || (n > 0 && slots == nullptr)) return BEAGLE_ERR_INVALID_ARG;
    if (n > kMaxCallBatch) return BEAGLE_ERR_CAPACITY;
    for (int i = 0; i < n; ++i) {
        if (slots[i] < 0 || slots[i] >= p->max_slots) return BEAGLE_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (slots[j] == slots[i]) return BEAGLE_ERR_INVALID_ARG;
        out->slot[i] = slots[i];
    }
    return BEAGLE_OK;
}

namespace {

constexpr int kBookThreads = 1024;
constexpr int kScanPer = 16;                     // reference counts per thread and scan step: a step covers 16384 pages
constexpr int kMoveThreads = 256;
constexpr int kMoveVecs = 4;                     // 16-byte pieces a thread keeps in flight

// What one append does to one of its rows, handed from the bookkeeping to the launch that writes.
struct AppendRow {
    int32_t len;        // positions before the call
    int32_t n;          // rows written
    int32_t cow_src, cow_dst;   // last page copied before it is written, or -1
};

// Layout of the call workspace (beagle_pages_workspace_bytes): header, the append's rows, three lists of n_pages.
struct BookWs {
    int32_t* header;    // [0] pages to move, [1] live pages
    AppendRow* rows;    // [64]
    int32_t* src;       // [n_pages] page to read of every move
    int32_t* dst;       // [n_pages] page to write
    int32_t* map;       // [n_pages] new id of a moved page
};
constexpr size_t kBookHead = 256 + (size_t)kMaxCallBatch * sizeof(AppendRow);

__host__ __device__ inline BookWs book_ws(void* ws, int n_pages) {
    BookWs b;
    char* base = static_cast<char*>(ws);
    b.header = reinterpret_cast<int32_t*>(base);
    b.rows = reinterpret_cast<AppendRow*>(base + 256);
    b.src = reinterpret_cast<int32_t*>(base + kBookHead);
    b.dst = b.src + n_pages;
    b.map = b.dst + n_pages;
    return b;
}

struct Book {               // the device pointers of beagle_pages, by value
    int32_t *table, *length, *refs;
    void* ws;
    int n_pages, page_size, max_pages;
    __device__ int32_t* row(int slot) const { return table + (size_t)slot * max_pages; }
    __device__ int clamp_len(int n) const { return min(max(n, 0), max_pages * page_size); }
    __device__ bool page_ok(int id) const { return id >= 0 && id < n_pages; }
};

// Exclusive sum over the CTA's threads; `total` for every thread.  s_warp: 33 words.
__device__ __forceinline__ int block_scan(int v, int* s_warp, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    __syncthreads();                             // the previous scan's words have been read
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int w = lane < warps ? s_warp[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    total = s_warp[warps - 1];
    return incl - v + (warp > 0 ? s_warp[warp - 1] : 0);
}

// The reference counts of ids [id0, id0 + 16), -1 past the end.
__device__ __forceinline__ void load_refs(const int32_t* refs, int id0, int n_pages, int* r) {
    if (id0 + kScanPer <= n_pages) {
#pragma unroll
        for (int i = 0; i < kScanPer; i += 4) {
            const int4 t = __ldcg(reinterpret_cast<const int4*>(refs + id0 + i));
            r[i] = t.x; r[i + 1] = t.y; r[i + 2] = t.z; r[i + 3] = t.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kScanPer; ++i) r[i] = id0 + i < n_pages ? __ldcg(refs + id0 + i) : -1;
    }
}

constexpr int kNear = 4096;                      // entries of the page list that fit shared memory

// The first `want` free pages, lowest id first, into list[]; returns how many there are (at most want).  `r`: this thread's counts
// of the first step, loaded beforehand.  Whole CTA.
__device__ __forceinline__ int find_free(const Book& b, int want, int32_t* list, int* s_warp, int* r) {
    int found = 0;
    for (int base = 0; base < b.n_pages && found < want; base += kBookThreads * kScanPer) {
        const int id0 = base + threadIdx.x * kScanPer;
        int mine = 0, total;
        if (base > 0) load_refs(b.refs, id0, b.n_pages, r);
#pragma unroll
        for (int i = 0; i < kScanPer; ++i) mine += r[i] == 0;
        int at = found + block_scan(mine, s_warp, total);
        if (mine > 0) {
#pragma unroll
            for (int i = 0; i < kScanPer; ++i)
                if (r[i] == 0) {
                    if (at < want) list[at] = id0 + i;
                    ++at;
                }
        }
        found += total;
    }
    return min(found, want);
}

// Gives back the pages of `row`.  One warp, four entries a lane in flight.
__device__ __forceinline__ void release_row(const Book& b, int32_t* row, int lane) {
    for (int j = lane; j < b.max_pages; j += 128) {
        int id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) id[u] = j + 32 * u < b.max_pages ? __ldcg(row + j + 32 * u) : -1;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (b.page_ok(id[u])) atomicSub(b.refs + id[u], 1);
            if (id[u] != -1) row[j + 32 * u] = -1;
        }
    }
}

__global__ void __launch_bounds__(kBookThreads) pages_append_book_kernel(const Book b, const __grid_constant__ PageSlots slots,
                                                                        const __grid_constant__ AppendRows rows, int batch, const int32_t* n_new,
                                                                        int32_t* ok_out) {
    __shared__ int s_warp[33];
    __shared__ int s_need[kMaxCallBatch], s_start[kMaxCallBatch], s_have[kMaxCallBatch], s_cow[kMaxCallBatch];
    __shared__ int32_t s_list[kNear];
    const int t = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const BookWs ws = book_ws(b.ws, b.n_pages);
    int refs[kScanPer];
    load_refs(b.refs, t * kScanPer, b.n_pages, refs);    // on their way while the rows are looked up
    AppendRow r = {0, 0, -1, -1};
    int need = 0, want = 0;
    bool fits = true;
    if (t < batch) {
        r.len = b.clamp_len(__ldcg(b.length + slots.slot[t]));
        r.n = n_new != nullptr ? min(max(__ldcg(n_new + t), 0), rows.count[t]) : rows.count[t];
        const int have = (r.len + b.page_size - 1) / b.page_size;
        fits = r.len + r.n <= b.max_pages * b.page_size;
        if (fits && r.n > 0) {
            if (r.len % b.page_size != 0) {              // the last page is partly filled: copied first if someone else holds it too
                const int tail = __ldcg(b.row(slots.slot[t]) + r.len / b.page_size);
                if (b.page_ok(tail) && __ldcg(b.refs + tail) > 1) r.cow_src = tail;
            }
            need = (r.len + r.n + b.page_size - 1) / b.page_size - have + (r.cow_src >= 0 ? 1 : 0);
        }
        s_have[t] = have;
    }
    const int start = block_scan(need, s_warp, want);
    int32_t* list = want <= kNear ? s_list : ws.src;
    const int got = find_free(b, want, list, s_warp, refs);
    __syncthreads();                                     // the list is complete (and, for the atomics below, read in full)
    if (t < batch) {
        const bool ok = fits && (need == 0 || start + need <= got);
        if (!ok) { need = 0; r.n = 0; r.cow_src = -1; }
        if (r.cow_src >= 0) {
            r.cow_dst = list[start];
            b.row(slots.slot[t])[r.len / b.page_size] = r.cow_dst;
            b.refs[r.cow_dst] = 1;
            atomicSub(b.refs + r.cow_src, 1);
        }
        s_need[t] = need; s_start[t] = start; s_cow[t] = r.cow_src >= 0 ? 1 : 0;
        ws.rows[t] = r;
        if (ok && r.n > 0) b.length[slots.slot[t]] = r.len + r.n;
        if (ok_out != nullptr) ok_out[t] = ok ? 1 : 0;
    }
    __syncthreads();
    const int lane = t & 31;
    for (int row = t >> 5; row < batch; row += kBookThreads / 32) {
        int32_t* dst = b.row(slots.slot[row]);
        for (int i = s_cow[row] + lane; i < s_need[row]; i += 32) {
            const int id = list[s_start[row] + i];
            dst[s_have[row] + i - s_cow[row]] = id;
            b.refs[id] = 1;
        }
    }
}

// Rows of the append, and the valid part of every page that is copied before it is written.  blockIdx.y = row of the call;
// blockIdx.x < chunks: that many 16-byte pieces of its new rows (keys, then values); past them: one CTA per K/V head for the copy.
__global__ void __launch_bounds__(kMoveThreads) pages_append_write_kernel(const Book b, const __grid_constant__ PageSlots slots,
                                                                         const __grid_constant__ AppendRows rows, uint4* K, uint4* V, const uint4* k_new,
                                                                         const uint4* v_new, long long k_stride, long long v_stride,
                                                                         int heads, int piece_shift, int chunks) {
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.y;
    const BookWs ws = book_ws(b.ws, b.n_pages);
    const AppendRow r = ws.rows[row];
    const int dv = 1 << piece_shift;                     // 16-byte pieces of one head's row
    if ((int)blockIdx.x >= chunks) {
        const int used = r.len % b.page_size;
        if (!b.page_ok(r.cow_src) || !b.page_ok(r.cow_dst)) return;
        const int h = blockIdx.x - chunks;
        const size_t from = ((size_t)r.cow_src * heads + h) * b.page_size * dv, to = ((size_t)r.cow_dst * heads + h) * b.page_size * dv;
        for (int i = threadIdx.x; i < used * dv; i += kMoveThreads) {
            const uint4 x = K[from + i], y = V[from + i];
            K[to + i] = x;
            V[to + i] = y;
        }
        return;
    }
    const int per_pos = heads << piece_shift;
    const long long pieces = (long long)r.n * per_pos;
    const int32_t* pages = b.row(slots.slot[row]);
    const long long base = (long long)blockIdx.x * (kMoveThreads * kMoveVecs) + threadIdx.x;
    const int shift = __ffs(b.page_size) - 1;
    uint4 x[kMoveVecs], y[kMoveVecs];
    size_t at[kMoveVecs];
#pragma unroll
    for (int u = 0; u < kMoveVecs; ++u) {
        const long long i = base + u * kMoveThreads;
        at[u] = ~(size_t)0;
        if (i < pieces) {
            const int tok = (int)(i / per_pos), off = (int)(i - (long long)tok * per_pos);
            const int h = off >> piece_shift, c = off & (dv - 1);
            const long long srow = rows.start[row] + tok;
            x[u] = __ldcs(k_new + srow * k_stride + off);
            y[u] = __ldcs(v_new + srow * v_stride + off);
            const int pos = r.len + tok;
            const int page = __ldcg(pages + (pos >> shift));
            if (b.page_ok(page)) at[u] = ((((size_t)page * heads + h) << shift) + (pos & (b.page_size - 1))) * dv + c;
        }
    }
#pragma unroll
    for (int u = 0; u < kMoveVecs; ++u)
        if (at[u] != ~(size_t)0) {
            K[at[u]] = x[u];
            V[at[u]] = y[u];
        }
}

__global__ void __launch_bounds__(128) pages_truncate_kernel(const Book b, const PageSlots slots, const int32_t* keep) {
    pdl_launch_dependents();
    pdl_wait();
    const int slot = slots.slot[blockIdx.x];
    const int len = b.clamp_len(__ldcg(b.length + slot));
    const int n = keep != nullptr ? min(max(__ldcg(keep + blockIdx.x), 0), len) : 0;
    int32_t* row = b.row(slot);
    for (int j = (n + b.page_size - 1) / b.page_size + threadIdx.x; j < b.max_pages; j += blockDim.x) {
        const int id = row[j];
        if (b.page_ok(id)) atomicSub(b.refs + id, 1);
        if (id != -1) row[j] = -1;
    }
    __syncthreads();                                     // every thread has read the old length
    if (threadIdx.x == 0) b.length[slot] = n;
}

// dst holds what src holds: the same pages, one more reference each.  Integer atomics: the order does not matter.
__global__ void __launch_bounds__(128) pages_fork_kernel(const Book b, const PageSlots src, const PageSlots dst) {
    pdl_launch_dependents();
    pdl_wait();
    const int32_t* from = b.row(src.slot[blockIdx.x]);
    int32_t* to = b.row(dst.slot[blockIdx.x]);
    for (int j = threadIdx.x; j < b.max_pages; j += blockDim.x) {
        const int old = to[j], id = __ldcg(from + j);
        if (b.page_ok(id)) atomicAdd(b.refs + id, 1);
        if (b.page_ok(old)) atomicSub(b.refs + old, 1);
        if (id != old) to[j] = id;
    }
    if (threadIdx.x == 0) b.length[dst.slot[blockIdx.x]] = b.clamp_len(__ldcg(b.length + src.slot[blockIdx.x]));
}

__global__ void __launch_bounds__(kBookThreads) pages_copy_book_kernel(const Book b, const PageSlots src, const PageSlots dst, int n, int32_t* ok_out) {
    __shared__ int s_warp[33];
    __shared__ int s_need[kMaxCallBatch], s_start[kMaxCallBatch];
    __shared__ int32_t s_list[kNear];
    const int t = threadIdx.x, lane = t & 31;
    pdl_launch_dependents();
    pdl_wait();
    const BookWs ws = book_ws(b.ws, b.n_pages);
    const int len = t < n ? b.clamp_len(__ldcg(b.length + src.slot[t])) : 0;
    for (int i = t >> 5; i < n; i += kBookThreads / 32) release_row(b, b.row(dst.slot[i]), lane);
    __threadfence();
    const int need = (len + b.page_size - 1) / b.page_size;
    int want = 0;
    const int start = block_scan(need, s_warp, want);    // (its barriers: what the destinations held is free now)
    int refs[kScanPer];
    load_refs(b.refs, t * kScanPer, b.n_pages, refs);
    int32_t* list = want <= kNear ? s_list : ws.dst;
    const int got = find_free(b, want, list, s_warp, refs);
    if (t < n) {
        const bool ok = need == 0 || start + need <= got;
        s_need[t] = ok ? need : 0;
        s_start[t] = start;
        b.length[dst.slot[t]] = ok ? len : 0;
        if (ok_out != nullptr) ok_out[t] = ok ? 1 : 0;
    }
    __syncthreads();
    // the rows that fit are the first ones, so the moves are a prefix of the list
    if (t == 0) {
        int moves = 0;
        for (int i = 0; i < n; ++i) moves = s_need[i] > 0 ? s_start[i] + s_need[i] : moves;
        ws.header[0] = moves;
    }
    for (int row = t >> 5; row < n; row += kBookThreads / 32) {
        const int32_t* from = b.row(src.slot[row]);
        int32_t* to = b.row(dst.slot[row]);
        for (int i = lane; i < s_need[row]; i += 128) {
            int page[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) page[u] = i + 32 * u < s_need[row] ? __ldcg(from + i + 32 * u) : -1;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + 32 * u < s_need[row]) {
                    const int at = s_start[row] + i + 32 * u, id = list[at];
                    to[i + 32 * u] = id;
                    b.refs[id] = 1;
                    ws.src[at] = page[u];
                    ws.dst[at] = id;
                }
        }
    }
}

// Live pages get the ids 0 .. live-1: those above move into the holes below, both in ascending order.
__global__ void __launch_bounds__(kBookThreads) pages_compact_book_kernel(const Book b) {
    __shared__ int s_warp[33];
    const int t = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const BookWs ws = book_ws(b.ws, b.n_pages);
    int live = 0, first[kScanPer];                       // this thread's counts of the first step, read once
    load_refs(b.refs, t * kScanPer, b.n_pages, first);
#pragma unroll
    for (int i = 0; i < kScanPer; ++i) live += first[i] > 0;
    for (int base = kBookThreads * kScanPer; base < b.n_pages; base += kBookThreads * kScanPer) {
        int r[kScanPer];
        load_refs(b.refs, base + t * kScanPer, b.n_pages, r);
#pragma unroll
        for (int i = 0; i < kScanPer; ++i) live += r[i] > 0;
    }
    {
        int total;
        block_scan(live, s_warp, total);
        live = total;
    }
    int holes = 0, high = 0;
    for (int base = 0; base < b.n_pages; base += kBookThreads * kScanPer) {
        const int id0 = base + t * kScanPer;
        int r[kScanPer], mine = 0, total;
        if (base > 0) load_refs(b.refs, id0, b.n_pages, r);
        else
#pragma unroll
            for (int i = 0; i < kScanPer; ++i) r[i] = first[i];
        // below `live`: holes; from there on: pages that move.  Both counted in one scan (16 bits would not do: two scans)
#pragma unroll
        for (int i = 0; i < kScanPer; ++i) mine += id0 + i < live && r[i] == 0;
        int at = holes + block_scan(mine, s_warp, total);
        holes += total;
#pragma unroll
        for (int i = 0; i < kScanPer; ++i)
            if (id0 + i < live && r[i] == 0) ws.dst[at++] = id0 + i;
        mine = 0;
#pragma unroll
        for (int i = 0; i < kScanPer; ++i) mine += id0 + i >= live && r[i] > 0;
        at = high + block_scan(mine, s_warp, total);
        high += total;
#pragma unroll
        for (int i = 0; i < kScanPer; ++i)
            if (id0 + i >= live && r[i] > 0) ws.src[at++] = id0 + i;
    }
    __syncthreads();
    const int moves = min(holes, high);                  // equal unless a count was negative
    for (int i = t; i < moves; i += kBookThreads) {
        const int from = ws.src[i], to = ws.dst[i];
        ws.map[from] = to;
        b.refs[to] = __ldcg(b.refs + from);
        b.refs[from] = 0;
    }
    if (t == 0) { ws.header[0] = moves; ws.header[1] = live; }
}

// The listed page moves (keys and values), a grid-stride walk over pieces of 16 KB or a page, whichever is smaller; with
// `remap` also the new ids of moved pages in the table.
__global__ void __launch_bounds__(kMoveThreads) pages_move_kernel(const Book b, uint4* K, uint4* V, int page_vecs, int remap, int table_entries) {
    pdl_launch_dependents();
    pdl_wait();
    const BookWs ws = book_ws(b.ws, b.n_pages);
    const int moves = min(max(__ldcg(ws.header), 0), b.n_pages);
    if (moves == 0) return;
    if (remap) {
        const int live = __ldcg(ws.header + 1);
        for (long long i = (long long)blockIdx.x * kMoveThreads + threadIdx.x; i < table_entries; i += (long long)gridDim.x * kMoveThreads) {
            const int id = b.table[i];
            if (id >= live && id < b.n_pages) b.table[i] = __ldcg(ws.map + id);
        }
    }
    constexpr int kChunk = kMoveThreads * kMoveVecs;
    const int chunks = (page_vecs + kChunk - 1) / kChunk;
    const long long total = (long long)moves * 2 * chunks;
    for (long long w = blockIdx.x; w < total; w += gridDim.x) {
        const int move = (int)(w / (2 * chunks)), rest = (int)(w % (2 * chunks));
        uint4* pool = rest >= chunks ? V : K;
        const int c0 = (rest >= chunks ? rest - chunks : rest) * kChunk + threadIdx.x;
        const int from = __ldcg(ws.src + move), to = __ldcg(ws.dst + move);
        if (!b.page_ok(from) || !b.page_ok(to)) continue;
        const uint4* s = pool + (size_t)from * page_vecs;
        uint4* d = pool + (size_t)to * page_vecs;
        uint4 x[kMoveVecs];
#pragma unroll
        for (int u = 0; u < kMoveVecs; ++u)
            if (c0 + u * kMoveThreads < page_vecs) x[u] = __ldcs(s + c0 + u * kMoveThreads);
#pragma unroll
        for (int u = 0; u < kMoveVecs; ++u)
            if (c0 + u * kMoveThreads < page_vecs) __stcs(d + c0 + u * kMoveThreads, x[u]);
    }
}

__global__ void __launch_bounds__(256) pages_reset_kernel(const Book b, int max_slots) {
    pdl_wait();
    const long long step = (long long)gridDim.x * 256, t = (long long)blockIdx.x * 256 + threadIdx.x;
    for (long long i = t; i < (long long)max_slots * b.max_pages; i += step) b.table[i] = -1;
    for (long long i = t; i < max_slots; i += step) b.length[i] = 0;
    for (long long i = t; i < b.n_pages; i += step) b.refs[i] = 0;
}

Book book_of(const beagle_pages* p) { return Book{p->table, p->length, p->refs, p->ws, p->n_pages, p->page_size, p->max_pages}; }
int elt_bytes(const beagle_pages* p) { return p->dtype == BEAGLE_BF16 ? 2 : 4; }
beagle_status launched() { return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA; }

void launch_move(const beagle_pages* p, int most_pages, int remap, cudaStream_t stream) {
    const int vecs = (int)((size_t)p->n_kv_heads * p->page_size * p->head_dim * elt_bytes(p) / 16);
    const int chunks = (vecs + kMoveThreads * kMoveVecs - 1) / (kMoveThreads * kMoveVecs);
    const long long most = (long long)most_pages * 2 * chunks;
    const int fit = device_sm_count() * 8;               // eight 256-thread CTAs fit an SM
    const int grid = (int)(most < fit ? (most > 0 ? most : 1) : fit);
    launch_pdl(pages_move_kernel, dim3(grid), dim3(kMoveThreads), 0, stream, book_of(p), static_cast<uint4*>(p->k), static_cast<uint4*>(p->v), vecs,
               remap, p->max_slots * p->max_pages);
}

}  // namespace

beagle_status pages_append_rows(const beagle_pages* p, int batch, const int32_t* slot_host, const AppendRows& rows, const int32_t* n_new_dev,
                                const void* k_new_dev, long long k_stride, const void* v_new_dev, long long v_stride, int32_t* ok_dev, cudaStream_t stream) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    PageSlots slots;
    st = pages_check_slots(p, batch, slot_host, &slots);
    if (st != BEAGLE_OK) return st;
    if (batch == 0) return BEAGLE_OK;
    int most = 0;
    for (int b = 0; b < batch; ++b) most = rows.count[b] > most ? rows.count[b] : most;
    const int e = elt_bytes(p), width = p->n_kv_heads * p->head_dim;
    if (most > 0 && (k_new_dev == nullptr || v_new_dev == nullptr || k_stride < width || v_stride < width)) return BEAGLE_ERR_INVALID_ARG;
    if ((((uintptr_t)k_new_dev | (uintptr_t)v_new_dev) & 15) || (k_stride * e) % 16 || (v_stride * e) % 16) return BEAGLE_ERR_INVALID_ARG;
    const int dv = p->head_dim * e / 16;
    int shift = 0;
    while ((1 << shift) < dv) ++shift;
    const long long pieces = (long long)most * p->n_kv_heads * dv;
    const long long chunks = (pieces + kMoveThreads * kMoveVecs - 1) / (kMoveThreads * kMoveVecs);
    if (chunks > 0x3fffffff) return BEAGLE_ERR_CAPACITY;
    launch_pdl(pages_append_book_kernel, dim3(1), dim3(kBookThreads), 0, stream, book_of(p), slots, rows, batch, n_new_dev, ok_dev);
    if (most > 0)
        launch_pdl(pages_append_write_kernel, dim3((unsigned)(chunks + p->n_kv_heads), batch), dim3(kMoveThreads), 0, stream, book_of(p), slots, rows,
                   static_cast<uint4*>(p->k), static_cast<uint4*>(p->v), static_cast<const uint4*>(k_new_dev), static_cast<const uint4*>(v_new_dev),
                   k_stride * e / 16, v_stride * e / 16, p->n_kv_heads, shift, (int)chunks);
    return launched();
}

}  // namespace beagle

extern "C" {

beagle_status beagle_pages_workspace_bytes(const beagle_pages* p, size_t* bytes) {
    if (p == nullptr || bytes == nullptr || p->n_pages <= 0) return BEAGLE_ERR_INVALID_ARG;
    *bytes = (kBookHead + (size_t)p->n_pages * 3 * sizeof(int32_t) + 255) / 256 * 256;
    return BEAGLE_OK;
}

beagle_status beagle_pages_reset(const beagle_pages* p, void* stream) {
    const beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    launch_pdl(pages_reset_kernel, dim3(device_sm_count()), dim3(256), 0, static_cast<cudaStream_t>(stream), book_of(p), p->max_slots);
    return launched();
}

beagle_status beagle_pages_append(const beagle_pages* p, int32_t batch, const int32_t* slot_host, int32_t T, const int32_t* n_new_dev,
                                  const void* k_new_dev, int64_t k_stride, const void* v_new_dev, int64_t v_stride, int32_t* ok_dev, void* stream) {
    const beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    if (T < 0) return BEAGLE_ERR_INVALID_ARG;
    if (T > 0x40000000) return BEAGLE_ERR_CAPACITY;
    AppendRows rows;
    for (int b = 0; b < kMaxCallBatch; ++b) {
        rows.start[b] = (long long)b * T;
        rows.count[b] = T;
    }
    return pages_append_rows(p, batch, slot_host, rows, n_new_dev, k_new_dev, k_stride, v_new_dev, v_stride, ok_dev, static_cast<cudaStream_t>(stream));
}

beagle_status beagle_pages_truncate(const beagle_pages* p, int32_t n, const int32_t* slot_host, const int32_t* keep_dev, void* stream) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    PageSlots slots;
    st = pages_check_slots(p, n, slot_host, &slots);
    if (st != BEAGLE_OK || n == 0) return st;
    launch_pdl(pages_truncate_kernel, dim3(n), dim3(128), 0, static_cast<cudaStream_t>(stream), book_of(p), slots, keep_dev);
    return launched();
}

// src in range (repeats allowed), dst in range and distinct, no slot in both.
static beagle_status check_pairs(const beagle_pages* p, int n, const int32_t* src, const int32_t* dst, PageSlots* s, PageSlots* d) {
    beagle_status st = pages_check_slots(p, n, dst, d);
    if (st != BEAGLE_OK) return st;
    if (n > 0 && src == nullptr) return BEAGLE_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        if (src[i] < 0 || src[i] >= p->max_slots) return BEAGLE_ERR_INVALID_ARG;
        for (int j = 0; j < n; ++j)
            if (dst[j] == src[i]) return BEAGLE_ERR_INVALID_ARG;
        s->slot[i] = src[i];
    }
    return BEAGLE_OK;
}

beagle_status beagle_pages_fork(const beagle_pages* p, int32_t n, const int32_t* src_host, const int32_t* dst_host, void* stream) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    PageSlots src, dst;
    st = check_pairs(p, n, src_host, dst_host, &src, &dst);
    if (st != BEAGLE_OK || n == 0) return st;
    launch_pdl(pages_fork_kernel, dim3(n), dim3(128), 0, static_cast<cudaStream_t>(stream), book_of(p), src, dst);
    return launched();
}

beagle_status beagle_pages_copy(const beagle_pages* p, int32_t n, const int32_t* src_host, const int32_t* dst_host, int32_t* ok_dev, void* stream_) {
    beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    PageSlots src, dst;
    st = check_pairs(p, n, src_host, dst_host, &src, &dst);
    if (st != BEAGLE_OK || n == 0) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    launch_pdl(pages_copy_book_kernel, dim3(1), dim3(kBookThreads), 0, stream, book_of(p), src, dst, n, ok_dev);
    const long long most = (long long)n * p->max_pages;
    launch_move(p, (int)(most < p->n_pages ? most : p->n_pages), 0, stream);
    return launched();
}

beagle_status beagle_pages_compact(const beagle_pages* p, void* stream_) {
    const beagle_status st = pages_check(p);
    if (st != BEAGLE_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    launch_pdl(pages_compact_book_kernel, dim3(1), dim3(kBookThreads), 0, stream, book_of(p));
    launch_move(p, p->n_pages / 2, 1, stream);           // at most every other page is live above a hole
    return launched();
}

}  // extern "C"
