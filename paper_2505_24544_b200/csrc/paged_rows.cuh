// One run of tiles with up to eight query rows a pair on mma.sync (bf16, head_dim 64 / 128): the body of the one-token kernel (paged_attn.cu) and
// of the rows' part of the grouped one (paged_grouped.cu).
#pragma once
#include <cuda.h>

#include "paged_attn.cuh"
#include "tc_ptx.cuh"

namespace beagle {

using namespace tc;

constexpr int kConsumers = 4;           // warps; each owns 16 positions of a tile
constexpr int kPerWarp = kTile / kConsumers;
constexpr int kStages = 3;
constexpr int kCtasPerSm = 2;

// The entries' pairs always leave partials, at a place of their own: the part of a pair that begins it at its number, a later one behind
// them at the run's.
__device__ __forceinline__ int part_at(const PagedArgs&, int, bool, int seg, int run) { return 2 * run + seg; }
__device__ __forceinline__ int part_at(const SharedArgs& a, int pair, bool begins, int, int run) { return begins ? pair : a.n_pairs + run; }

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
// D (16 x 8, fp32) += A (16 x 16) B (16 x 8); rows 8..15 of A are zero (at most eight query heads share a K/V head)
__device__ __forceinline__ void mma_rows8(float* d, uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
    float z0 = 0.f, z1 = 0.f;
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%5}, {%7,%8}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(z0), "+f"(z1)
                 : "r"(a0), "r"(0u), "r"(a2), "r"(b0), "r"(b1));
}
// Untiled copy: both addresses 16-byte aligned, `bytes` a multiple of 16.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <int DH>
struct PagedSmem {
    static constexpr int kTileBytes = kTile * DH * 2;                       // one of K / V
    static constexpr int kJoin = 2 * 8 * DH * 4;                            // two warps' O rows on their way to the other two
    static constexpr int kBytes = kStages * 2 * kTileBytes + kJoin + 1024;  // + alignment slack
};

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// The units [u0, u1) of run `run`.  Warp `warp`: 0..3 consumers, 4 producer, which fills the ring at `base` (1024-byte aligned, kStages * 2 tiles); join: kJoin
// bytes, and s_m, s_l, where the warps meet (the shared form does not use them); full, empty: kStages barriers each, of 1 and kConsumers arrivals.  Barriers have not been used before.
template <int DH, typename Args>
__device__ __forceinline__ void attn_rows(const CUtensorMap& tmK, const CUtensorMap& tmV, const Args& a, const ScheduleOf<Args::kEntries>& s, uint32_t base,
                                          float* join, uint32_t full, uint32_t empty, float (*s_m)[8], float (*s_l)[8], volatile int* s_abort, int warp, int run,
                                          int u0, int u1) {
    using SM = PagedSmem<DH>;
    const int lane = threadIdx.x & 31;
    Walk w;
    w.seek(s, u0, a.Hkv);

    if (warp == kConsumers) {
        // ---------------- producer: lane p copies page p of the tile (a tile spans 1, 2, 4 or 8 pages)
        const int rows = min(1 << a.page_shift, kTile);          // rows of one copy
        const int parts = kTile / rows;
        const uint32_t part_bytes = (uint32_t)rows * DH * 2;
        const uint64_t once = policy_evict_first();
        bool ok = true;
        int issued = 0;
        int next_page = -1;
        auto page_of = [&](const Walk& x) {                      // this lane's page of the walk's tile, -1 if it holds no position
            const int pos = x.tile(s) * kTile + lane * rows;
            int id = -1;
            // (a part without a visible position stays what it was: its weights and its V rows count as 0)
            if (lane < parts && pos < s.len[x.b] && (pos + rows > s.lo[x.b] || pos < a.sinks)) id = __ldcg(a.table + (size_t)slot_of(a, x.b) * a.max_pages + (pos >> a.page_shift));
            return (id >= 0 && id < a.n_pages) ? id : -1;
        };
        next_page = page_of(w);
        for (int u = u0; u < u1; ++u) {
            const int st = issued % kStages;
            const int page = next_page;
            const int pos = w.tile(s) * kTile + lane * rows;
            const int row = page >= 0 ? ((page * a.Hkv + w.kvh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : 0;
            w.next(s, a.batch, a.Hkv);
            if (u + 1 < u1) next_page = page_of(w);              // the next tile's entry is on its way while this one waits for its slot
            const int copies = __popc(__ballot_sync(0xffffffffu, page >= 0));
            ok = mbar_wait(empty + 8 * st, ((issued / kStages) & 1) ^ 1, s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (lane == 0) {
                if (copies > 0) mbar_expect_tx(full + 8 * st, 2 * copies * part_bytes);
                else mbar_arrive(full + 8 * st);
            }
            __syncwarp();
            if (page >= 0) {
                const uint32_t dst = base + st * 2 * SM::kTileBytes + lane * part_bytes;
#pragma unroll
                for (int h = 0; h < DH / 64; ++h) tma_load_2d_hint(dst + h * rows * 128, &tmK, full + 8 * st, 64 * h, row, once);
#pragma unroll
                for (int h = 0; h < DH / 64; ++h) tma_load_2d_hint(dst + SM::kTileBytes + h * rows * 128, &tmV, full + 8 * st, 64 * h, row, once);
            }
            ++issued;
        }
        if (!ok)                         // copies already requested still land: wait (bounded) for the last of each stage
            for (int n = max(0, issued - kStages); n < issued; ++n)
                for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(full + 8 * (n % kStages), (n / kStages) & 1); ++i) {}
        return;
    }

    // ---------------- consumers
    const int g = lane >> 2, c = lane & 3;
    const int r_log = min(a.page_shift, 6);                      // log2 rows of a copy
    const int half_step = 128 << r_log, part_step = DH * 2 << r_log, r_mask = (1 << r_log) - 1;
    // byte offset of 16-byte piece `chunk` of row r: [copy][64-column half][row][128 bytes], swizzled inside 8 rows
    auto off = [&](int r, int chunk) {
        return (uint32_t)((r >> r_log) * part_step + (chunk >> 3) * half_step + (r & r_mask) * 128 + (((chunk & 7) ^ (r & 7)) << 4));
    };
    const int row0 = warp * kPerWarp;
    float o[DH / 8][2], m = -INFINITY, l = 0.f;
    uint32_t qa[DH / 16][2];
    int have_q = -1;                                             // the pair whose queries are in registers
    int seg = 0;                                                 // partial slot: the run's first pair that continues, else the second
    bool ok = true, first_pair_open = w.i > 0;                   // the first pair began in an earlier run
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = 0.f;
    int step = 0;
    for (int u = u0; u < u1; ++u, ++step) {
        const int pair = w.b * a.Hkv + w.kvh;
        if (pair != have_q) {
            have_q = pair;
            const bool some = g < rows_of(a, w.b);
            const uint32_t* qrow = reinterpret_cast<const uint32_t*>(static_cast<const bf16*>(a.q) + query_at(a, w.b, w.kvh, some ? g : 0, DH));
#pragma unroll
            for (int ks = 0; ks < DH / 16; ++ks) {
                qa[ks][0] = some ? __ldcg(qrow + ks * 8 + c) : 0u;
                qa[ks][1] = some ? __ldcg(qrow + ks * 8 + 4 + c) : 0u;
            }
        }
        const int st = step % kStages;
        const int pos0 = w.tile(s) * kTile + row0;               // first position of this warp
        const int len = s.len[w.b], lo = s.lo[w.b];
        const bool plain = pos0 + kPerWarp <= len && (pos0 >= lo || pos0 + kPerWarp <= a.sinks);
        // A wait that runs out leaves NaN in what depends on it; the warp still meets the others where pairs end.
        if (ok) ok = mbar_wait(full + 8 * st, (step / kStages) & 1, s_abort);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) l = __int_as_float(0x7fffffff);
        const uint32_t sK = base + st * 2 * SM::kTileBytes, sV = sK + SM::kTileBytes;
        if (ok && pos0 < len && (pos0 + kPerWarp > lo || pos0 < a.sinks)) {
            float sc[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
            for (int dg = 0; dg < DH / 32; ++dg)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    uint32_t b0, b1, b2, b3;
                    ldsm4(sK + off(row0 + nt * 8 + (lane & 7), 4 * dg + (lane >> 3)), b0, b1, b2, b3);
                    mma_rows8(sc[nt], qa[2 * dg][0], qa[2 * dg][1], b0, b1);
                    mma_rows8(sc[nt], qa[2 * dg + 1][0], qa[2 * dg + 1][1], b2, b3);
                }
            uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;   // V rows (2c, 2c+1) and (2c+8, 2c+9) as 16-bit lanes
            float mx = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = sc[nt][e] * a.scale_log2;
                    if (!plain) {
                        const int pos = pos0 + nt * 8 + 2 * c + e;
                        const bool vis = pos < len && (pos >= lo || pos < a.sinks);
                        x = vis ? x : -INFINITY;
                        if (!vis) (nt == 0 ? keep0 : keep1) &= e == 0 ? 0xffff0000u : 0x0000ffffu;
                    }
                    sc[nt][e] = x;
                    mx = fmaxf(mx, x);
                }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            // the reference point moves only when a score exceeds it by more than kSlack: weights stay below 2^8
            const bool grow = mx > m + kSlack;
            if (__any_sync(0xffffffffu, grow)) {
                const float f = (grow && m != -INFINITY) ? exp2f(m - mx) : 1.f;
                if (grow) m = mx;
                l *= f;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) { o[i][0] *= f; o[i][1] *= f; }
            }
            const float neg = m == -INFINITY ? 0.f : -m;         // no visible position so far: every score is -inf, every weight 0
            uint32_t pa[2];
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const float p0 = exp2f(sc[nt][0] + neg), p1 = exp2f(sc[nt][1] + neg);
                l += p0 + p1;                                    // fp32, unrounded; the product below takes the weights in bf16
                pa[nt] = pack2(p0, p1);
            }
            const int mi = lane >> 3;
#pragma unroll
            for (int jp = 0; jp < DH / 16; ++jp) {
                uint32_t b0, b1, b2, b3;
                ldsm4_t(sV + off(row0 + 8 * (mi & 1) + (lane & 7), 2 * jp + (mi >> 1)), b0, b1, b2, b3);
                if (!plain) { b0 &= keep0; b1 &= keep1; b2 &= keep0; b3 &= keep1; }
                mma_rows8(o[2 * jp], pa[0], pa[1], b0, b1);
                mma_rows8(o[2 * jp + 1], pa[0], pa[1], b2, b3);
            }
        }
        __syncwarp();
        if (ok && lane == 0) mbar_arrive(empty + 8 * st);
        const int b = w.b, kvh = w.kvh;
        const bool last = w.i + 1 == w.n;
        w.next(s, a.batch, a.Hkv);
        if (!last && u + 1 < u1) continue;

        // ---- the pair (or this run's part of it) is done: join the four warps, rows = heads
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if constexpr (Args::kShared) {
            // many short pairs: every warp leaves its part for the join, the warps need not meet
            if (g < rows_of(a, b)) {
                float* dst = a.part + (((size_t)part_at(a, b * a.Hkv + kvh, !first_pair_open, seg, run) * kConsumers + warp) * 8 + g) * (DH + 2);
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<float2*>(dst + 8 * i + 2 * c) = make_float2(o[i][0], o[i][1]);
                if (c == 0) *reinterpret_cast<float2*>(dst + DH) = make_float2(m, l);
            }
            first_pair_open = false;
            m = -INFINITY; l = 0.f;
#pragma unroll
            for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = 0.f;
            continue;
        }
        if (c == 0) { s_m[warp][g] = m; s_l[warp][g] = l; }
        consumers_sync();
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int i = 0; i < kConsumers; ++i) M = fmaxf(M, s_m[i][g]);
#pragma unroll
        for (int i = 0; i < kConsumers; ++i) L += s_m[i][g] == -INFINITY ? s_l[i][g] : s_l[i][g] * exp2f(s_m[i][g] - M);      // (no position seen: the sum is 0)
        const float f = m == -INFINITY ? 0.f : exp2f(m - M);
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) { o[i][0] *= f; o[i][1] *= f; }
        // warps 2, 3 hand theirs to 0, 1; then 1 to 0
#pragma unroll
        for (int from = 2; from >= 1; --from) {
            if (warp >= from && warp < 2 * from) {
                float* dst = join + (size_t)(warp - from) * 8 * DH + g * DH + 2 * c;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<float2*>(dst + 8 * i) = make_float2(o[i][0], o[i][1]);
            }
            consumers_sync();
            if (warp < from) {
                const float* src = join + (size_t)warp * 8 * DH + g * DH + 2 * c;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) {
                    const float2 x = *reinterpret_cast<const float2*>(src + 8 * i);
                    o[i][0] += x.x; o[i][1] += x.y;
                }
            }
            consumers_sync();
        }
        if (warp == 0 && g < rows_of(a, b)) {
            const int head = kvh * a.G + g;
            if (last && !first_pair_open) {    // all of the pair's tiles were in this run
                const float inv = L != 0.f ? 1.f / L : 0.f;
                uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<bf16*>(a.o) + ((size_t)b * a.Hq + head) * DH) + c;
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) dst[4 * i] = pack2(o[i][0] * inv, o[i][1] * inv);
                if (c == 0 && a.lse != nullptr) a.lse[(size_t)b * a.Hq + head] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
            } else {
                float* dst = a.part + ((size_t)part_at(a, b * a.Hkv + kvh, !first_pair_open, seg, run) * 8 + g) * (DH + 2);
#pragma unroll
                for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<float2*>(dst + 8 * i + 2 * c) = make_float2(o[i][0], o[i][1]);
                if (c == 0) { dst[DH] = M; dst[DH + 1] = L; }
            }
        }
        first_pair_open = false;
        seg = 1;
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = 0.f;
    }
}

}  // namespace beagle
