// Attention of groups of rows whose slots begin with the same positions (beagle_paged_attn_shared) where the groups are large enough for the
// tensor cores: one launch for the common parts, on tcgen05, and for what each row has behind them (paged_rows.cuh, mma.sync).
//
// Common part: up to 128 query rows of a group (rows times grouped heads) that read one K/V head are the rows of a tcgen05 tile, so each
// cached tile is read once for all of them: R G flop per byte.  More than 128 of them are blocks of their own, each of which reads every tile; from
// DRAM the tiles still come once (64 rows of four grouped heads over 65536 positions: 544 MB read, 534 of cache), the second time from L2.
// The tiles of 64 positions of all (block of query rows, K/V head) pairs, one after the other, are cut into equal runs on the device
// (paged_attn.cuh); a run leaves one partial per pair that it touches (O in fp32, not normalised, with the maximum and sum of each row),
// which the join launch adds to what the rows see behind the common part, in a fixed order.
//
// Two CTAs per SM, each with one kind of work, shared out by the tiles, the kinds side by side as far as possible: common parts wait
// for the hand-over between softmax and products, rows for memory.  Measured: 32 rows over 8192 common positions, 32/8 heads of 128, some hundred
// positions behind: 28 us with the join, of which the join takes 9 (the two kinds in launches of their own: 48, in one 41, at that time); four groups of 16 rows over
// 2094 to 3511, 32/32 heads: 81 us; 64 rows over 65536, 100 to 2048 behind: 146 us, tensor pipe 0.43 busy (all CTAs first one kind, then the other: 167); alone the
// common parts run at 207 tiles a microsecond (868 TFLOP/s with 128 query rows, half of the tensor cores' rate) and the rows at 5.8 TB/s.
//
// A common part's CTA: a producer warp (pages by TMA, 128-byte swizzle, two stages of K and V; the queries of the block as one box of a
// [row, head, component] map), a warp that issues the products, and four warps with one thread per query row: S = Q K^T into tensor memory ->
// P = exp2(S - m) in bf16 over S -> O += P V with P as the tensor-memory operand.  m is the row's reference point, moved only when a tile
// exceeds it by more than 2^8.  S is double-buffered.  All positions of the common part are visible: nothing is masked.  P is rounded to
// bf16 because the product takes both operands in one type; its row sum is of the unrounded weights, in fp32.  (Results are 2.3e-3 from 64 bits, of
// which rounding the result itself to bf16 is 1.7e-3.)
#include <cuda.h>

#include "paged_rows.cuh"
#include "tensor_map.h"
#include "win_ptx.cuh"

namespace beagle {
namespace {

constexpr int kThreads = 192;            // warp 0: TMA producer, warp 1: issues the products, warps 2-5: softmax
constexpr int kRows = 128;               // query rows of a tile

template <int DH>
struct PrefixSmem {
    static_assert(4 * (DH + 2) * 4 % 32 == 0 && DH * 4 % 32 == 0, "partials are stored 32 bytes at once");
    static constexpr int kQ = kRows * DH * 2, kT = kTile * DH * 2;           // Q; a K or V tile, two stages of each
    static constexpr int kRing = kQ + 4 * kT;                                // as much as the rows' ring
    static_assert(kRing == kStages * 2 * PagedSmem<DH>::kTileBytes, "both kinds of work use the same memory in turn");
    static constexpr int kBytes = kRing + 1024;                              // + alignment slack
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

// 32 bytes, a whole sector, at once: each thread writes a row of its own.  p on 32 bytes: partials begin on multiples of that (kWsAlign, four rows
// of DH + 2 floats), and so do their rows.
__device__ __forceinline__ void store32(float* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// The common parts' run [u, u1) of this CTA: warp 0 producer, 1 issues the products, 2..5 softmax.  Ends with all of shared and tensor memory free.
template <int DH>
__device__ __forceinline__ void attn_prefix(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PrefixArgs& a,
                                            const ScheduleOf<SharedArgs::kEntries>& s, uint8_t* smem, uint64_t* bars, uint32_t tmem, volatile int* s_abort, int warp,
                                            int run, int u, int u1) {
    using SM = PrefixSmem<DH>;
    constexpr int kHalves = DH / 64;
    constexpr uint32_t kO = 128;                                 // S / P at columns 0 and 64, O at 128
    const uint32_t sQ = smem_u32(smem), sK = sQ + SM::kQ, sV = sK + 2 * SM::kT;
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, k_full = bar0 + 16, k_empty = bar0 + 32, v_full = bar0 + 48, s_full = bar0 + 64, p_full = bar0 + 80,
                   pv_done = bar0 + 96;                          // all but the first: one per stage
    const int lane = threadIdx.x & 31;
    bool ok = *s_abort == 0;
    int done = 0;                                                // tiles of this CTA's earlier pairs: stages and phases run on
    for (int seg = 0; u < u1; ++seg) {
        Walk w;
        w.seek(s, u, a.Hkv);
        const int J = min(u1 - u, w.n - w.i);                    // tiles of this pair in this run
        const SharedEntry e = a.entry[w.b];
        if (warp == 0) {
            // lane p copies page p of a tile (a tile spans 1, 2, 4 or 8 pages)
            const int rows = min(1 << a.page_shift, kTile), parts = kTile / rows;
            const uint32_t bytes = (uint32_t)rows * 128;         // of one half of a part
            const int32_t* table = a.table + (size_t)a.slots.slot[e.row0] * a.max_pages;
            auto page_of = [&](int j) {
                const int pos = (w.i + j) * kTile + lane * rows;
                const int id = lane < parts ? __ldcg(table + (pos >> a.page_shift)) : -1;
                return id >= 0 && id < a.n_pages ? id : -1;
            };
            int page = page_of(0);                               // this lane's of the tile whose values come next
            if (ok && lane == 0) {
                mbar_expect_tx(q_full, kHalves * (kRows / a.G) * a.G * 128);
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) tma_load_3d(sQ + hf * (kRows * 128), &tmQ, q_full, hf * 64, w.kvh * a.G, e.row0 + e.j0 / a.G);
            }
            const bool waiting = ok;                             // a request for the queries is out
            int k_issued = done, v_issued = done;
            auto copy = [&](int j, int id, const CUtensorMap* tm, uint32_t dst, uint32_t full) {
                const int pos = (w.i + j) * kTile + lane * rows;
                const int row = id >= 0 ? ((id * a.Hkv + w.kvh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : 0;
                const int copies = __popc(__ballot_sync(0xffffffffu, id >= 0));
                if (lane == 0) {
                    if (copies > 0) mbar_expect_tx(full, kHalves * copies * bytes);
                    else mbar_arrive(full);
                }
                __syncwarp();
                if (id >= 0)
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_2d(dst + hf * (kTile * 128) + lane * bytes, tm, full, 64 * hf, row);
                __syncwarp();
            };
            auto keys = [&](int j, int id) {
                const int jg = done + j, st = jg & 1;
                ok = warp_wait(k_empty + 8 * st, ((jg >> 1) & 1) ^ 1, s_abort);
                if (!ok) return;
                copy(j, id, &tmK, sK + st * SM::kT, k_full + 8 * st);
                ++k_issued;
            };
            if (ok) keys(0, page);
            for (int j = 0; j < J && ok; ++j) {
                // the next tile's keys before this one's values, whose place is free later
                const int next = j + 1 < J ? page_of(j + 1) : -1;
                if (j + 1 < J) keys(j + 1, next);
                if (!ok) break;
                const int jg = done + j, st = jg & 1;
                ok = warp_wait(pv_done + 8 * st, ((jg >> 1) & 1) ^ 1, s_abort);
                if (!ok) break;
                copy(j, page, &tmV, sV + st * SM::kT, v_full + 8 * st);
                ++v_issued;
                page = next;
            }
            if (!ok) {                                           // copies already requested still land (bounded)
                if (waiting)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(q_full, seg & 1); ++i) {}
                for (int n = max(0, k_issued - 2); n < k_issued; ++n)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(k_full + 8 * (n & 1), (n >> 1) & 1); ++i) {}
                for (int n = max(0, v_issued - 2); n < v_issued; ++n)
                    for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(v_full + 8 * (n & 1), (n >> 1) & 1); ++i) {}
            }
        } else if (warp == 1) {
            const bool leader = elect_one();
            constexpr uint32_t idesc_s = make_idesc(kRows, kTile), idesc_o = make_idesc_major(kRows, DH, false, true);
            if (ok) ok = warp_wait(q_full, seg & 1, s_abort);
            auto issue_s = [&](int j) {
                const int jg = done + j, st = jg & 1;
                if (ok) ok = warp_wait(k_full + 8 * st, (jg >> 1) & 1, s_abort);
                if (ok && jg >= 2) ok = warp_wait(pv_done + 8 * st, ((jg >> 1) & 1) ^ 1, s_abort);     // P of tile j - 2 lies where S goes now
                if (!ok) return;
                fence_after();
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    const uint64_t dq = umma_desc(sQ + hf * (kRows * 128)), dk = umma_desc(sK + st * SM::kT + hf * (kTile * 128));
#pragma unroll
                    for (int k = 0; k < BK / UMMA_K; ++k) {
                        const uint64_t off = static_cast<uint64_t>((k * UMMA_K * 2) >> 4);
                        umma_ss(leader, tmem + st * kTile, dq + off, dk + off, idesc_s, (hf > 0 || k > 0) ? 1u : 0u);
                    }
                }
                commit_el(leader, k_empty + 8 * st);
                commit_el(leader, s_full + 8 * st);
            };
            if (ok) issue_s(0);
            for (int j = 0; j < J && ok; ++j) {
                const int jg = done + j, st = jg & 1, ph = (jg >> 1) & 1;
                if (j + 1 < J) issue_s(j + 1);
                if (ok) ok = warp_wait(v_full + 8 * st, ph, s_abort);
                if (ok) ok = warp_wait(p_full + 8 * st, ph, s_abort);
                if (!ok) break;
                fence_after();
                const uint64_t dv = umma_desc_mn(sV + st * SM::kT, kTile * 128);
#pragma unroll
                for (int k = 0; k < kTile / UMMA_K; ++k)
                    umma_ts(leader, tmem + kO, tmem + st * kTile + 8 * k, dv + static_cast<uint64_t>((k * UMMA_K * 128) >> 4), idesc_o, (j > 0 || k > 0) ? 1u : 0u);
                commit_el(leader, pv_done + 8 * st);
            }
        } else {
            const int q = warp & 3, jr = q * 32 + lane;          // tensor-memory lane quarter of this warp; query row of this thread
            const uint32_t lanes = static_cast<uint32_t>(q * 32) << 16;
            const uint64_t scale2 = pk2(a.scale_log2, a.scale_log2);
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < J; ++j) {
                const int jg = done + j, st = jg & 1, ph = (jg >> 1) & 1;
                if (ok) ok = warp_wait(s_full + 8 * st, ph, s_abort);
                if (!ok) break;
                fence_after();
                const uint32_t ts = tmem + st * kTile + lanes;
                uint32_t r[2][32];
                tmem_ld32(ts, r[0]);
                tmem_ld32(ts + 32, r[1]);
                tmem_ld_wait();
                const float mx = chunk_max<false>(r[1], 0u, chunk_max<false>(r[0], 0u, -INFINITY)) * a.scale_log2;
                const float m_old = m;
                const bool grow = mx > m_old + kSlack;
                m = grow ? mx : m_old;
                const float factor = (grow && m_old != -INFINITY) ? exp2f(m_old - m) : 1.f;
                if (__any_sync(0xffffffffu, factor != 1.f)) {    // (never in a pair's first tile: m was -inf there)
                    ok = warp_wait(pv_done + 8 * (st ^ 1), ((jg - 1) >> 1) & 1, s_abort);      // O is complete up to the last tile
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
                const float neg = m == -INFINITY ? 0.f : -m;     // (a row of scores that are all -inf)
                const uint64_t neg2 = pk2(neg, neg);
                uint64_t sum0 = 0, sum1 = 0;                     // row sum in fp32 over the unrounded weights
                uint32_t p[16];
                chunk_exp(r[0], scale2, neg2, p, sum0, sum1);
                tmem_st16(ts, p);                                // over S: this thread has its row in registers
                chunk_exp(r[1], scale2, neg2, p, sum0, sum1);
                tmem_st16(ts + 16, p);
                float x0, x1;
                un2(add2(sum0, sum1), x0, x1);
                l = fmaf(l, factor, x0 + x1);
                tmem_st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * st);
            }
            if (ok) ok = warp_wait(pv_done + 8 * ((done + J - 1) & 1), ((done + J - 1) >> 1) & 1, s_abort);
            const int part = w.i == 0 ? w.b * a.Hkv + w.kvh : a.n_pairs + run;
            float* dst = a.part + (size_t)part * a.part_rows * (DH + 2);
            fence_after();
#pragma unroll
            for (int c0 = 0; c0 < DH; c0 += 32) {
                uint32_t o[32];
                tmem_ld32(tmem + kO + c0 + lanes, o);
                tmem_ld_wait();
                if (jr < e.n)
#pragma unroll
                    for (int x = 0; x < 32; x += 8) store32(dst + jr * DH + c0 + x, o + x);
            }
            // a wait that ran out leaves NaN in what depends on it
            if (jr < e.n) *reinterpret_cast<float2*>(dst + a.part_rows * DH + 2 * jr) = make_float2(m, ok ? l : __int_as_float(0x7fffffff));
            fence_before();
        }
        done += J;
        u += J;
        __syncthreads();                                         // O is read, Q may be overwritten
        fence_after();
        ok = *s_abort == 0;
    }
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 2) paged_grouped_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                                                                   const __grid_constant__ CUtensorMap tmV, const __grid_constant__ SharedArgs rows,
                                                                   const __grid_constant__ PrefixArgs prefix) {
    using SM = PrefixSmem<DH>;
    constexpr uint32_t kTmem = 256;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ __align__(8) uint64_t bars[14 + 2 * kStages];
    __shared__ ScheduleOf<SharedArgs::kEntries> s_rows, s_prefix;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const uint32_t full = smem_u32(bars + 14), empty = full + 8 * kStages;
    if (threadIdx.x == 0) {
        const uint32_t bar0 = smem_u32(bars);
        mbar_init(bar0, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar0 + 16 + 8 * i, 1); mbar_init(bar0 + 32 + 8 * i, 1); mbar_init(bar0 + 48 + 8 * i, 1);
            mbar_init(bar0 + 64 + 8 * i, 1); mbar_init(bar0 + 80 + 8 * i, 4); mbar_init(bar0 + 96 + 8 * i, 1);
        }
        for (int i = 0; i < kStages; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kConsumers); }
        s_abort = 0;
        fence_barrier_init();
    }
    if (threadIdx.x == 32 * 3) { prefetch_tensormap(&tmQ); prefetch_tensormap(&tmK); prefetch_tensormap(&tmV); }
    // Tensor memory is taken after the kernels before have ended and before those behind may begin: a block that waits for its turn holds none that
    // a block in front of it could still ask for, and nobody behind it can take what it is about to ask for.
    pdl_wait();
    if (warp == 1) tmem_alloc<kTmem>(smem_u32(&s_tmem));
    fence_before();
    build_schedules(rows, s_rows, prefix, s_prefix);
    fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    // The CTAs do one kind of work each, shared out by its tiles, the two kinds side by side on an SM as far as possible: one waits for
    // memory, the other for the products.  64 rows over 65536: 146 us; with a common part's tile counted as 0.8, 1.2 and 1.4 of a row's 159, 151, 172.
    const int total_p = s_prefix.start[SharedArgs::kEntries], total_r = s_rows.start[SharedArgs::kEntries], n = (int)gridDim.x;
    int n_prefix = total_p > 0 || total_r > 0 ? (int)((float)n * (float)total_p / ((float)total_p + (float)total_r) + 0.5f) : 0;
    if (total_p > 0) n_prefix = max(n_prefix, 1);
    if (total_r > 0) n_prefix = min(n_prefix, n - 1);
    const int half = (n + 1) / 2, at = (int)blockIdx.x < half ? 2 * (int)blockIdx.x : 2 * ((int)blockIdx.x - half) + 1;       // neighbours share an SM
    const int before = (int)((long long)at * n_prefix / n);      // CTAs of the first kind in front of this one
    const bool does_prefix = (int)((long long)(at + 1) * n_prefix / n) > before;
    const int helper = (int)threadIdx.x - 32;                    // the second warp, which has the least to do
    int u0, u1, p0, p1;
    begin_shared(rows, s_rows, does_prefix ? -1 : at - before, n - n_prefix, helper, kThreads - 32, u0, u1);
    begin_shared(prefix, s_prefix, does_prefix ? before : -1, n_prefix, helper, kThreads - 32, p0, p1);
    if (does_prefix) {
        attn_prefix<DH>(tmQ, tmK, tmV, prefix, s_prefix, smem, bars, tmem, &s_abort, warp, before, p0, p1);
    } else {
        const int role = warp == 0 ? kConsumers : warp - 2;      // (the second warp: none)
        if (u0 < u1 && role >= 0)
            attn_rows<DH>(tmK, tmV, rows, s_rows, smem_u32(smem), nullptr, full, empty, nullptr, nullptr, &s_abort, role, at - before, u0, u1);
    }
    fence_before();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        tmem_dealloc<kTmem>(tmem);
    }
}

template <int DH>
beagle_status launch(const beagle_pages* p, const SharedArgs& rows, const PrefixArgs& a, int runs, cudaStream_t stream) {
    using SM = PrefixSmem<DH>;
    const EncodeTiled encode = tensor_map_encoder();
    if (encode == nullptr) return BEAGLE_ERR_CUDA;
    CUtensorMap mq, mk, mv;
    {
        const cuuint64_t dims[3] = {DH, (cuuint64_t)a.Hq, (cuuint64_t)a.rows}, strides[2] = {DH * 2, (cuuint64_t)a.q_stride * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)a.G, (cuuint32_t)(kRows / a.G)}, one[3] = {1, 1, 1};
        if (encode(&mq, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return BEAGLE_ERR_CUDA;
    }
    const cuuint64_t dims[2] = {DH, (cuuint64_t)p->n_pages * p->n_kv_heads * p->page_size}, strides[1] = {DH * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)(p->page_size < kTile ? p->page_size : kTile)}, one[2] = {1, 1};
    for (int i = 0; i < 2; ++i)
        if (encode(i ? &mv : &mk, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, i ? p->v : p->k, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return BEAGLE_ERR_CUDA;
    static PerDeviceOnce attr;
    if (!attr.ensure([] { return cudaFuncSetAttribute(paged_grouped_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::kBytes) == cudaSuccess; }))
        return BEAGLE_ERR_CUDA;
    launch_pdl(paged_grouped_kernel<DH>, dim3(runs), dim3(kThreads), (size_t)SM::kBytes, stream, mq, mk, mv, rows, a);
    return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

}  // namespace

int prefix_block(int G) { return kRows / G * G; }

beagle_status launch_grouped(const beagle_pages* p, const SharedArgs& rows, const PrefixArgs& prefix, int runs, cudaStream_t stream) {
    return p->head_dim == 128 ? launch<128>(p, rows, prefix, runs, stream) : launch<64>(p, rows, prefix, runs, stream);
}

}  // namespace beagle
