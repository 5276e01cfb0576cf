// Rotation of the queries and keys of whole rows by their positions, and its transpose (beagle_rotary_apply).
//
// Bound by memory: every element is read and written once, 3 flop each.  A CTA takes a few rows: its threads form the (cosine, sine)
// entries of those rows in shared memory, one double-precision product and one fp32 sine and cosine per entry, while their first
// loads are on their way; then each thread keeps the entries of its unit (16 bytes of a head and, in the half layout, their partners)
// in registers and walks over the heads.  Queries and keys go in one launch, so that the entries are formed once for both.
//
// Measured: 8 x 2048 positions, 32 + 32 heads of 128, bf16, forward and backward (1.07 GB): 174 us, 6.1 TB/s; 8191 positions, 32 + 8 heads,
// interleaved, a quarter rotated (168 MB): 37 us.  One head at a time in a thread and six CTAs per SM; four heads in flight in two
// CTAs per SM took 240 and 53, entries formed by every thread for itself, without shared memory, 179 and 47.
#include <cfloat>
#include <cmath>
#include <cstring>

#include "rotary.cuh"
#include "tensor_map.h"

namespace beagle {

namespace {

struct RotaryRows {
    const void *q, *k;
    void *q_out, *k_out;
    long long q_stride, k_stride, q_out_stride, k_out_stride;      // elements
    const int32_t* pos;                  // or NULL: pos0 + row % period
    long long rows, period;
    int pos0, Hq, Hk, dh;
    RotaryGrid g;
};

template <typename T, int E, bool INTER>
__global__ void __launch_bounds__(kRotThreads, kRotCtas) rotary_kernel(const __grid_constant__ RotaryArgs r, const __grid_constant__ RotaryRows a) {
    __shared__ __align__(16) float2 s_cs[kRotEntries];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const long long row0 = (long long)blockIdx.x * a.g.rows;
    const int u = t % a.g.units, slot = t / a.g.units, rl = slot / a.g.lanes, lane = slot - rl * a.g.lanes, H = a.Hq + a.Hk;
    const long long row = row0 + rl;
    const bool mine = rl < a.g.rows && row < a.rows;
    RotUnit<T, E, INTER> unit;
    typename RotUnit<T, E, INTER>::V x, y;
    unit.place(u, r.pairs);
    const T *q = static_cast<const T*>(a.q) + row * a.q_stride, *k = static_cast<const T*>(a.k) + row * a.k_stride;
    T *qo = static_cast<T*>(a.q_out) + row * a.q_out_stride, *ko = static_cast<T*>(a.k_out) + row * a.k_out_stride;
    auto load = [&](int h) { unit.load(h < a.Hq ? q + h * a.dh : k + (h - a.Hq) * a.dh, x, y); };
    if (mine && lane < H) load(lane);
    for (int i = t; i < a.g.rows * r.pairs; i += kRotThreads) {
        const long long at = row0 + i / r.pairs;
        if (at < a.rows) {
            const int pos = a.pos != nullptr ? __ldcg(a.pos + at) : (int)(a.pos0 + at % a.period);
            s_cs[i] = rot_angle(r.turns[i % r.pairs], pos, r.m, r.sign);
        }
    }
    __syncthreads();
    if (!mine) return;
    unit.entries(s_cs + rl * r.pairs);
    for (int h = lane; h < H; h += a.g.lanes) {
        if (h != lane) load(h);
        unit.turn(x, y);
        unit.store(h < a.Hq ? qo + h * a.dh : ko + (h - a.Hq) * a.dh, x, y);
    }
}

}  // namespace

// (the kernels multiply by it in fp32: an infinite factor would make NaN of every 0)
static bool finite_in_fp32(double x) { return std::fabs(x) <= FLT_MAX; }

beagle_status rotary_check(const beagle_rotary* r, int dtype) {
    if (r == nullptr || (dtype != BEAGLE_FP32 && dtype != BEAGLE_BF16)) return BEAGLE_ERR_INVALID_ARG;
    const int full = dtype == BEAGLE_BF16 ? 8 : 4;
    if (r->head_dim <= 0 || r->rot_dim <= 0 || (r->interleaved != 0 && r->interleaved != 1) || !finite_in_fp32(r->mscale)) return BEAGLE_ERR_INVALID_ARG;
    if (r->head_dim > 2 * BEAGLE_ROTARY_MAX_PAIRS || r->head_dim % full || r->rot_dim % 2 || r->rot_dim > r->head_dim) return BEAGLE_ERR_SHAPE;
    for (int i = 0; i < r->rot_dim / 2; ++i)
        if (!std::isfinite(r->freq[i])) return BEAGLE_ERR_INVALID_ARG;
    return BEAGLE_OK;
}

void rotary_args(const beagle_rotary* r, int inverse, RotaryArgs* out) {
    out->pairs = r->rot_dim / 2;
    out->interleaved = r->interleaved;
    out->m = (float)r->mscale;
    out->sign = inverse ? -1.f : 1.f;
    for (int i = 0; i < out->pairs; ++i) out->turns[i] = r->freq[i] * 0.15915494309189533577;        // 1 / 2 pi
}

int rotary_unit(const beagle_rotary* r, int dtype) {
    const int full = dtype == BEAGLE_BF16 ? 8 : 4;
    if (r->interleaved) return full;
    int e = full;                        // partners lie rot_dim / 2 apart: both sides aligned
    while ((r->rot_dim / 2) % e) e /= 2;
    return e;
}

RotaryGrid rotary_grid(const beagle_rotary* r, int dtype, long long rows, int heads) {
    const int e = rotary_unit(r, dtype), pairs = r->rot_dim / 2;
    RotaryGrid g;
    g.units = r->interleaved ? r->head_dim / e : pairs / e + (r->head_dim - r->rot_dim) / e;
    const int slots = kRotThreads / g.units;         // a head has at most 256 elements
    // many rows: a CTA takes several, so that it has entries to form for all of its threads, and a thread several heads with the same
    // ones; few rows: the heads of a row over as many threads as there are.  Measured, 8 heads side by side / all, us, heads of 128, bf16: 32 rows of
    // 32 + 8 heads 11 / 9, of 128 + 8 19 / 11; 1184 rows 14 / 14 and 27 / 23; 2368 rows 16 / 18 and 37 / 35; 9472 rows 40 / 48 and 111 / 107.
    g.lanes = rows >= (long long)device_sm_count() * 8 ? 8 : heads;
    if (g.lanes > slots) g.lanes = slots;
    g.rows = slots / g.lanes;
    if (g.rows > kRotEntries / pairs) g.rows = kRotEntries / pairs;
    return g;
}

}  // namespace beagle

using namespace beagle;

extern "C" {

beagle_status beagle_rotary_make(int32_t head_dim, int32_t rot_dim, int32_t interleaved, double theta, int32_t scaling, double factor, double original,
                                 double low, double high, double mscale, beagle_rotary* out) {
    if (out == nullptr || head_dim <= 0 || rot_dim <= 0 || (interleaved != 0 && interleaved != 1)) return BEAGLE_ERR_INVALID_ARG;
    if (head_dim > 2 * BEAGLE_ROTARY_MAX_PAIRS || rot_dim > head_dim || rot_dim % 2) return BEAGLE_ERR_SHAPE;
    if (!std::isfinite(theta) || !(theta > 1.0) || !finite_in_fp32(mscale) || mscale < 0.0) return BEAGLE_ERR_INVALID_ARG;
    if (scaling < BEAGLE_ROTARY_NONE || scaling > BEAGLE_ROTARY_RAMP) return BEAGLE_ERR_INVALID_ARG;
    if (scaling != BEAGLE_ROTARY_NONE && (!std::isfinite(factor) || !(factor >= 1.0))) return BEAGLE_ERR_INVALID_ARG;
    const bool by_turns = scaling == BEAGLE_ROTARY_BANDS || scaling == BEAGLE_ROTARY_RAMP;
    if (by_turns && (!std::isfinite(original) || !(original > 0.0) || !std::isfinite(high) || !(low > 0.0) || !(high > low))) return BEAGLE_ERR_INVALID_ARG;
    if (scaling == BEAGLE_ROTARY_BASE && rot_dim == 2) return BEAGLE_ERR_SHAPE;          // the exponent r / (r - 2) needs more than one pair
    const double two_pi = 6.283185307179586476925, r = rot_dim;
    memset(out, 0, sizeof(*out));
    out->head_dim = head_dim;
    out->rot_dim = rot_dim;
    out->interleaved = interleaved;
    out->mscale = mscale > 0.0 ? mscale : scaling == BEAGLE_ROTARY_RAMP ? 0.1 * std::log(factor) + 1.0 : 1.0;
    if (scaling == BEAGLE_ROTARY_BASE) theta *= std::pow(factor, r / (r - 2.0));
    double first = 0.0, last = 1.0;                  // ramp: from pair `first` (kept) to pair `last` (divided by factor)
    if (scaling == BEAGLE_ROTARY_RAMP) {
        first = std::fmax(std::floor(r * std::log(original / (two_pi * high)) / (2.0 * std::log(theta))), 0.0);
        last = std::fmin(std::ceil(r * std::log(original / (two_pi * low)) / (2.0 * std::log(theta))), r - 1.0);
        last = std::fmax(last, first + 0.001);
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(theta, -2.0 * i / r);
        if (scaling == BEAGLE_ROTARY_LINEAR) f /= factor;
        if (by_turns) {
            const double at = scaling == BEAGLE_ROTARY_BANDS ? (original * f / two_pi - low) / (high - low) : (last - i) / (last - first);
            const double keep = std::fmin(std::fmax(at, 0.0), 1.0);
            f *= keep + (1.0 - keep) / factor;
        }
        out->freq[i] = f;
    }
    return BEAGLE_OK;
}

beagle_status beagle_rotary_apply(const beagle_rotary* rot, int32_t dtype, int64_t rows, const int32_t* pos_dev, int32_t pos0, int64_t period,
                                  int32_t n_q_heads, const void* q_dev, int64_t q_stride, void* q_out_dev, int64_t q_out_stride, int32_t n_k_heads,
                                  const void* k_dev, int64_t k_stride, void* k_out_dev, int64_t k_out_stride, int32_t inverse, void* stream_) {
    const beagle_status st = rotary_check(rot, dtype);
    if (st != BEAGLE_OK) return st;
    if (rows < 0 || n_q_heads < 0 || n_k_heads < 0 || n_q_heads + (int64_t)n_k_heads == 0 || period < 0) return BEAGLE_ERR_INVALID_ARG;
    if (n_q_heads > 65535 || n_k_heads > 65535) return BEAGLE_ERR_SHAPE;
    if (rows == 0) return BEAGLE_OK;
    const int e = dtype == BEAGLE_BF16 ? 2 : 4;
    const int64_t strides[4] = {q_stride, q_out_stride, k_stride, k_out_stride};
    const void* ptrs[4] = {q_dev, q_out_dev, k_dev, k_out_dev};
    for (int i = 0; i < 4; ++i) {
        const int heads = i < 2 ? n_q_heads : n_k_heads;
        if (heads == 0) continue;
        if (ptrs[i] == nullptr || strides[i] < (int64_t)heads * rot->head_dim) return BEAGLE_ERR_INVALID_ARG;
        if (((uintptr_t)ptrs[i] & 15) || strides[i] * e % 16) return BEAGLE_ERR_INVALID_ARG;
    }
    // in place means exactly in place
    if (n_q_heads > 0 && q_dev == q_out_dev && q_stride != q_out_stride) return BEAGLE_ERR_INVALID_ARG;
    if (n_k_heads > 0 && k_dev == k_out_dev && k_stride != k_out_stride) return BEAGLE_ERR_INVALID_ARG;
    if ((uintptr_t)pos_dev & 3) return BEAGLE_ERR_INVALID_ARG;
    RotaryArgs r;
    rotary_args(rot, inverse, &r);
    RotaryRows a;
    memset(&a, 0, sizeof(a));
    a.q = q_dev; a.k = k_dev; a.q_out = q_out_dev; a.k_out = k_out_dev;
    a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
    a.pos = pos_dev; a.rows = rows; a.period = period > 0 ? period : rows; a.pos0 = pos0;
    a.Hq = n_q_heads; a.Hk = n_k_heads; a.dh = rot->head_dim;
    if (a.Hq == 0) { a.q = k_dev; a.q_out = k_out_dev; a.q_stride = a.q_out_stride = 0; }       // never read: no head maps there
    if (a.Hk == 0) { a.k = q_dev; a.k_out = q_out_dev; a.k_stride = a.k_out_stride = 0; }
    if (pos_dev == nullptr && (long long)pos0 + (a.period < rows ? a.period : rows) - 1 > 0x7fffffffll) return BEAGLE_ERR_CAPACITY;
    a.g = rotary_grid(rot, dtype, rows, n_q_heads + n_k_heads);
    const long long grid = (rows + a.g.rows - 1) / a.g.rows;
    if (grid > 0x7fffffffll) return BEAGLE_ERR_CAPACITY;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
#define BEAGLE_ROTARY_LAUNCH(T, E, INTER) launch_pdl(rotary_kernel<T, E, INTER>, dim3((unsigned)grid), dim3(kRotThreads), 0, stream, r, a)
    if (dtype == BEAGLE_BF16) BEAGLE_ROTARY_DISPATCH(bf16, rotary_unit(rot, dtype), rot->interleaved, BEAGLE_ROTARY_LAUNCH);
    else BEAGLE_ROTARY_DISPATCH(float, rotary_unit(rot, dtype), rot->interleaved, BEAGLE_ROTARY_LAUNCH);
#undef BEAGLE_ROTARY_LAUNCH
    return cudaGetLastError() == cudaSuccess ? BEAGLE_OK : BEAGLE_ERR_CUDA;
}

}  // extern "C"
