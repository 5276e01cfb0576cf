// Rotary positions: what the rotation of whole rows (rotary.cu) and the append that rotates on the way (pages.cu) share.
//
// A pair (x_a, x_b) of a head at position p becomes  m (c x_a - s x_b, s x_a + c x_b),  c + i s = exp(i p f),  for the rot_dim / 2
// frequencies f; pair i is (i, i + rot_dim / 2), or (2i, 2i + 1) in the interleaved layout, and components from rot_dim on pass.
// The angle is formed in turns, p * f / 2 pi, in double precision and reduced to [-1/2, 1/2] there: in fp32 the product alone
// would be off by 2^-24 of the angle, a quarter of a turn at position 10^6 times a few.  Cosine and sine of the reduced turn are fp32.
#pragma once
#include "../../include/beagle.h"
#include "common.cuh"

namespace beagle {

struct RotaryArgs {                      // by value in the kernel parameters
    double turns[BEAGLE_ROTARY_MAX_PAIRS];       // f / 2 pi
    float m;                             // factor of cosine and sine
    float sign;                          // -1: the transpose
    int pairs, interleaved;
};

beagle_status rotary_check(const beagle_rotary* r, int dtype);                  // the structure's own values, and the head for this type
void rotary_args(const beagle_rotary* r, int inverse, RotaryArgs* out);
// Elements of a unit (see below) for this head and type: 16 bytes where the layout allows it.
int rotary_unit(const beagle_rotary* r, int dtype);

constexpr int kRotThreads = 256;
constexpr int kRotEntries = 2048;        // (cosine, sine) entries of a CTA in shared memory
constexpr int kRotCtas = 6;              // per SM: a thread has one or two 16-byte pieces in flight, the rest is up to the number of threads

// How a CTA of kRotThreads divides `rows` rows of `heads` heads: `units` threads share a head, `lanes` heads of a row are worked on
// side by side, `rows` rows.
struct RotaryGrid { int units, lanes, rows; };
RotaryGrid rotary_grid(const beagle_rotary* r, int dtype, long long rows, int heads);

// Elements [at, at + E) of a head.
template <typename T, int E> struct RotVec;
template <> struct RotVec<bf16, 8> { typedef uint4 type; };
template <> struct RotVec<bf16, 4> { typedef uint2 type; };
template <> struct RotVec<bf16, 2> { typedef uint32_t type; };
template <> struct RotVec<bf16, 1> { typedef uint16_t type; };
template <> struct RotVec<float, 4> { typedef uint4 type; };
template <> struct RotVec<float, 2> { typedef uint2 type; };
template <> struct RotVec<float, 1> { typedef uint32_t type; };

template <typename T, int E>
__device__ __forceinline__ void rot_unpack(const typename RotVec<T, E>::type& v, float* f) {
    T x[E];
    *reinterpret_cast<typename RotVec<T, E>::type*>(x) = v;
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = to_float<T>(x[i]);
}
template <typename T, int E>
__device__ __forceinline__ typename RotVec<T, E>::type rot_pack(const float* f) {
    alignas(16) T x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = from_float<T>(f[i]);
    return *reinterpret_cast<typename RotVec<T, E>::type*>(x);
}

// (cosine, sine) of pair i at position pos.
__device__ __forceinline__ float2 rot_angle(double turns, int pos, float m, float sign) {
    double t = (double)pos * turns;
    t -= rint(t);
    float s, c;
    sincospif(2.f * (float)t, &s, &c);
    return make_float2(c * m, s * m * sign);
}

// A unit is what one thread does of a head: E elements, or E and their partners rot_dim / 2 further on.
//   half layout:  unit u < pairs / E: elements [uE, uE + E) and [pairs + uE, ..);  the others: E elements that pass, from 2 pairs on
//   interleaved:  unit u: elements [uE, uE + E), of which those below 2 pairs are rotated
template <typename T, int E, bool INTER>
struct RotUnit {
    typedef typename RotVec<T, E>::type V;
    static constexpr int kCs = INTER ? (E + 1) / 2 : E;
    float2 cs[kCs];
    int at, partner;                     // element offsets; partner < 0: none
    bool rotates;
    int count;                           // interleaved: pairs of the unit that are rotated
    __device__ __forceinline__ void place(int u, int pairs) {
        partner = -1;
        count = 0;
        if (INTER) {
            at = u * E;
            rotates = at < 2 * pairs;
            count = min(kCs, pairs - at / 2);
        } else {
            const int n = pairs / E;
            rotates = u < n;
            at = rotates ? u * E : 2 * pairs + (u - n) * E;
            partner = rotates ? at + pairs : -1;
        }
    }
    // cs_row: the row's (cosine, sine) entries
    __device__ __forceinline__ void entries(const float2* cs_row) {
        const int first = INTER ? at / 2 : at, n = INTER ? count : kCs;
#pragma unroll
        for (int i = 0; i < kCs; ++i) cs[i] = rotates && i < n ? cs_row[first + i] : make_float2(1.f, 0.f);
    }
    __device__ __forceinline__ void load(const T* head, V& x, V& y) const {
        x = *reinterpret_cast<const V*>(head + at);
        if (!INTER && rotates) y = *reinterpret_cast<const V*>(head + partner);
    }
    __device__ __forceinline__ void store(T* head, const V& x, const V& y) const {
        *reinterpret_cast<V*>(head + at) = x;
        if (!INTER && rotates) *reinterpret_cast<V*>(head + partner) = y;
    }
    __device__ __forceinline__ void turn(V& x, V& y) const {
        if (!rotates) return;
        float a[E], b[E];
        rot_unpack<T, E>(x, a);
        if (INTER) {
            const V was = x;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                b[2 * i] = a[2 * i] * cs[i].x - a[2 * i + 1] * cs[i].y;
                b[2 * i + 1] = a[2 * i + 1] * cs[i].x + a[2 * i] * cs[i].y;
            }
            x = rot_pack<T, E>(b);
            if (count < kCs) {           // the last rotated unit: what lies past the rotated pairs passes as it is
                alignas(16) T n[E], o[E];
                *reinterpret_cast<V*>(n) = x;
                *reinterpret_cast<V*>(o) = was;
#pragma unroll
                for (int i = 0; i < E; ++i) n[i] = i < 2 * count ? n[i] : o[i];
                x = *reinterpret_cast<V*>(n);
            }
        } else {
            float c[E], d[E];
            rot_unpack<T, E>(y, b);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                c[i] = a[i] * cs[i].x - b[i] * cs[i].y;
                d[i] = b[i] * cs[i].x + a[i] * cs[i].y;
            }
            x = rot_pack<T, E>(c);
            y = rot_pack<T, E>(d);
        }
    }
};

// Calls f<E, INTER>() for the unit of this head and type.
#define BEAGLE_ROTARY_DISPATCH(T, unit, inter, F)                                                   \
    do {                                                                                            \
        constexpr int kFull = 16 / (int)sizeof(T);                                                  \
        if (inter) F(T, kFull, true);                                                               \
        else if ((unit) == kFull) F(T, kFull, false);                                               \
        else if ((unit) == 4 && kFull > 4) F(T, (kFull > 4 ? 4 : 1), false);                        \
        else if ((unit) == 2) F(T, 2, false);                                                       \
        else F(T, 1, false);                                                                        \
    } while (0)

}  // namespace beagle
