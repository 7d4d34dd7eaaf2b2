// Rotary positions on the device.  Pair i of a token at position p turns by the angle p f_i (Su et al. 2021):
//   x' = s (x cos a - y sin a),  y' = s (y cos a + x sin a).
//
// Everything is held in 64 bits until the result is rounded to float: at position 131072 an angle in 32 bits is 2^-8 off,
// and a key on its way into 4 or 8 bits falls on the same side of a border whoever computes it.  The vector unit's 64-bit
// products cost what its 32-bit ones do.
#pragma once

#include "sekv_page_store.h"

namespace sekv {
namespace page {

// (cos, sin) of an angle.  k quarter turns are taken off with pi / 2 in two parts, each product exact within its fused
// step, so that what is left is as exact as the angle; then the series up to x^15 and x^16, whose next terms are below
// 2^-54 at pi / 4.  Up to 2^50 quarter turns the quotient's roundings leave k at most a fifth beside the nearest one, and
// the next terms below 2^-46; angles past that, which a double holds to a quarter at best, are no number.
__device__ inline double2 cos_sin(double angle) {
    double k = __builtin_rint(angle * 0.63661977236758134308);
    const bool far = !(fabs(k) < 1125899906842624.0);
    k = far ? 0.0 : k;
    const double left = fma(-k, 6.123233995736766036e-17, fma(-k, 1.57079632679489661923, angle));
    const double r = far ? __builtin_nan("") : left, z = r * r;
    double s = -1.0 / 1307674368000.0;
    s = fma(s, z, 1.0 / 6227020800.0);
    s = fma(s, z, -1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, -1.0 / 5040.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, -1.0 / 6.0);
    s = fma(s * z, r, r);
    double c = 1.0 / 20922789888000.0;
    c = fma(c, z, -1.0 / 87178291200.0);
    c = fma(c, z, 1.0 / 479001600.0);
    c = fma(c, z, -1.0 / 3628800.0);
    c = fma(c, z, 1.0 / 40320.0);
    c = fma(c, z, -1.0 / 720.0);
    c = fma(c, z, 1.0 / 24.0);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const int q = int(k - 4.0 * __builtin_floor(0.25 * k));
    const double a = q & 1 ? s : c, b = q & 1 ? c : s;
    return make_double2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

// A lane's part of turning a row: its piece of kN values, each with its pair's cos and sin.  In the half layout the pair's
// other value is in the lane `other` of the wave, in the interleaved one beside it.  Pieces behind rot_dim stay.
template <class T, int D, bool kHalf>
struct Turn {
    static constexpr int N = Piece<T>::kN, M = kHalf ? N : N / 2, L = D / N;
    double c[M], s[M];
    int other;
    bool on;

    // pairs: (cos, sin) of the row's token, rot_dim / 2 of them
    __device__ void init(const double2 *pairs, int rot_dim, int lane) {
        const int half = rot_dim / 2 / N;                    // pieces of the first half
        on = lane * N < rot_dim;
        const bool second = kHalf && on && lane >= half;
        other = int(threadIdx.x & 63u) + (!kHalf || !on ? 0 : second ? -half : half);
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const double2 p = pairs[!on ? 0 : kHalf ? (second ? lane - half : lane) * N + i : lane * M + i];
            c[i] = p.x;
            s[i] = kHalf && !second ? -p.y : p.y;
        }
    }
    // by all lanes of a wave together
    __device__ Computed<T> apply(const u4v &w) const {
        float x[N];
        Piece<T>{w}.up(x);
        Computed<T> r;
        if constexpr (kHalf) {
            u4v o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __shfl(w[i], other);
            float y[N];
            Piece<T>{o}.up(y);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float t = float(fma(double(y[i]), s[i], double(x[i]) * c[i]));
                r.x[i] = on ? t : x[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const double u = x[2 * i], v = x[2 * i + 1];
                const float a = float(fma(-v, s[i], u * c[i])), b = float(fma(u, s[i], v * c[i]));
                r.x[2 * i] = on ? a : x[2 * i];
                r.x[2 * i + 1] = on ? b : x[2 * i + 1];
            }
        }
        return r;
    }
};

}  // namespace page
}  // namespace sekv
