// Rows of queries and keys divided by their root mean square, times a weight per dimension, in front of their turn:
//     y = w x r,  r = (mean of x^2 + eps)^(-1/2),
// for the kernels whose lanes hold a row by groups of pairs (rotary.h).  Everything between the loaded row and the stored one is fp32.
#pragma once

#include <type_traits>

#include "rotary.h"

namespace sepattn {

// sum over the LANES (4, 8 or 16) neighbouring lanes that hold one row; every one of them gets it
template <int LANES>
__device__ inline float row_sum(float x) {
    static_assert(LANES == 4 || LANES == 8 || LANES == 16, "");
    auto plus = [](float y, auto CTRL) {
        return y + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), decltype(CTRL)::value, 0xF, 0xF, true));
    };
    x = plus(x, std::integral_constant<int, 0xB1>{});                             // quad_perm [1, 0, 3, 2]
    x = plus(x, std::integral_constant<int, 0x4E>{});                             // quad_perm [2, 3, 0, 1]
    if constexpr (LANES >= 8) x = plus(x, std::integral_constant<int, 0x141>{});  // row_half_mirror
    if constexpr (LANES == 16) x = plus(x, std::integral_constant<int, 0x140>{}); // row_mirror
    return x;
}

// a weight per dimension (NormWeight, common.h), the same for all heads
template <typename T, PairLayout LAYOUT>
struct Weights {
    static constexpr int E = 16 / (int)sizeof(T);
    float u[E], v[E];
    __device__ void load(const NormWeight &w, int group, int n_pairs, int half) {
        if (!w.w) {
#pragma unroll
            for (int e = 0; e < E; ++e) u[e] = v[e] = 1.f;
        } else if (w.dtype == SEPATTN_BF16) {
            load_from(static_cast<const uint16_t *>(w.w), group, n_pairs, half);
        } else {
            load_from(static_cast<const float *>(w.w), group, n_pairs, half);
        }
    }

private:
    template <typename W>
    __device__ void load_from(const W *w, int group, int n_pairs, int half) {
        if constexpr (LAYOUT == kHalvesOdd) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                int i, j;
                members_of<LAYOUT, E>(group, e, n_pairs, half, i, j);
                u[e] = widened(w[i]), v[e] = widened(w[j]);
            }
        } else {  // two pieces of E values, as Pairs has them
            int first;
            const int second = Pairs<T, LAYOUT>::second_piece(group, n_pairs, half, first);
            const W *a = w + first, *b = w + second;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if constexpr (LAYOUT == kNeighbours) {
                    const W *r = e < E / 2 ? a : b;
                    u[e] = widened(r[2 * e % E]), v[e] = widened(r[2 * e % E + 1]);
                } else {
                    u[e] = widened(a[e]), v[e] = widened(b[e]);
                }
            }
        }
    }
};

// 1 / root mean square of a row of which this lane holds u, v
template <int D, int LANES, int E>
__device__ inline float row_rms(const float (&u)[E], const float (&v)[E], float eps) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(u[e], u[e], fmaf(v[e], v[e], ss));
    return rsqrtf(fmaf(row_sum<LANES>(ss), 1.f / D, eps));
}

// the pairs that are turned, by their angles (back: Angles formed with sign -1)
template <typename T, PairLayout LAYOUT, int E>
__device__ inline void turn_pairs(float (&u)[E], float (&v)[E], const Angles<T, LAYOUT> &w, int group, int n_pairs, int half) {
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (pair_of<LAYOUT, E>(group, e, half) < n_pairs) {
            const float x = u[e], y = v[e];
            u[e] = fmaf(x, w.cs[e], -(y * w.sn[e]));
            v[e] = fmaf(y, w.cs[e], x * w.sn[e]);
        }
}

// a row normed, and turned where it is
template <typename T, PairLayout LAYOUT, int D, int LANES>
__device__ inline void norm_and_turn(Pairs<T, LAYOUT> &row, const Weights<T, LAYOUT> &g, const Angles<T, LAYOUT> &w, float eps, bool turned,
                                     int group, int n_pairs) {
    constexpr int E = 16 / (int)sizeof(T);
    float u[E], v[E];
    row.widen(u, v);
    const float r = row_rms<D, LANES>(u, v, eps);
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] *= r * g.u[e], v[e] *= r * g.v[e];
    if (turned) turn_pairs(u, v, w, group, n_pairs, D / 2);
    row.narrow(u, v);
}

}  // namespace sepattn
