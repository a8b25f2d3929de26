// Pieces shared by the kernels that turn pairs of dimensions by positions (rope.hip, cache_append.hip).
//
// A row of d values is cut into groups of 16 bytes worth of pairs: group j holds pairs E j .. E j + E - 1 (E = 8 in bf16, 4 in
// fp32), every group is one lane's, and a lane reads both members of its pairs before it writes any, so a turn may be in place.
// Pair p of the first rotary_dim / 2 is (p, p + rotary_dim/2), or (2p, 2p+1) where interleaved; the others are the values
// 2p, 2p+1, which are copied bit for bit.
#pragma once

#include "common.h"

namespace sepattn {

enum PairLayout {
    kNeighbours,  // (2p, 2p+1): a group is 32 contiguous bytes
    kHalves,      // (p, p + rotary_dim/2), rotary_dim/2 a multiple of E: a group is two runs of 16 bytes
    kHalvesOdd,   // the same with any even rotary_dim: value by value
};
template <typename T>
inline int pair_layout(int rotary_dim, int interleaved) {
    if (interleaved) return kNeighbours;
    return (rotary_dim / 2) % (16 / (int)sizeof(T)) == 0 ? kHalves : kHalvesOdd;
}

__device__ inline float widened(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ inline float widened(float x) { return x; }
template <typename T>
__device__ inline T narrowed(float x);
template <>
__device__ inline float narrowed<float>(float x) { return x; }
template <>
__device__ inline uint16_t narrowed<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }  // to nearest even

// cos and sin of the angle at position t of a pair with frequency f (radians per position).  The angle is brought to turns and to
// [-1/2, 1/2] in fp64: in fp32 a position of 4 million would be off by a quarter of a radian.
__device__ inline void angle_of(int t, double f, float &cs, float &sn) {
    double turns = (double)t * (f * 0.15915494309189533577);
    turns -= rint(turns);
    sincospif((float)(turns + turns), &sn, &cs);
}

// cos / sin of the E pairs of a group at one position
template <typename T>
struct Angles {
    static constexpr int E = 16 / (int)sizeof(T);
    float cs[E], sn[E];
    // sign -1: the opposite angles.  Pairs from n_pairs on are not looked at later.
    __device__ void form(const double *__restrict__ freqs, int n_pairs, int group, int t, float sign) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            angle_of(t, freqs[min(group * E + e, n_pairs - 1)], cs[e], sn[e]);
            sn[e] *= sign;
        }
    }
};

// the 2 E values of a group: x[e], y[e] are pair e's
template <typename T>
struct Pairs {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T Run __attribute__((ext_vector_type(16 / sizeof(T))));
    Run a, b;  // as they lie: two runs of 16 bytes (kHalves: the first and the second members; else neighbouring values)

    template <PairLayout LAYOUT>
    __device__ static int first(int group, int n_pairs, int e) {  // place of pair e's first member
        const int p = group * E + e;
        return LAYOUT != kNeighbours && p < n_pairs ? p : 2 * p;
    }
    template <PairLayout LAYOUT>
    __device__ void load(const T *row, int group, int n_pairs) {
        if constexpr (LAYOUT == kHalvesOdd) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int at = first<LAYOUT>(group, n_pairs, e);
                a[e] = row[at];
                b[e] = row[group * E + e < n_pairs ? at + n_pairs : at + 1];
            }
        } else {
            const bool halves = LAYOUT == kHalves && group * E < n_pairs;
            const T *p = row + (halves ? group * E : 2 * group * E);
            a = *reinterpret_cast<const Run *>(p);
            b = *reinterpret_cast<const Run *>(p + (halves ? n_pairs : E));
        }
    }
    template <PairLayout LAYOUT>
    __device__ void store(T *row, int group, int n_pairs) const {
        if constexpr (LAYOUT == kHalvesOdd) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int at = first<LAYOUT>(group, n_pairs, e);
                row[at] = a[e];
                row[group * E + e < n_pairs ? at + n_pairs : at + 1] = b[e];
            }
        } else {
            const bool halves = LAYOUT == kHalves && group * E < n_pairs;
            T *p = row + (halves ? group * E : 2 * group * E);
            *reinterpret_cast<Run *>(p) = a;
            *reinterpret_cast<Run *>(p + (halves ? n_pairs : E)) = b;
        }
    }
    template <PairLayout LAYOUT>
    __device__ void turn(const Angles<T> &w, int group, int n_pairs) {
        Run x = a, y = b;
        if constexpr (LAYOUT == kNeighbours) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = 2 * e < E ? a[(2 * e) % E] : b[(2 * e) % E];
                y[e] = 2 * e < E ? a[(2 * e + 1) % E] : b[(2 * e + 1) % E];
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float u = widened((T)x[e]), v = widened((T)y[e]);
            // (a select, not an angle of 0: 0 times an infinity next to it would be NaN)
            if (group * E + e < n_pairs) {
                x[e] = narrowed<T>(fmaf(u, w.cs[e], -(v * w.sn[e])));
                y[e] = narrowed<T>(fmaf(v, w.cs[e], u * w.sn[e]));
            }
        }
        if constexpr (LAYOUT == kNeighbours) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (2 * e < E) {
                    a[(2 * e) % E] = x[e];
                    a[(2 * e + 1) % E] = y[e];
                } else {
                    b[(2 * e) % E] = x[e];
                    b[(2 * e + 1) % E] = y[e];
                }
            }
        } else {
            a = x, b = y;
        }
    }
};

}  // namespace sepattn
