// Pieces shared by the kernels that turn pairs of dimensions by positions (rope.hip, cache_append.hip).
//
// A row of d values is cut into groups of two pieces of 16 bytes, E pairs (E = 8 in bf16, 4 in fp32); every group is one lane's, and a lane
// reads both members of its pairs before it writes any, so a turn may be in place.  Pair p of the first rotary_dim / 2 is
// (p, p + rotary_dim/2), or (2p, 2p+1) where interleaved; the others are the values 2p, 2p+1, which are copied bit for bit.
#pragma once

#include "common.h"

namespace sepattn {

enum PairLayout {
    kNeighbours,  // (2p, 2p+1): a lane's pieces are the same place in the two halves of the row, so that a load instruction covers half a row
    kHalves,      // (p, p + rotary_dim/2), rotary_dim/2 a multiple of E: a piece of first members, the piece of their partners
    kHalvesOdd,   // the same with any even rotary_dim: value by value, so that rows have not to be regrouped, and slow (8192 tokens, 32/8 heads, d = 128, bf16:
                  // rotary_dim 20 178 us, 100 129; 16 and 96, by pieces, 44; 128 37; neighbours with any 36.  fp32, 4096 tokens, 100: 68, neighbours 35)
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

// Which pair element e of a group is; `half` = d / 2
template <PairLayout LAYOUT, int E>
__device__ inline int pair_of(int group, int e, int half) {
    if (LAYOUT == kNeighbours) return (e < E / 2 ? group * (E / 2) : half / 2 + group * (E / 2) - E / 2) + e;
    return group * E + e;
}
// whether a group has a pair that is turned
template <PairLayout LAYOUT, int E>
__device__ inline bool has_turned(int group, int n_pairs) { return pair_of<LAYOUT, E>(group, 0, 0) < n_pairs; }

// where the members of pair e of a group stand in the row
template <PairLayout LAYOUT, int E>
__device__ inline void members_of(int group, int e, int n_pairs, int half, int &first, int &second) {
    const int p = pair_of<LAYOUT, E>(group, e, half);
    if (LAYOUT == kNeighbours) first = 2 * p, second = 2 * p + 1;
    else if (LAYOUT == kHalves && group * E >= n_pairs) first = 2 * group * E + e, second = first + E;  // a piece, and the piece behind it
    else if (p < n_pairs) first = p, second = p + n_pairs;
    else first = 2 * p, second = 2 * p + 1;
}

// cos / sin of the E pairs of a group at one position
template <typename T, PairLayout LAYOUT>
struct Angles {
    static constexpr int E = 16 / (int)sizeof(T);
    float cs[E], sn[E];
    // sign -1: the opposite angles.  Pairs from n_pairs on are not looked at later.  ONE_BY_ONE: in turn, for kernels that have no registers for all at once
    template <bool ONE_BY_ONE = false>
    __device__ void form(const double *__restrict__ freqs, int n_pairs, int half, int group, int t, float sign) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            angle_of(t, freqs[min(pair_of<LAYOUT, E>(group, e, half), n_pairs - 1)], cs[e], sn[e]);
            sn[e] *= sign;
            if constexpr (ONE_BY_ONE) __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// the 2 E values of a group
template <typename T, PairLayout LAYOUT>
struct Pairs {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T Run __attribute__((ext_vector_type(16 / sizeof(T))));
    Run a, b;  // kNeighbours: pieces of whole pairs; else first and second members

    static __device__ int second_piece(int group, int n_pairs, int half, int &first) {
        if (LAYOUT == kNeighbours) {
            first = group * E;
            return first + half;
        }
        const bool turned = group * E < n_pairs;
        first = turned ? group * E : 2 * group * E;
        return first + (turned ? n_pairs : E);
    }
    __device__ void clear() { a = b = Run(T(0)); }
    // STREAM: the non-temporal hint, for rows whose pieces one instruction reads by whole cache lines
    template <bool STREAM = false>
    __device__ void load(const T *row, int group, int n_pairs, int half) {
        if constexpr (LAYOUT == kHalvesOdd) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int p = group * E + e;
                a[e] = row[p < n_pairs ? p : 2 * p];
                b[e] = row[p < n_pairs ? p + n_pairs : 2 * p + 1];
            }
        } else {
            int first;
            const int second = second_piece(group, n_pairs, half, first);
            const Run *pa = reinterpret_cast<const Run *>(row + first), *pb = reinterpret_cast<const Run *>(row + second);
            a = STREAM ? __builtin_nontemporal_load(pa) : *pa;
            b = STREAM ? __builtin_nontemporal_load(pb) : *pb;
        }
    }
    __device__ void store(T *row, int group, int n_pairs, int half) const {
        if constexpr (LAYOUT == kHalvesOdd) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int p = group * E + e;
                row[p < n_pairs ? p : 2 * p] = a[e];
                row[p < n_pairs ? p + n_pairs : 2 * p + 1] = b[e];
            }
        } else {
            int first;
            const int second = second_piece(group, n_pairs, half, first);
            *reinterpret_cast<Run *>(row + first) = a;
            *reinterpret_cast<Run *>(row + second) = b;
        }
    }
    // first and second members in fp32, and back (rounded to nearest even)
    __device__ void widen(float (&u)[E], float (&v)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (LAYOUT == kNeighbours) {
                const Run &r = e < E / 2 ? a : b;
                u[e] = widened(r[2 * e % E]), v[e] = widened(r[2 * e % E + 1]);
            } else {
                u[e] = widened(a[e]), v[e] = widened(b[e]);
            }
        }
    }
    __device__ void narrow(const float (&u)[E], const float (&v)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (LAYOUT == kNeighbours) {
                Run &r = e < E / 2 ? a : b;
                r[2 * e % E] = narrowed<T>(u[e]), r[2 * e % E + 1] = narrowed<T>(v[e]);
            } else {
                a[e] = narrowed<T>(u[e]), b[e] = narrowed<T>(v[e]);
            }
        }
    }
    __device__ void turn(const Angles<T, LAYOUT> &w, int group, int n_pairs, int half) {
        auto one = [&](int e, T &x, T &y) {
            const float u = widened(x), v = widened(y);
            // (a select, not an angle of 0: 0 times an infinity next to it would be NaN)
            if (pair_of<LAYOUT, E>(group, e, half) < n_pairs) {
                x = narrowed<T>(fmaf(u, w.cs[e], -(v * w.sn[e])));
                y = narrowed<T>(fmaf(v, w.cs[e], u * w.sn[e]));
            }
        };
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (LAYOUT == kNeighbours) {
                Run &r = e < E / 2 ? a : b;
                T x = r[2 * e % E], y = r[2 * e % E + 1];
                one(e, x, y);
                r[2 * e % E] = x, r[2 * e % E + 1] = y;
            } else {
                T x = a[e], y = b[e];
                one(e, x, y);
                a[e] = x, b[e] = y;
            }
        }
    }
};

}  // namespace sepattn
