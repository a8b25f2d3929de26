// The four-block KV cache in 4 bits (fp4.h): codes [S, Hkv, c, d/2] and scale bytes [S, Hkv, c, d/32] of keys and of values.
//
//   fill     a prompt's kept rows, rounded on the way (cache_fill.hip says which)
//   append   a token's key and value, as they are or normed and turned first (rotary.h, norm.h)
//   expand   the values that a cache stands for, in a plain cache
// Eight consecutive values of a row are one lane's: the largest magnitude of a block of 32 is found over four neighbouring lanes, each lane
// leaves four bytes of codes and the first one of a row its scale bytes.
#include "decode_common.h"
#include "fp4.h"
#include "norm.h"

namespace sepattn {

namespace {

constexpr int kThreads = 256;
// Cache slots per workgroup and rows that a thread has in flight.  8 sequences, 8 KV heads of 128, bf16, 3332 slots: the hand-over takes 21.2 us with 64 slots
// and 4 rows, 23.6 with 32 and 2 or 256 and 8;  in fp32, 3 sequences, 12 heads of 64, 601 slots 5.4, 6.8 with 128 and 8.  The expansion 20.2 us with 32 and 2,
// 22.5 with 64 and 4, 23.8 with 128 and 8.
constexpr int kFillSlots = 64, kFillRows = 4;
constexpr int kExpandSlots = 32, kExpandRows = 2;

// eight values of T
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    uint4 x;
    __device__ void load(const uint16_t *p) { x = *reinterpret_cast<const uint4 *>(p); }
    __device__ void stream(const uint16_t *p) { x = nt_load(reinterpret_cast<const uint4 *>(p)); }
    __device__ void clear() { x = make_uint4(0u, 0u, 0u, 0u); }
    __device__ void from_fp4(uint32_t codes, float scale) { x = __builtin_bit_cast(uint4, fp4_to_bf16(codes, scale)); }
    __device__ void store(uint16_t *p) const { nt_store(x, reinterpret_cast<uint4 *>(p)); }
    template <int D>
    __device__ Fp4Piece round(int piece) const { return fp4_round<D>(x, piece); }
};
template <>
struct Eight<float> {
    uint4 x, y;
    __device__ void load(const float *p) { x = reinterpret_cast<const uint4 *>(p)[0], y = reinterpret_cast<const uint4 *>(p)[1]; }
    __device__ void stream(const float *p) { x = nt_load(reinterpret_cast<const uint4 *>(p)), y = nt_load(reinterpret_cast<const uint4 *>(p) + 1); }
    __device__ void clear() { x = y = make_uint4(0u, 0u, 0u, 0u); }
    __device__ void from_fp4(uint32_t codes, float scale) {
        float v[8];
        fp4_to_f32(codes, scale, v);
        auto b = [](float f) { return __float_as_uint(f); };
        x = make_uint4(b(v[0]), b(v[1]), b(v[2]), b(v[3])), y = make_uint4(b(v[4]), b(v[5]), b(v[6]), b(v[7]));
    }
    __device__ void store(float *p) const { nt_store(x, reinterpret_cast<uint4 *>(p)), nt_store(y, reinterpret_cast<uint4 *>(p) + 1); }
    template <int D>
    __device__ Fp4Piece round(int piece) const { return fp4_round<D>(x, y, piece); }
};

// a rounded piece -> its row of a head's cache
template <int D>
__device__ inline void put_piece(const Fp4Piece &f, uint32_t *codes, Fp4Scales<D> *scales, long slot, int piece) {
    codes[slot * (D / 8) + piece] = f.codes;
    if (piece == 0) scales[slot] = (Fp4Scales<D>)f.scales;
}

// ---- hand-over of a prompt -------------------------------------------------------------------------
// As cache_fill_kernel: which position a slot receives, and the sizes and window flags, are the same.
template <typename T, int D, bool ZERO>
__global__ __launch_bounds__(kThreads) void fill_fp4_kernel(sepkv_params p, int L, int nw, int cap, const T *__restrict__ K,
                                                             const T *__restrict__ V, const uint8_t *__restrict__ is_sep,
                                                             const int32_t *__restrict__ sep_idx, const int32_t *__restrict__ sep_prefix,
                                                             Fp4Cache cache, uint8_t *__restrict__ win_is_sep, int32_t *__restrict__ sizes) {
    const int which = blockIdx.y & 1, kv = (blockIdx.y >> 1) % p.Hkv, sq = (blockIdx.y >> 1) / p.Hkv;
    const int32_t *prefix = sep_prefix + (long)sq * (L + 1), *idx = sep_idx + (long)sq * cap;
    const int n_init = min(p.a, L), wstart = L - nw, wcap = p.c - p.a - p.s;
    const int seps_before = prefix[wstart], n_old = min(p.s, seps_before - prefix[n_init]);
    const int first_kept = seps_before - n_old, kept = min(n_old, max(cap - first_kept, 0));  // listed ones only
    if (blockIdx.x == 0 && kv == 0 && which == 0) {
        const int wl = min(p.w, nw);
        if (threadIdx.x == 0) {
            int32_t *sz = sizes + SEPKV_SIZES_COLS * sq;
            sz[0] = n_init, sz[1] = kept, sz[2] = nw - wl, sz[3] = wl, sz[4] = 0, sz[5] = 0;
        }
        for (int u = threadIdx.x; u < (ZERO ? wcap : nw); u += kThreads)
            win_is_sep[(long)sq * wcap + u] = u < nw ? is_sep[(long)sq * L + wstart + u] : 0;
    }
    const long head = (long)sq * p.Hkv + kv;
    const T *src = (which ? V : K) + head * L * D;
    uint32_t *codes = reinterpret_cast<uint32_t *>(which ? cache.Vc : cache.Kc) + head * p.c * (D / 8);
    Fp4Scales<D> *scales = reinterpret_cast<Fp4Scales<D> *>(which ? cache.Vs : cache.Ks) + head * p.c;
    constexpr int PIECES = D / 8, ROWS = kThreads / PIECES;
    const int r_in = threadIdx.x / PIECES, piece = threadIdx.x % PIECES, t_end = min((int)(blockIdx.x + 1) * kFillSlots, p.c);
    for (int t0 = blockIdx.x * kFillSlots; t0 < t_end; t0 += ROWS * kFillRows) {
        int from[kFillRows];  // source position of the slot, -1: the slot is not in use
#pragma unroll
        for (int u = 0; u < kFillRows; ++u) {
            const int t = t0 + u * ROWS + r_in;
            from[u] = -1;
            if (t >= t_end) continue;
            if (t < p.a) {
                if (t < n_init) from[u] = t;
            } else if (t < p.a + p.s) {
                // the clamp keeps a stale list entry from faulting
                if (t - p.a < kept) from[u] = min(max(idx[first_kept + t - p.a], 0), L - 1);
            } else if (t - p.a - p.s < nw) {
                from[u] = wstart + t - p.a - p.s;
            }
        }
        Eight<T> v[kFillRows];
#pragma unroll
        for (int u = 0; u < kFillRows; ++u) {
            v[u].clear();
            if (from[u] >= 0) v[u].stream(src + (long)from[u] * D + piece * 8);
        }
#pragma unroll
        for (int u = 0; u < kFillRows; ++u) {
            const int t = t0 + u * ROWS + r_in;
            Fp4Piece f = v[u].template round<D>(piece);  // (all lanes of a row take part)
            if (from[u] < 0) f = {0u, 0u};
            if (from[u] >= 0 || (ZERO && t < t_end)) put_piece<D>(f, codes, scales, t, piece);
        }
    }
}

// ---- a token -----------------------------------------------------------------------------------------
enum TokenMode { kAsIs, kTurn, kNormTurn };

// Workgroup (s, 0): key and value; (s, 1): the query, where it is turned.  Turned rows pass through LDS in T, as they would stand in a plain
// cache: a lane's pairs lie in two pieces of the row, the blocks of 32 in four neighbouring ones.
template <typename T, int D, PairLayout LAYOUT, TokenMode MODE>
__global__ __launch_bounds__(kThreads) void append_fp4_kernel(sepkv_params p, int n_pairs, float eps, const double *__restrict__ freqs,
                                                               const int32_t *__restrict__ positions, NormWeight q_weight, NormWeight k_weight,
                                                               const T *q, const T *__restrict__ k_new, const T *__restrict__ v_new,
                                                               const uint8_t *__restrict__ is_sep_new, T *q_out, Fp4Cache cache,
                                                               uint8_t *__restrict__ win_is_sep, int32_t *__restrict__ sizes) {
    constexpr int E = 16 / (int)sizeof(T), GROUPS = D / (2 * E), ROWS = kThreads / GROUPS;
    const long sq = blockIdx.x;
    const int group = threadIdx.x % GROUPS, row = threadIdx.x / GROUPS;
    const bool turned = MODE != kAsIs && has_turned<LAYOUT, E>(group, n_pairs);
    Angles<T, LAYOUT> w;
    Weights<T, LAYOUT> weight;
    auto change = [&](Pairs<T, LAYOUT> &x) {
        if constexpr (MODE == kNormTurn) norm_and_turn<T, LAYOUT, D, GROUPS>(x, weight, w, eps, turned, group, n_pairs);
        else if (turned) x.turn(w, group, n_pairs, D / 2);
    };
    auto angles = [&] {
        if (turned) w.form(freqs, n_pairs, D / 2, group, positions[sq], 1.f);
    };
    if (MODE != kAsIs && blockIdx.y == 1) {
        if constexpr (MODE == kNormTurn) weight.load(q_weight, group, n_pairs, D / 2);
        angles();
        for (int h = row; h < p.Hq; h += ROWS) {
            Pairs<T, LAYOUT> x;
            x.load(q + (sq * p.Hq + h) * D, group, n_pairs, D / 2);
            change(x);
            x.store(q_out + (sq * p.Hq + h) * D, group, n_pairs, D / 2);
        }
        return;
    }
    int32_t *sz = sizes + SEPKV_SIZES_COLS * sq;
    const CacheMap cm = cache_map(p, sz);
    const int u = cm.n_past + cm.n_loc;
    __syncthreads();  // every thread has the old sizes before thread 0 replaces them
    int slot;
    if (cm.n_init < p.a) slot = cm.n_init;
    else if (u < cm.wcap) slot = p.a + p.s + win_index(cm, u);
    else return;  // window region full (uniform over the workgroup)
    constexpr int PIECES = D / 8, ROWS4 = kThreads / PIECES;
    const int piece = threadIdx.x % PIECES, row4 = threadIdx.x / PIECES;
    auto enter = [&](const Eight<T> &x, int i) {  // row i: keys, then values
        const bool value = i >= p.Hkv;
        const long at = (sq * p.Hkv + (value ? i - p.Hkv : i)) * p.c + slot;
        put_piece<D>(x.template round<D>(piece), reinterpret_cast<uint32_t *>(value ? cache.Vc : cache.Kc),
                     reinterpret_cast<Fp4Scales<D> *>(value ? cache.Vs : cache.Ks), at, piece);
    };
    const int first = MODE == kAsIs ? 0 : p.Hkv;  // rows from here on are rounded as they come
    if constexpr (MODE != kAsIs) {
        __shared__ __attribute__((aligned(16))) T rows[ROWS][D];
        if constexpr (MODE == kNormTurn) weight.load(k_weight, group, n_pairs, D / 2);
        angles();
        for (int h0 = 0; h0 < p.Hkv; h0 += ROWS) {
            const int n = min(ROWS, p.Hkv - h0);
            if (row < n) {
                Pairs<T, LAYOUT> x;
                x.load(k_new + (sq * p.Hkv + h0 + row) * D, group, n_pairs, D / 2);
                change(x);
                x.store(rows[row], group, n_pairs, D / 2);
            }
            __syncthreads();
            for (int i = row4; i < n; i += ROWS4) {
                Eight<T> x;
                x.load(&rows[i][piece * 8]);
                enter(x, h0 + i);
            }
            __syncthreads();
        }
    }
    for (int i = first + row4; i < 2 * p.Hkv; i += ROWS4) {
        const bool value = i >= p.Hkv;
        Eight<T> x;
        x.load((value ? v_new : k_new) + (sq * p.Hkv + (value ? i - p.Hkv : i)) * D + piece * 8);
        enter(x, i);
    }
    if (threadIdx.x == 0) count_appended(p, cm, sq, is_sep_new[sq], win_is_sep, sz);
}

// ---- the values of a cache -----------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void expand_fp4_kernel(sepkv_params p, const int32_t *__restrict__ sizes, Fp4Cache cache, T *__restrict__ K,
                                                               T *__restrict__ V) {
    const int which = blockIdx.y & 1;
    const long head = blockIdx.y >> 1;
    const CacheMap cm = cache_map(p, sizes + SEPKV_SIZES_COLS * (head / p.Hkv));
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(which ? cache.Vc : cache.Kc) + head * p.c * (D / 8);
    const Fp4Scales<D> *scales = reinterpret_cast<const Fp4Scales<D> *>(which ? cache.Vs : cache.Ks) + head * p.c;
    T *dst = (which ? V : K) + head * p.c * D;
    constexpr int PIECES = D / 8, ROWS = kThreads / PIECES, N = kExpandRows;
    const int r_in = threadIdx.x / PIECES, piece = threadIdx.x % PIECES, t_end = min((int)(blockIdx.x + 1) * kExpandSlots, p.c);
    for (int t0 = blockIdx.x * kExpandSlots; t0 < t_end; t0 += ROWS * N) {
        uint32_t c[N], s[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int t = t0 + u * ROWS + r_in;
            c[u] = s[u] = 0u;
            if (t < t_end && rank_of_slot(cm, t) >= 0) c[u] = codes[(long)t * PIECES + piece], s[u] = scales[t];
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int t = t0 + u * ROWS + r_in;
            if (t >= t_end) continue;
            Eight<T> x;
            x.from_fp4(c[u], fp4_scale(s[u], piece >> 2));
            x.store(dst + (long)t * D + piece * 8);
        }
    }
}

template <typename F>
void by_type(const sepkv_params &p, F go) {
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (p.dtype == SEPATTN_BF16) p.d == 64 ? go(uint16_t{}, D64{}) : go(uint16_t{}, D128{});
    else p.d == 64 ? go(float{}, D64{}) : go(float{}, D128{});
}

}  // namespace

int launch_fill_fp4(const sepkv_params &p, int L, int nw, const void *K, const void *V, const uint8_t *is_sep, const int32_t *sep_idx, int cap,
                    const int32_t *sep_prefix, const Fp4Cache &cache, uint8_t *win_is_sep, int32_t *sizes, bool zero_rest, hipStream_t st) {
    const dim3 grid((p.c + kFillSlots - 1) / kFillSlots, 2 * p.S * p.Hkv);
    ProfScope prof(SEPATTN_K_CACHE_FILL, st);
    by_type(p, [&](auto T_, auto D_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        auto go = [&](auto ZERO_) {
            hipLaunchKernelGGL((fill_fp4_kernel<T, D, decltype(ZERO_)::value>), grid, dim3(kThreads), 0, st, p, L, nw, cap, static_cast<const T *>(K),
                               static_cast<const T *>(V), is_sep, sep_idx, sep_prefix, cache, win_is_sep, sizes);
        };
        zero_rest ? go(std::true_type{}) : go(std::false_type{});
    });
    return launch_status();
}

int launch_append_fp4(const sepkv_params &p, const TokenTurn *turn, const void *q, const void *k_new, const void *v_new, const uint8_t *is_sep_new,
                      void *q_out, const Fp4Cache &cache, uint8_t *win_is_sep, int32_t *sizes, hipStream_t st) {
    ProfScope prof(SEPATTN_K_CACHE_APPEND, st);
    by_type(p, [&](auto T_, auto D_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        auto go = [&](auto LAYOUT_, auto MODE_) {
            constexpr PairLayout LAYOUT = decltype(LAYOUT_)::value;
            constexpr TokenMode MODE = decltype(MODE_)::value;
            const TokenTurn t = turn ? *turn : TokenTurn{};
            hipLaunchKernelGGL((append_fp4_kernel<T, D, LAYOUT, MODE>), dim3(p.S, MODE == kAsIs ? 1 : 2), dim3(kThreads), 0, st, p, t.rotary_dim / 2, t.eps,
                               t.freqs, t.positions, t.q_weight, t.k_weight, static_cast<const T *>(q), static_cast<const T *>(k_new),
                               static_cast<const T *>(v_new), is_sep_new, static_cast<T *>(q_out), cache, win_is_sep, sizes);
        };
        if (!turn) return go(std::integral_constant<PairLayout, kHalves>{}, std::integral_constant<TokenMode, kAsIs>{});
        auto mode = [&](auto LAYOUT_) {
            turn->norm ? go(LAYOUT_, std::integral_constant<TokenMode, kNormTurn>{}) : go(LAYOUT_, std::integral_constant<TokenMode, kTurn>{});
        };
        const int layout = pair_layout<T>(turn->rotary_dim, turn->interleaved);
        if (layout == kNeighbours) mode(std::integral_constant<PairLayout, kNeighbours>{});
        else if (layout == kHalves) mode(std::integral_constant<PairLayout, kHalves>{});
        else mode(std::integral_constant<PairLayout, kHalvesOdd>{});
    });
    return launch_status();
}

int launch_expand_fp4(const sepkv_params &p, const int32_t *sizes, const Fp4Cache &cache, void *K, void *V, hipStream_t st) {
    const dim3 grid((p.c + kExpandSlots - 1) / kExpandSlots, 2 * p.S * p.Hkv);
    by_type(p, [&](auto T_, auto D_) {
        using T = decltype(T_);
        hipLaunchKernelGGL((expand_fp4_kernel<T, decltype(D_)::value>), grid, dim3(kThreads), 0, st, p, sizes, cache, static_cast<T *>(K),
                           static_cast<T *>(V));
    });
    return launch_status();
}

}  // namespace sepattn
