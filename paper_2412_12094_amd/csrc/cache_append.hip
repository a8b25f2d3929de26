// One new token per sequence enters the four-block KV cache (Sec. 3.3 "Framework").  The first a
// tokens of a sequence fill the Initial Cache; every later token is written behind the newest window
// entry (the window region is a ring: entry u sits at index (head + u) mod its capacity) and joins the
// Local Window Cache, whose oldest entry passes to the Past Window Cache once the Local Window holds
// more than w (the window is ordered oldest first, so that hand-over is a change of the two sizes only).  A sequence whose window region [a+s, c) is full is left untouched: the
// compression step has to run first.
//
// One workgroup per sequence; a thread copies 16-byte pieces of the 2 * Hkv rows.  All threads read
// the sizes, then (after a barrier) thread 0 writes the new ones.
//
// cache_append_rope_kernel: the same for a token whose query and key are turned by its position in the text on the way (rope.hip), in one
// launch: a launch of its own for the turn is what a step of generation would wait for longest.  A second workgroup per sequence
// turns the query, which needs nothing of the cache.  One sequence, 32/8 heads, d = 128, bf16: 3.0 us, 64 sequences 4.1: one chain of
// round trips (sizes, row, store) behind a launch; the bytes would take 0.3.
#include "decode_common.h"
#include "norm.h"

namespace sepattn {

namespace {

constexpr int kAppendThreads = 256;

__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(
    sepkv_params p, int row16, const uint4 *__restrict__ k_new, const uint4 *__restrict__ v_new,
    const uint8_t *__restrict__ is_sep_new, uint4 *__restrict__ Kc, uint4 *__restrict__ Vc,
    uint8_t *__restrict__ win_is_sep, int32_t *__restrict__ sizes) {
    const int sq = blockIdx.x;
    int32_t *sz = sizes + SEPKV_SIZES_COLS * sq;
    const CacheMap cm = cache_map(p, sz);
    const int wcap = cm.wcap;
    const int n_init = cm.n_init;
    const int n_past = cm.n_past, n_loc = cm.n_loc;
    const int u = n_past + n_loc;
    __syncthreads();  // every thread has the old sizes before thread 0 replaces them
    int slot;
    if (n_init < p.a)
        slot = n_init;
    else if (u < wcap)
        slot = p.a + p.s + win_index(cm, u);
    else
        return;  // window region full (uniform over the workgroup)
    for (int item = threadIdx.x; item < 2 * p.Hkv * row16; item += kAppendThreads) {
        const int piece = item % row16, kv = (item / row16) % p.Hkv, which = item / (row16 * p.Hkv);
        const uint4 *src = (which ? v_new : k_new) + ((long)sq * p.Hkv + kv) * row16;
        uint4 *dst = (which ? Vc : Kc) + (((long)sq * p.Hkv + kv) * p.c + slot) * (long)row16;
        dst[piece] = src[piece];
    }
    if (threadIdx.x == 0) {
        if (n_init < p.a) {
            sz[0] = n_init + 1;
        } else {
            win_is_sep[(long)sq * wcap + win_index(cm, u)] = is_sep_new[sq] ? 1 : 0;
            const int over = (n_loc + 1 > p.w) ? 1 : 0;
            sz[2] = n_past + over;
            sz[3] = n_loc + 1 - over;
        }
    }
}

// NORM: the rows of query and key are normed first (norm.h)
template <typename T, int D, PairLayout LAYOUT, bool NORM>
__global__ __launch_bounds__(kAppendThreads) void cache_append_rope_kernel(
    sepkv_params p, int n_pairs, float eps, const double *__restrict__ freqs, const int32_t *__restrict__ positions, NormWeight q_weight,
    NormWeight k_weight, const T *q, const T *__restrict__ k_new, const T *__restrict__ v_new, const uint8_t *__restrict__ is_sep_new, T *q_out, T *__restrict__ Kc,
    T *__restrict__ Vc, uint8_t *__restrict__ win_is_sep, int32_t *__restrict__ sizes) {
    const long sq = blockIdx.x;
    constexpr int E = Angles<T, LAYOUT>::E, GROUPS = D / (2 * E), half = D / 2, rows = kAppendThreads / GROUPS;
    const int group = threadIdx.x % GROUPS, row = threadIdx.x / GROUPS;
    const bool turned = has_turned<LAYOUT, E>(group, n_pairs);
    const int t = turned ? positions[sq] : 0;
    Angles<T, LAYOUT> w;
    Weights<T, LAYOUT> weight;
    auto change = [&](Pairs<T, LAYOUT> &x) {
        if constexpr (NORM) norm_and_turn<T, LAYOUT, D, GROUPS>(x, weight, w, eps, turned, group, n_pairs);
        else if (turned) x.turn(w, group, n_pairs, half);
    };
    if (blockIdx.y == 1) {  // the query
        if constexpr (NORM) weight.load(q_weight, group, n_pairs, half);
        if (turned) w.form(freqs, n_pairs, half, group, t, 1.f);
        for (int h = row; h < p.Hq; h += rows) {
            Pairs<T, LAYOUT> x;
            x.load(q + (sq * p.Hq + h) * D, group, n_pairs, half);
            change(x);
            x.store(q_out + (sq * p.Hq + h) * D, group, n_pairs, half);
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
    if constexpr (NORM) weight.load(k_weight, group, n_pairs, half);
    if (turned) w.form(freqs, n_pairs, half, group, t, 1.f);
    for (int i = row; i < 2 * p.Hkv; i += rows) {
        const bool value = i >= p.Hkv;
        const int h = value ? i - p.Hkv : i;
        Pairs<T, LAYOUT> x;
        x.load((value ? v_new : k_new) + (sq * p.Hkv + h) * D, group, n_pairs, half);
        if (!value) change(x);
        x.store((value ? Vc : Kc) + ((sq * p.Hkv + h) * p.c + slot) * D, group, n_pairs, half);
    }
    if (threadIdx.x == 0) count_appended(p, cm, sq, is_sep_new[sq], win_is_sep, sz);
}

}  // namespace

int launch_cache_append(const sepkv_params &p, const void *k_new, const void *v_new, const uint8_t *is_sep_new,
                        void *Kc, void *Vc, uint8_t *win_is_sep, int32_t *sizes, hipStream_t st) {
    const int elem = (p.dtype == SEPATTN_BF16) ? 2 : 4;
    const int row16 = p.d * elem / 16;
    ProfScope prof(SEPATTN_K_CACHE_APPEND, st);
    hipLaunchKernelGGL(cache_append_kernel, dim3(p.S), dim3(kAppendThreads), 0, st, p, row16,
                       static_cast<const uint4 *>(k_new), static_cast<const uint4 *>(v_new), is_sep_new,
                       static_cast<uint4 *>(Kc), static_cast<uint4 *>(Vc), win_is_sep, sizes);
    return launch_status();
}

int launch_cache_append_rope(const sepkv_params &p, const TokenTurn &turn, const void *q, const void *k_new, const void *v_new,
                             const uint8_t *is_sep_new, void *q_out, void *Kc, void *Vc, uint8_t *win_is_sep, int32_t *sizes, hipStream_t st) {
    ProfScope prof(SEPATTN_K_CACHE_APPEND, st);
    auto go = [&](auto T_, auto D_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        const int layout = pair_layout<T>(turn.rotary_dim, turn.interleaved);
#define APPEND(LAYOUT, NORM)                                                                                                          \
    hipLaunchKernelGGL((cache_append_rope_kernel<T, D, LAYOUT, NORM>), dim3(p.S, 2), dim3(kAppendThreads), 0, st, p, turn.rotary_dim / 2, turn.eps, \
                       turn.freqs, turn.positions, turn.q_weight, turn.k_weight, static_cast<const T *>(q), static_cast<const T *>(k_new),          \
                       static_cast<const T *>(v_new), is_sep_new, static_cast<T *>(q_out), static_cast<T *>(Kc), static_cast<T *>(Vc), win_is_sep, sizes)
        if (turn.norm) {
            if (layout == kNeighbours) APPEND(kNeighbours, true);
            else if (layout == kHalves) APPEND(kHalves, true);
            else APPEND(kHalvesOdd, true);
        } else {
            if (layout == kNeighbours) APPEND(kNeighbours, false);
            else if (layout == kHalves) APPEND(kHalves, false);
            else APPEND(kHalvesOdd, false);
        }
#undef APPEND
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (p.dtype == SEPATTN_BF16) p.d == 64 ? go(uint16_t{}, D64{}) : go(uint16_t{}, D128{});
    else p.d == 64 ? go(float{}, D64{}) : go(float{}, D128{});
    return launch_status();
}

}  // namespace sepattn
