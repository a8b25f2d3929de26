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
#include "rotary.h"

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

// the new sizes and the window's flag
__device__ inline void count_appended(const sepkv_params &p, const CacheMap &cm, long sq, bool is_sep, uint8_t *__restrict__ win_is_sep,
                                      int32_t *__restrict__ sz) {
    if (cm.n_init < p.a) {
        sz[0] = cm.n_init + 1;
    } else {
        win_is_sep[sq * cm.wcap + win_index(cm, cm.n_past + cm.n_loc)] = is_sep ? 1 : 0;
        const int over = (cm.n_loc + 1 > p.w) ? 1 : 0;
        sz[2] = cm.n_past + over;
        sz[3] = cm.n_loc + 1 - over;
    }
}

template <typename T, PairLayout LAYOUT>
__global__ __launch_bounds__(kAppendThreads) void cache_append_rope_kernel(
    sepkv_params p, int n_pairs, int log_groups, const double *__restrict__ freqs, const int32_t *__restrict__ positions, const T *q,
    const T *__restrict__ k_new, const T *__restrict__ v_new, const uint8_t *__restrict__ is_sep_new, T *q_out, T *__restrict__ Kc,
    T *__restrict__ Vc, uint8_t *__restrict__ win_is_sep, int32_t *__restrict__ sizes) {
    const long sq = blockIdx.x;
    const int group = threadIdx.x & ((1 << log_groups) - 1), row = threadIdx.x >> log_groups, rows = kAppendThreads >> log_groups;
    constexpr int E = Angles<T, LAYOUT>::E;
    const int half = p.d / 2;
    const bool turned = has_turned<LAYOUT, E>(group, n_pairs);
    const int t = positions[sq];
    Angles<T, LAYOUT> w;
    if (blockIdx.y == 1) {  // the query
        if (turned) w.form(freqs, n_pairs, half, group, t, 1.f);
        for (int h = row; h < p.Hq; h += rows) {
            Pairs<T, LAYOUT> x;
            x.load(q + (sq * p.Hq + h) * p.d, group, n_pairs, half);
            if (turned) x.turn(w, group, n_pairs, half);
            x.store(q_out + (sq * p.Hq + h) * p.d, group, n_pairs, half);
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
    if (turned) w.form(freqs, n_pairs, half, group, t, 1.f);
    for (int i = row; i < 2 * p.Hkv; i += rows) {
        const bool value = i >= p.Hkv;
        const int h = value ? i - p.Hkv : i;
        Pairs<T, LAYOUT> x;
        x.load((value ? v_new : k_new) + (sq * p.Hkv + h) * p.d, group, n_pairs, half);
        if (turned && !value) x.turn(w, group, n_pairs, half);
        x.store((value ? Vc : Kc) + ((sq * p.Hkv + h) * p.c + slot) * p.d, group, n_pairs, half);
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

int launch_cache_append_rope(const sepkv_params &p, int rotary_dim, int interleaved, const double *freqs, const int32_t *positions,
                             const void *q, const void *k_new, const void *v_new, const uint8_t *is_sep_new, void *q_out, void *Kc,
                             void *Vc, uint8_t *win_is_sep, int32_t *sizes, hipStream_t st) {
    const int groups = p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4) / 32;
    int log_groups = 0;
    while ((1 << log_groups) < groups) ++log_groups;
    ProfScope prof(SEPATTN_K_CACHE_APPEND, st);
    auto go = [&](auto T_) {
        using T = decltype(T_);
        const int layout = pair_layout<T>(rotary_dim, interleaved);
#define APPEND(LAYOUT)                                                                                                               \
    hipLaunchKernelGGL((cache_append_rope_kernel<T, LAYOUT>), dim3(p.S, 2), dim3(kAppendThreads), 0, st, p, rotary_dim / 2, log_groups, \
                       freqs, positions, static_cast<const T *>(q), static_cast<const T *>(k_new), static_cast<const T *>(v_new),    \
                       is_sep_new, static_cast<T *>(q_out), static_cast<T *>(Kc), static_cast<T *>(Vc), win_is_sep, sizes)
        if (layout == kNeighbours) APPEND(kNeighbours);
        else if (layout == kHalves) APPEND(kHalves);
        else APPEND(kHalvesOdd);
#undef APPEND
    };
    if (p.dtype == SEPATTN_BF16) go(uint16_t{});
    else go(float{});
    return launch_status();
}

}  // namespace sepattn
