// Rotary positions in front of the attention, forward and backward, and the keys of a cache turned by their positions within it.
//
//   (x, y) -> (x cos - y sin, y cos + x sin)   for every pair of dimensions, the angle = position * the pair's frequency;
// the gradient is the same with the opposite angles (the turn is orthogonal).  Nothing is summed: the work is one read and one
// write of q, k, v, and the change of layout between token by token (the projections) and head by head (the attention) costs
// nothing on the way.  What has to be formed per (token, pair) and not per (token, pair, head) is the angle, some sixty
// instructions: a lane owns one token and one group of pairs (rotary.h), forms its angles once, in fp64 up to the fraction
// of a turn, and walks through heads, four rows' loads in flight.  What bounds it is the memory: 8192 tokens of 32/8 heads, d = 128, bf16, take
// 36.2 us forward and 34.8 backward (201 MB read and written: 5.6 and 5.8 TB/s, a large copy on the same card 5.0), 8 x 2048 tokens of
// 12/12 heads, d = 64, 28.3 us (151 MB, 5.3 TB/s), 3 x 1531 of 28/4 heads in fp32 31.0 (169 MB, 5.5 TB/s).  With a thread per (row, group), which
// forms the angles for every head, the first took 46.9.
#include "decode_common.h"
#include "rotary.h"

#include <cmath>
#include <type_traits>

namespace sepattn {

namespace {

constexpr int kRopeThreads = 256;

// q, k, v -> Q, K, V: element strides of (batch, head, token)
struct RopeTensors {
    const void *src[3];
    void *dst[3];
    sepattn_strides from[3], to[3];
    int heads[3];
};

// Threads of a workgroup: group of pairs (fastest), `tokens` tokens, head slots; grid (token tiles, head chunks, B).  A thread walks through the
// heads  slot, slot + slots, ...  of its chunk.
template <typename T, PairLayout LAYOUT, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeTensors x, int L, int n_pairs, int log_groups, int log_tokens, int chunk,
                                                             float sign, const double *__restrict__ freqs,
                                                             const int32_t *__restrict__ positions, const int32_t *__restrict__ doc_start) {
    const int group = threadIdx.x & ((1 << log_groups) - 1);
    const int l = ((int)blockIdx.x << log_tokens) + ((threadIdx.x >> log_groups) & ((1 << log_tokens) - 1));
    const int slot = threadIdx.x >> (log_groups + log_tokens), slots = kRopeThreads >> (log_groups + log_tokens);
    const int b = blockIdx.z;
    if (l >= L) return;
    const long at = (long)b * L + l;
    const int t = positions ? positions[at] : l - (doc_start ? doc_start[at] : 0);
    const int h0 = blockIdx.y * chunk, all = x.heads[0] + x.heads[1] + x.heads[2], h1 = min(h0 + chunk, all);
    constexpr int E = Angles<T, LAYOUT>::E;
    const int half = E << log_groups;
    const bool turned = has_turned<LAYOUT, E>(group, n_pairs);
    Angles<T, LAYOUT> w;
    if (turned && h0 < x.heads[0] + x.heads[1]) w.form(freqs, n_pairs, half, group, t, sign);
    int before = 0;
#pragma unroll
    for (int which = 0; which < 3; ++which) {  // q, k, v
        const sepattn_strides from = x.from[which], to = x.to[which];
        const T *src = static_cast<const T *>(x.src[which]) + b * from.b + l * from.l;
        T *dst = static_cast<T *>(x.dst[which]) + b * to.b + l * to.l;
        const int lo = max(h0 - before, 0), hi = min(h1 - before, x.heads[which]);
        constexpr int N = 4;
        for (int h = lo + slot; h < hi; h += N * slots) {
            Pairs<T, LAYOUT> row[N];
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (h + n * slots < hi) row[n].template load<STREAM>(src + (h + n * slots) * from.h, group, n_pairs, half);
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (h + n * slots < hi) {
                    if (which < 2 && turned) row[n].turn(w, group, n_pairs, half);
                    row[n].store(dst + (h + n * slots) * to.h, group, n_pairs, half);
                }
        }
        before += x.heads[which];
    }
}

// Keys of a four-block cache turned by their rank among the valid entries (oldest first), dimension i with i + D/2, angles from the
// table: the prefix caches of the shared decode, whose entries never move.  Threads: group of pairs (fastest), slots of the cache;
// grid (slot tiles, chunks of KV heads, caches).  A thread reads its slot's table row once and walks through the heads of its chunk.
// 8192 entries of 8 heads, d = 128, bf16, in place: 8.2 us (37.7 MB with the table: 4.6 TB/s).
template <typename T, int D>
__global__ __launch_bounds__(kRopeThreads) void rope_cache_kernel(sepkv_params p, int chunk, const int32_t *__restrict__ sizes,
                                                                   const float *__restrict__ rope, int n_pos, const T *Kc, T *K_out) {
    constexpr int GROUPS = D / (2 * Angles<T, kHalves>::E), SLOTS = kRopeThreads / GROUPS, E = Angles<T, kHalves>::E;
    const int group = threadIdx.x % GROUPS, slot = blockIdx.x * SLOTS + threadIdx.x / GROUPS;
    const long cache = blockIdx.z;
    if (slot >= p.c) return;
    const int e = rank_of_slot(cache_map(p, sizes + SEPKV_SIZES_COLS * cache), slot);
    if (e < 0) return;
    Angles<T, kHalves> w;
    const float *row = rope + (long)min(e, n_pos - 1) * D + group * E;
#pragma unroll
    for (int i = 0; i < E; ++i) w.cs[i] = row[i], w.sn[i] = row[D / 2 + i];
    const int h0 = blockIdx.y * chunk, h1 = min(h0 + chunk, p.Hkv);
    constexpr int N = 4;
    for (int h = h0; h < h1; h += N) {
        Pairs<T, kHalves> x[N];
        const long at = ((cache * p.Hkv + h) * p.c + slot) * D, pitch = (long)p.c * D;
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (h + n < h1) x[n].load(Kc + at + n * pitch, group, D / 2, D / 2);
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (h + n < h1) {
                x[n].turn(w, group, D / 2, D / 2);
                x[n].store(K_out + at + n * pitch, group, D / 2, D / 2);
            }
    }
}

}  // namespace

int launch_rope_cache(const sepkv_params &p, const int32_t *sizes, const float *rope, int n_pos, const void *Kc, void *K_out, hipStream_t st) {
    const int slots = kRopeThreads / (p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4) / 32), tiles = (p.c + slots - 1) / slots;
    // chunks of heads: eight workgroups per compute unit, as in launch_rope
    const long want = (8L * compute_units() + (long)tiles * p.S - 1) / ((long)tiles * p.S);
    const int chunk = (int)((p.Hkv + want - 1) / want);
    const dim3 grid(tiles, (p.Hkv + chunk - 1) / chunk, p.S);
    auto go = [&](auto T_, auto D_) {
        using T = decltype(T_);
        hipLaunchKernelGGL((rope_cache_kernel<T, decltype(D_)::value>), grid, dim3(kRopeThreads), 0, st, p, chunk, sizes, rope, n_pos,
                           static_cast<const T *>(Kc), static_cast<T *>(K_out));
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (p.dtype == SEPATTN_BF16) p.d == 64 ? go(uint16_t{}, D64{}) : go(uint16_t{}, D128{});
    else p.d == 64 ? go(float{}, D64{}) : go(float{}, D128{});
    return launch_status();
}

int rope_frequencies(int rotary_dim, double base, double factor, double low, double high, int original_length, double *freqs) {
    for (int p = 0; p < rotary_dim / 2; ++p) {
        const double f = std::pow(base, -2.0 * p / rotary_dim);
        double keep = 0.0;  // share of the frequency that is not interpolated
        if (original_length > 0) {
            const double turns = original_length * f * 0.15915494309189533577;
            keep = turns <= low ? 0.0 : turns >= high ? 1.0 : (turns - low) / (high - low);
        }
        freqs[p] = f * ((1.0 - keep) / factor + keep);
    }
    return SEPATTN_OK;
}

int launch_rope(const sepattn_rope_params &p, const double *freqs, const int32_t *positions, const int32_t *doc_start,
                const void *const (&src)[3], const sepattn_strides (&from)[3], void *const (&dst)[3], const sepattn_strides (&to)[3],
                bool backward, hipStream_t st) {
    RopeTensors x;
    for (int i = 0; i < 3; ++i) {
        x.src[i] = src[i], x.dst[i] = dst[i], x.from[i] = from[i], x.to[i] = to[i];
        x.heads[i] = i == 0 ? p.Hq : (src[i] ? p.Hkv : 0);
    }
    const int heads = x.heads[0] + x.heads[1] + x.heads[2];
    const int groups = p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4) / 32;  // 4, 8 or 16
    int log_groups = 0, log_tokens = 0;
    while ((1 << log_groups) < groups) ++log_groups;
    while ((1 << log_tokens) < p.L && (1 << (log_groups + log_tokens)) < kRopeThreads) ++log_tokens;
    const int tiles = (p.L + (1 << log_tokens) - 1) >> log_tokens, slots = kRopeThreads >> (log_groups + log_tokens);
    // More than half of the last cache level (256 MB) passes through: the rows are read with the non-temporal hint, if an instruction covers whole
    // cache lines of them (rows of 256 bytes and more; rows of 128 lose 2 us of 31), so that the results find room there (microseconds without
    // / with it, 32/8 heads, d = 128: 8192 tokens 45 / 36, backward 43 / 35, fp32 42 / 34; 3 x 700 tokens 10.4 / 12.0).  Chunks of heads: as many as make
    // this many workgroups per compute unit (4 / 8 / 32: with the hint 36.2 / 37.0 / 39.2; 3 x 700 tokens 10.4 / 10.7 / 12.3; 8 x 12/12 heads, d = 64,
    // 2048 tokens 31.1 / 31.6 / 28.3).
    const long row_bytes = p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4);
    const bool large = 2 * row_bytes * p.B * p.L * heads > 128L << 20, stream = large && row_bytes >= 256;
    const long per_unit = stream ? 4 : large ? 32 : 8;
    const long want = (per_unit * compute_units() + (long)tiles * p.B - 1) / ((long)tiles * p.B);
    int chunk = (int)((heads + want - 1) / want);
    chunk = (chunk + slots - 1) / slots * slots;
    const dim3 grid(tiles, (heads + chunk - 1) / chunk, p.B);
    const float sign = backward ? -1.f : 1.f;
    auto go = [&](auto T_) {
        using T = decltype(T_);
        const int layout = pair_layout<T>(p.rotary_dim, p.interleaved);
#define ROPE(LAYOUT, STREAM)                                                                                                 \
    hipLaunchKernelGGL((rope_kernel<T, LAYOUT, STREAM>), grid, dim3(kRopeThreads), 0, st, x, p.L, p.rotary_dim / 2, log_groups, log_tokens, \
                       chunk, sign, freqs, positions, doc_start)
        if (layout == kNeighbours) { if (stream) ROPE(kNeighbours, true); else ROPE(kNeighbours, false); }
        else if (layout == kHalves) { if (stream) ROPE(kHalves, true); else ROPE(kHalves, false); }
        else ROPE(kHalvesOdd, false);
#undef ROPE
    };
    if (p.dtype == SEPATTN_BF16) go(uint16_t{});
    else go(float{});
    return launch_status();
}

}  // namespace sepattn
