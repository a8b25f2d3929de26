// Norms of queries and keys with their rotary positions, forward and backward.
//
//   z = R(theta) (w x r),  r = (mean of x^2 + eps)^(-1/2) over the d values of a row;
// with g = R(-theta) dz and u = w g:   dx = r (u - x r^2 mean(u x)),   dw = sum over all rows of g x r.
//
// Forward: one read and one write of q, k, v, as in rope.hip: the norm adds a sum over the 4 to 16 lanes that hold a row.  Backward: x and dz are
// read and dx is written; r is formed again from x, which is cheaper than a read of it.  dw is a sum over all tokens and heads: a
// workgroup walks through several tiles of tokens, keeps the sums of its dimensions in registers, adds them up in LDS and leaves one row
// of partial sums, which a second kernel adds in fp64, in a fixed order, so that two runs give the same bits.
#include "norm.h"

#include <type_traits>

namespace sepattn {

namespace {

constexpr int kNormThreads = 256;

template <typename T, int D, PairLayout LAYOUT, bool STREAM>
__global__ __launch_bounds__(kNormThreads) void norm_rope_kernel(NormRopeTensors x, int L, int n_pairs, int log_tokens, int chunk, float eps,
                                                                  const double *__restrict__ freqs, const int32_t *__restrict__ positions,
                                                                  const int32_t *__restrict__ doc_start) {
    constexpr int E = 16 / (int)sizeof(T), GROUPS = D / (2 * E), half = D / 2;
    const int group = threadIdx.x % GROUPS, row_slot = threadIdx.x / GROUPS;
    const int l = ((int)blockIdx.x << log_tokens) + (row_slot & ((1 << log_tokens) - 1));
    const int slot = row_slot >> log_tokens, slots = (kNormThreads / GROUPS) >> log_tokens;
    const int b = blockIdx.z;
    if (l >= L) return;
    const long at = (long)b * L + l;
    const int t = positions ? positions[at] : l - (doc_start ? doc_start[at] : 0);
    const int h0 = blockIdx.y * chunk, all = x.heads[0] + x.heads[1] + x.heads[2], h1 = min(h0 + chunk, all);
    const bool turned = has_turned<LAYOUT, E>(group, n_pairs);
    Angles<T, LAYOUT> w;
    if (turned && h0 < x.heads[0] + x.heads[1]) w.form(freqs, n_pairs, half, group, t, 1.f);
    int before = 0;
#pragma unroll
    for (int which = 0; which < 3; ++which) {  // q, k, v
        const int lo = max(h0 - before, 0), hi = min(h1 - before, x.heads[which]);
        before += x.heads[which];
        if (lo >= hi) continue;
        const sepattn_strides from = x.from[which], to = x.to[which];
        const T *src = static_cast<const T *>(x.src[which]) + b * from.b + l * from.l;
        T *dst = static_cast<T *>(x.dst[which]) + b * to.b + l * to.l;
        Weights<T, LAYOUT> weight;
        if (which < 2) weight.load(x.weight[which], group, n_pairs, half);
        constexpr int N = 4;
        for (int h = lo + slot; h < hi; h += N * slots) {
            Pairs<T, LAYOUT> row[N];
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (h + n * slots < hi) row[n].template load<STREAM>(src + (h + n * slots) * from.h, group, n_pairs, half);
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (h + n * slots < hi) {
                    if (which < 2) norm_and_turn<T, LAYOUT, D, GROUPS>(row[n], weight, w, eps, turned, group, n_pairs);
                    row[n].store(dst + (h + n * slots) * to.h, group, n_pairs, half);
                }
        }
    }
}

// Grid (walkers over the tiles of tokens, chunks of heads).  A chunk is of q, of k or of v.  Row blockIdx.x of the partial sums of chunk y.
template <typename T, int D, PairLayout LAYOUT, bool STREAM>
__global__ __launch_bounds__(kNormThreads) void norm_rope_backward_kernel(NormRopeTensors x, NormRopeGrid grid, int L, int n_pairs, float eps,
                                                                           const double *__restrict__ freqs,
                                                                           const int32_t *__restrict__ positions,
                                                                           const int32_t *__restrict__ doc_start, float *__restrict__ part) {
    constexpr int E = 16 / (int)sizeof(T), GROUPS = D / (2 * E), half = D / 2, ROWS = kNormThreads / GROUPS;
    const int group = threadIdx.x % GROUPS, row_slot = threadIdx.x / GROUPS;
    const int token = row_slot & ((1 << grid.log_tokens) - 1), slot = row_slot >> grid.log_tokens, slots = ROWS >> grid.log_tokens;
    const int y = blockIdx.y, which = y < grid.chunks[0] ? 0 : y < grid.chunks[0] + grid.chunks[1] ? 1 : 2;
    const int c = y - (which > 0 ? grid.chunks[0] : 0) - (which > 1 ? grid.chunks[1] : 0);
    const int h0 = c * grid.chunk, h1 = min(h0 + grid.chunk, x.heads[which]);
    const sepattn_strides from = x.from[which], to = x.to[which], gs = x.grad_strides[which];
    const bool turned = has_turned<LAYOUT, E>(group, n_pairs);
    Weights<T, LAYOUT> weight;
    float su[E], sv[E];
    if (which < 2) {
        weight.load(x.weight[which], group, n_pairs, half);
#pragma unroll
        for (int e = 0; e < E; ++e) su[e] = sv[e] = 0.f;
    }
    for (int tile = blockIdx.x; tile < grid.tiles_per_row * grid.B; tile += gridDim.x) {
        const int b = tile / grid.tiles_per_row, l = ((tile - b * grid.tiles_per_row) << grid.log_tokens) + token;
        if (l >= L) continue;
        const T *g = static_cast<const T *>(x.grad[which]) + b * gs.b + l * gs.l;
        T *dst = static_cast<T *>(x.dst[which]) + b * to.b + l * to.l;
        if (which == 2) {  // values: moved only
            constexpr int N = 4;
            for (int h = h0 + slot; h < h1; h += N * slots) {
                Pairs<T, LAYOUT> row[N];
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (h + n * slots < h1) row[n].template load<STREAM>(g + (h + n * slots) * gs.h, group, n_pairs, half);
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (h + n * slots < h1) row[n].store(dst + (h + n * slots) * to.h, group, n_pairs, half);
            }
            continue;
        }
        const T *src = static_cast<const T *>(x.src[which]) + b * from.b + l * from.l;
        const long at = (long)b * L + l;
        Angles<T, LAYOUT> w;
        if (turned) w.form(freqs, n_pairs, half, group, positions ? positions[at] : l - (doc_start ? doc_start[at] : 0), -1.f);
        constexpr int N = 2;
        for (int h = h0 + slot; h < h1; h += N * slots) {
            Pairs<T, LAYOUT> rx[N], rg[N];
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (h + n * slots < h1) {
                    rx[n].template load<STREAM>(src + (h + n * slots) * from.h, group, n_pairs, half);
                    rg[n].template load<STREAM>(g + (h + n * slots) * gs.h, group, n_pairs, half);
                }
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (h + n * slots < h1) {
                    float xu[E], xv[E], gu[E], gv[E];
                    rx[n].widen(xu, xv);
                    rg[n].widen(gu, gv);
                    if (turned) turn_pairs(gu, gv, w, group, n_pairs, half);
                    const float r = row_rms<D, GROUPS>(xu, xv, eps);
                    float dot = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        su[e] = fmaf(gu[e], xu[e] * r, su[e]);
                        sv[e] = fmaf(gv[e], xv[e] * r, sv[e]);
                        gu[e] *= weight.u[e], gv[e] *= weight.v[e];
                        dot = fmaf(gu[e], xu[e], fmaf(gv[e], xv[e], dot));
                    }
                    const float back = row_sum<GROUPS>(dot) * (r * r) * (1.f / D);
#pragma unroll
                    for (int e = 0; e < E; ++e) gu[e] = r * fmaf(-back, xu[e], gu[e]), gv[e] = r * fmaf(-back, xv[e], gv[e]);
                    rg[n].narrow(gu, gv);
                    rg[n].store(dst + (h + n * slots) * to.h, group, n_pairs, half);
                }
        }
    }
    if (which == 2 || !part) return;
    __shared__ float sums[ROWS][D];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        int i, j;
        members_of<LAYOUT, E>(group, e, n_pairs, half, i, j);
        sums[row_slot][i] = su[e], sums[row_slot][j] = sv[e];
    }
    __syncthreads();
    for (int rows = ROWS / 2; rows >= 1; rows /= 2) {
        for (int i = threadIdx.x; i < rows * D; i += kNormThreads) sums[i / D][i % D] += sums[i / D + rows][i % D];
        __syncthreads();
    }
    if (threadIdx.x < D) part[((long)y * gridDim.x + blockIdx.x) * D + threadIdx.x] = sums[0][threadIdx.x];
}

// dw of q (blockIdx.y 0) and of k (1): rows of partial sums, eight columns per workgroup
__global__ __launch_bounds__(kNormThreads) void norm_weights_kernel(int D, int rows_q, int rows_k, const float *__restrict__ part,
                                                                     float *__restrict__ dq_weight, float *__restrict__ dk_weight) {
    float *out = blockIdx.y ? dk_weight : dq_weight;
    if (!out) return;
    const int col = blockIdx.x * 8 + threadIdx.x % 8, first = threadIdx.x / 8, rows = blockIdx.y ? rows_k : rows_q;
    const float *p = part + (blockIdx.y ? (long)rows_q * D : 0) + col;
    constexpr int STEP = kNormThreads / 8, N = 8;
    double sum = 0.0;
    for (int r = first; r < rows; r += N * STEP) {
        float v[N];
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = r + n * STEP < rows ? p[(long)(r + n * STEP) * D] : 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) sum += v[n];
    }
    __shared__ double sums[kNormThreads];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int n = kNormThreads / 2; n >= 8; n /= 2) {
        if (threadIdx.x < n) sums[threadIdx.x] += sums[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x < 8) out[col] = (float)sums[threadIdx.x];
}

int log_tokens_of(int L, int rows) {
    int n = 0;
    while ((1 << n) < L && (2 << n) <= rows) ++n;
    return n;
}
int groups_of(const sepattn_norm_rope_params &p) { return p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4) / 32; }
bool streams(const sepattn_norm_rope_params &p, long rows) {  // as in launch_rope
    const long row_bytes = p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4);
    return row_bytes * rows > 128L << 20 && row_bytes >= 256;
}

template <typename F>
void by_layout(const sepattn_norm_rope_params &p, F go) {
    auto with = [&](auto T_, auto D_) {
        using T = decltype(T_);
        const int layout = pair_layout<T>(p.rotary_dim, p.interleaved);
        if (layout == kNeighbours) go(T_, D_, std::integral_constant<PairLayout, kNeighbours>{});
        else if (layout == kHalves) go(T_, D_, std::integral_constant<PairLayout, kHalves>{});
        else go(T_, D_, std::integral_constant<PairLayout, kHalvesOdd>{});
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (p.dtype == SEPATTN_BF16) p.d == 64 ? with(uint16_t{}, D64{}) : with(uint16_t{}, D128{});
    else p.d == 64 ? with(float{}, D64{}) : with(float{}, D128{});
}

}  // namespace

NormRopeGrid norm_rope_grid(const sepattn_norm_rope_params &p, bool values, int units) {
    NormRopeGrid g;
    const int rows = kNormThreads / groups_of(p);
    g.B = p.B;
    g.log_tokens = log_tokens_of(p.L, rows);
    g.tiles_per_row = (int)(((long)p.L + (1 << g.log_tokens) - 1) >> g.log_tokens);
    const int heads[3] = {p.Hq, p.Hkv, values ? p.Hkv : 0}, slots = rows >> g.log_tokens;
    const long tiles = (long)g.tiles_per_row * p.B, want = 6L * units;
    // a chunk of heads such that there are `want` workgroups, if there is work for them; then walkers for as many
    const long all = heads[0] + heads[1] + heads[2], per = (all * tiles + want - 1) / want;
    g.chunk = (int)(per < 8 ? per : 8);
    g.chunk = (g.chunk + slots - 1) / slots * slots;
    int chunks = 0;
    for (int i = 0; i < 3; ++i) chunks += g.chunks[i] = (heads[i] + g.chunk - 1) / g.chunk;
    const long walkers = (want + chunks - 1) / chunks;
    g.walkers = (int)(walkers < tiles ? walkers : tiles);
    return g;
}

size_t norm_rope_backward_workspace(const sepattn_norm_rope_params &p) {
    // with and without values a call is cut differently
    const NormRopeGrid a = norm_rope_grid(p, true, compute_units()), b = norm_rope_grid(p, false, compute_units());
    auto rows = [](const NormRopeGrid &g) { return (size_t)(g.chunks[0] + g.chunks[1]) * g.walkers; };
    return align_up((rows(a) > rows(b) ? rows(a) : rows(b)) * p.d * sizeof(float), 256);
}

int launch_norm_rope(const sepattn_norm_rope_params &p, const double *freqs, const int32_t *positions, const int32_t *doc_start,
                     const NormRopeTensors &x, hipStream_t st) {
    const int rows = kNormThreads / groups_of(p), log_tokens = log_tokens_of(p.L, rows), slots = rows >> log_tokens;
    const int heads = x.heads[0] + x.heads[1] + x.heads[2], tiles = (int)(((long)p.L + (1 << log_tokens) - 1) >> log_tokens);
    const bool stream = streams(p, 2L * p.B * p.L * heads);
    const long row_bytes = p.d * (p.dtype == SEPATTN_BF16 ? 2 : 4), per_unit = stream ? 4 : 2 * row_bytes * p.B * p.L * heads > 128L << 20 ? 32 : 8;
    const long want = (per_unit * compute_units() + (long)tiles * p.B - 1) / ((long)tiles * p.B);
    int chunk = (int)((heads + want - 1) / want);
    chunk = (chunk + slots - 1) / slots * slots;
    const dim3 grid(tiles, (heads + chunk - 1) / chunk, p.B);
    by_layout(p, [&](auto T_, auto D_, auto LAYOUT_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        constexpr PairLayout LAYOUT = decltype(LAYOUT_)::value;
        auto go = [&](auto STREAM_) {
            hipLaunchKernelGGL((norm_rope_kernel<T, D, LAYOUT, decltype(STREAM_)::value>), grid, dim3(kNormThreads), 0, st, x, p.L, p.rotary_dim / 2,
                               log_tokens, chunk, p.eps, freqs, positions, doc_start);
        };
        if (LAYOUT != kHalvesOdd && stream) go(std::bool_constant<LAYOUT != kHalvesOdd>{});
        else go(std::false_type{});
    });
    return launch_status();
}

int launch_norm_rope_backward(const sepattn_norm_rope_params &p, const double *freqs, const int32_t *positions, const int32_t *doc_start,
                              const NormRopeTensors &x, float *dq_weight, float *dk_weight, float *part, hipStream_t st) {
    const NormRopeGrid g = norm_rope_grid(p, x.heads[2] > 0, compute_units());
    const int chunks = g.chunks[0] + g.chunks[1] + g.chunks[2];
    if (chunks > 65535) return SEPATTN_ERR_SHAPE;
    const bool sums = dq_weight || dk_weight;
    by_layout(p, [&](auto T_, auto D_, auto LAYOUT_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        constexpr PairLayout LAYOUT = decltype(LAYOUT_)::value;
        auto go = [&](auto STREAM_) {
            hipLaunchKernelGGL((norm_rope_backward_kernel<T, D, LAYOUT, decltype(STREAM_)::value>), dim3(g.walkers, chunks), dim3(kNormThreads), 0, st, x,
                               g, p.L, p.rotary_dim / 2, p.eps, freqs, positions, doc_start, sums ? part : nullptr);
        };
        if (LAYOUT != kHalvesOdd && streams(p, (long)p.B * p.L * (3L * (x.heads[0] + x.heads[1]) + 2L * x.heads[2]))) go(std::bool_constant<LAYOUT != kHalvesOdd>{});
        else go(std::false_type{});
    });
    if (!sums) return launch_status();
    if (hipGetLastError() != hipSuccess) return SEPATTN_ERR_HIP;
    hipLaunchKernelGGL(norm_weights_kernel, dim3(p.d / 8, 2), dim3(kNormThreads), 0, st, p.d, g.chunks[0] * g.walkers, g.chunks[1] * g.walkers, part,
                       dq_weight, dk_weight);
    return launch_status();
}

}  // namespace sepattn
