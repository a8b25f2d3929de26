// Norms of queries and keys with their rotary positions, forward and backward.
//
//   z = R(theta) (w x r),  r = (mean of x^2 + eps)^(-1/2) over the d values of a row;
// with g = R(-theta) dz and u = w g:   dx = r (u - x r^2 mean(u x)),   dw = sum over all rows of g x r.
//
// Forward: one read and one write of q, k, v, as in rope.hip: the norm adds a sum over the 4 to 16 lanes that hold a row.  Backward: x and dz are
// read and dx is written; r is formed again from x, which is cheaper than a read of it.  dw is a sum over all tokens and heads: a
// workgroup walks through several tiles of tokens, keeps the sums of its dimensions in registers, adds them up in LDS and leaves one row
// of partial sums, which a second kernel adds in fp64, in a fixed order, so that two runs give the same bits.
//
// Memory bounds both.  8192 tokens, 32 + 8 heads of 128, bf16: forward 201 MB in 37 us, 5.4 TB/s (rope.hip without the norm: 36); backward 285 MB in
// 58 us, 4.9 TB/s, and 4.9 for the second kernel.  8 x 2048 tokens, 12 + 12 heads of 64: backward 201 MB in 43 us.  fp32, 4096 tokens, 32 + 8 heads of 128:
// forward 35 us, backward 52, and 4.7.
// The forward's registers decide: with the weights behind a branch per dimension it took 140 of them and 41 us, with one branch 96 and 37.
#include "norm.h"

#include <type_traits>

namespace sepattn {

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormRows = 2;   // rows of q or k that a lane of the backward has in flight
constexpr int kMovedRows = 4;  // ... of v

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

// sum over the lanes of a wave that hold the same group of pairs: lanes l, l + GROUPS, l + 2 GROUPS, ...
template <int GROUPS>
__device__ inline float rows_sum(float x) {
    auto turned_by = [](float y, auto CTRL) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), decltype(CTRL)::value, 0xF, 0xF, true)); };
    if constexpr (GROUPS <= 8) x += turned_by(x, std::integral_constant<int, 0x128>{});  // row_ror 8
    if constexpr (GROUPS <= 4) x += turned_by(x, std::integral_constant<int, 0x124>{});  // row_ror 4
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A workgroup has q, k or v (grid.first) and a run of that tensor's items, which are (tile of tokens, group of heads), the groups fastest, so that angles
// serve all heads of a tile.  At 8192 tokens, 32 + 8 heads of 128: q, k and v in one workgroup in turn and no request ahead 70 us, so 58; one row in
// flight instead of two, four instead of three workgroups per compute unit, and stores with the non-temporal hint were slower each.
template <typename T, int D, PairLayout LAYOUT, bool STREAM>
__global__ __launch_bounds__(kNormThreads, LAYOUT == kHalvesOdd ? 2 : 3) void norm_rope_backward_kernel(
    NormRopeTensors x, NormRopeGrid grid, int L, int n_pairs, float eps, const double *__restrict__ freqs, const int32_t *__restrict__ positions,
    const int32_t *__restrict__ doc_start, float *__restrict__ part) {
    constexpr int E = 16 / (int)sizeof(T), GROUPS = D / (2 * E), half = D / 2, ROWS = kNormThreads / GROUPS;
    const int group = threadIdx.x % GROUPS, row_slot = threadIdx.x / GROUPS;
    const int token = row_slot & ((1 << grid.log_tokens) - 1), slot = row_slot >> grid.log_tokens, slots = ROWS >> grid.log_tokens;
    const int which = (int)blockIdx.x < grid.first[1] ? 0 : (int)blockIdx.x < grid.first[2] ? 1 : 2;
    const int mine = blockIdx.x - grid.first[which], sharers = grid.first[which + 1] - grid.first[which];
    const int heads = x.heads[which], step = (which < 2 ? kNormRows : kMovedRows) * slots, groups = (heads + step - 1) / step;
    const long items = (long)grid.tiles_per_row * grid.B * groups, last = items * (mine + 1) / sharers;
    long item = items * mine / sharers;
    int tile = (int)(item / groups), h0 = (int)(item - (long)tile * groups) * step;
    const sepattn_strides from = x.from[which], to = x.to[which], gs = x.grad_strides[which];
    // the token of a tile: row of the batch, index in it
    auto place = [&](int &b, int &l) {
        b = tile / grid.tiles_per_row;
        l = ((tile - b * grid.tiles_per_row) << grid.log_tokens) + token;
    };
    int b, l;
    if (which == 2) {  // values: moved only
        for (place(b, l); item < last; ++item, h0 += step) {
            if (h0 >= heads) h0 = 0, ++tile, place(b, l);
            const T *g = static_cast<const T *>(x.grad[which]) + b * gs.b + l * gs.l;
            T *dst = static_cast<T *>(x.dst[which]) + b * to.b + l * to.l;
            Pairs<T, LAYOUT> row[kMovedRows];
#pragma unroll
            for (int n = 0; n < kMovedRows; ++n)
                if (l < L && h0 + slot + n * slots < heads) row[n].template load<STREAM>(g + (h0 + slot + n * slots) * gs.h, group, n_pairs, half);
#pragma unroll
            for (int n = 0; n < kMovedRows; ++n)
                if (l < L && h0 + slot + n * slots < heads) row[n].store(dst + (h0 + slot + n * slots) * to.h, group, n_pairs, half);
        }
        return;
    }
    const bool turned = has_turned<LAYOUT, E>(group, n_pairs);
    Weights<T, LAYOUT> weight;
    weight.load(x.weight[which], group, n_pairs, half);
    float su[E], sv[E];
#pragma unroll
    for (int e = 0; e < E; ++e) su[e] = sv[e] = 0.f;
    // All lanes go through the whole loop, those beyond the tokens and heads with rows of zeros that are not stored: where lanes drop out, the sums are
    // kept twice.  The rows of the next item are requested before those of this one are worked on.
    struct Item {
        int h0, b, l;
        Pairs<T, LAYOUT> x[kNormRows], g[kNormRows];
    };
    auto request = [&](Item &i) __attribute__((always_inline)) {
        const T *src = static_cast<const T *>(x.src[which]) + i.b * from.b + i.l * from.l, *g = static_cast<const T *>(x.grad[which]) + i.b * gs.b + i.l * gs.l;
#pragma unroll
        for (int n = 0; n < kNormRows; ++n) {
            const int h = i.h0 + slot + n * slots;
            i.x[n].clear(), i.g[n].clear();
            if (i.l < L && h < heads) {
                i.x[n].template load<STREAM>(src + h * from.h, group, n_pairs, half);
                i.g[n].template load<STREAM>(g + h * gs.h, group, n_pairs, half);
            }
        }
    };
    Item now, next;
    now.h0 = h0;
    place(now.b, now.l);
    Angles<T, LAYOUT> w;
    if (item < last) request(now);
    for (bool fresh = true; item < last; ++item) {
        next.h0 = now.h0 + step, next.b = now.b, next.l = now.l;
        const bool turn_over = next.h0 >= heads;
        if (turn_over) next.h0 = 0, ++tile, place(next.b, next.l);
        if (item + 1 < last) request(next);
        if (fresh) {
            const long at = (long)now.b * L + now.l;
            asm volatile("" : "+s"(freqs));  // (read for every tile: kept, they and their products are 32 registers)
            if (turned) w.template form<true>(freqs, n_pairs, half, group, now.l >= L ? 0 : positions ? positions[at] : now.l - (doc_start ? doc_start[at] : 0), -1.f);
        }
        fresh = turn_over;
        T *dst = static_cast<T *>(x.dst[which]) + now.b * to.b + now.l * to.l;
        const int h = now.h0 + slot;
#pragma unroll
        for (int n = 0; n < kNormRows; ++n) {
            const bool row = now.l < L && h + n * slots < heads;
            float xu[E], xv[E], gu[E], gv[E];
            now.x[n].widen(xu, xv);
            now.g[n].widen(gu, gv);
            if (turned) turn_pairs(gu, gv, w, group, n_pairs, half);
            float r = row_rms<D, GROUPS>(xu, xv, eps), dot = 0.f;
            r = row ? r : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                su[e] = fmaf(gu[e], xu[e] * r, su[e]);
                sv[e] = fmaf(gv[e], xv[e] * r, sv[e]);
                asm volatile("" : "+v"(su[e]), "+v"(sv[e]));  // now: put off, the sums keep the values of all rows alive
                gu[e] *= weight.u[e], gv[e] *= weight.v[e];
                dot = fmaf(gu[e], xu[e], fmaf(gv[e], xv[e], dot));
            }
            const float back = row_sum<GROUPS>(dot) * (r * r) * (1.f / D);
#pragma unroll
            for (int e = 0; e < E; ++e) gu[e] = r * fmaf(-back, xu[e], gu[e]), gv[e] = r * fmaf(-back, xv[e], gv[e]);
            now.g[n].narrow(gu, gv);
            if (row) now.g[n].store(dst + (h + n * slots) * to.h, group, n_pairs, half);
            __builtin_amdgcn_sched_barrier(0);  // row by row: the fp32 values of several leave no room for more waves
        }
        now = next;
    }
    if (!part) return;
    __shared__ float sums[kNormThreads / kWave][D];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        int i, j;
        members_of<LAYOUT, E>(group, e, n_pairs, half, i, j);
        const float u = rows_sum<GROUPS>(su[e]), v = rows_sum<GROUPS>(sv[e]);
        if (lane < GROUPS) sums[wave][i] = u, sums[wave][j] = v;
    }
    __syncthreads();
    if (threadIdx.x < D)
        part[(long)blockIdx.x * D + threadIdx.x] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

// dw of q (blockIdx.y 0) and of k (1): rows of partial sums, four columns per workgroup, a row per thread
__global__ __launch_bounds__(kNormThreads) void norm_weights_kernel(int D, int rows_q, int rows_k, const float *__restrict__ part,
                                                                     float *__restrict__ dq_weight, float *__restrict__ dk_weight) {
    float *out = blockIdx.y ? dk_weight : dq_weight;
    if (!out) return;
    const int rows = blockIdx.y ? rows_k : rows_q, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float *p = part + (blockIdx.y ? (long)rows_q * D : 0) + 4 * blockIdx.x;
    constexpr int N = 4;  // rows of a thread on their way
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    for (int r = threadIdx.x; r < rows; r += N * kNormThreads) {
        float4 v[N];
#pragma unroll
        for (int n = 0; n < N; ++n)
            v[n] = r + n * kNormThreads < rows ? *reinterpret_cast<const float4 *>(p + (long)(r + n * kNormThreads) * D) : float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < N; ++n) sum[0] += v[n].x, sum[1] += v[n].y, sum[2] += v[n].z, sum[3] += v[n].w;
    }
    static_assert(kNormThreads == 256, "a wave per column");
    __shared__ double sums[4][kNormThreads];
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[i][threadIdx.x] = sum[i];
    __syncthreads();
    double x = (sums[wave][lane] + sums[wave][lane + 64]) + (sums[wave][lane + 128] + sums[wave][lane + 192]);
#pragma unroll
    for (int n = 32; n > 0; n /= 2) x += __shfl_xor(x, n);
    if (lane == 0) out[4 * blockIdx.x + wave] = (float)x;
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
    const long want = 3L * units;
    // workgroups by the bytes that a tensor moves: q and k are read twice and written once, v is read and written
    const long heads[3] = {p.Hq, p.Hkv, values ? p.Hkv : 0}, moved[3] = {3 * heads[0], 3 * heads[1], 2 * heads[2]}, all = moved[0] + moved[1] + moved[2];
    g.first[0] = 0;
    for (int i = 0; i < 3; ++i) {
        const long step = (long)(i < 2 ? kNormRows : kMovedRows) * (rows >> g.log_tokens), items = (long)g.tiles_per_row * g.B * ((heads[i] + step - 1) / step);
        long n = (want * moved[i] + all / 2) / all;
        n = n < 1 ? 1 : n;
        g.first[i + 1] = g.first[i] + (int)(n < items ? n : items);
    }
    return g;
}

size_t norm_rope_backward_workspace(const sepattn_norm_rope_params &p) {
    // with and without values a call is cut differently
    const int units = compute_units(), a = norm_rope_grid(p, true, units).first[2], b = norm_rope_grid(p, false, units).first[2];
    return align_up((size_t)(a > b ? a : b) * p.d * sizeof(float), 256);
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
    const bool sums = dq_weight || dk_weight;
    by_layout(p, [&](auto T_, auto D_, auto LAYOUT_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        constexpr PairLayout LAYOUT = decltype(LAYOUT_)::value;
        auto go = [&](auto STREAM_) {
            hipLaunchKernelGGL((norm_rope_backward_kernel<T, D, LAYOUT, decltype(STREAM_)::value>), dim3(g.first[3]), dim3(kNormThreads), 0, st, x,
                               g, p.L, p.rotary_dim / 2, p.eps, freqs, positions, doc_start, sums ? part : nullptr);
        };
        if (LAYOUT != kHalvesOdd && streams(p, (long)p.B * p.L * (3L * (x.heads[0] + x.heads[1]) + 2L * x.heads[2]))) go(std::bool_constant<LAYOUT != kHalvesOdd>{});
        else go(std::false_type{});
    });
    if (!sums) return launch_status();
    if (hipGetLastError() != hipSuccess) return SEPATTN_ERR_HIP;
    hipLaunchKernelGGL(norm_weights_kernel, dim3(p.d / 4, 2), dim3(kNormThreads), 0, st, p.d, g.first[1], g.first[2] - g.first[1], part,
                       dq_weight, dk_weight);
    return launch_status();
}

}  // namespace sepattn
