// Single-query attention over the four-block KV cache in 4 bits (fp4.h), bf16 and fp32 queries, any number of query heads per KV head.
//
// Eq. 1 with one query row per head and M = 1, over the values that the cache stands for.  Every one of them is a bf16 number, so the
// matrix cores work on them as they are, and what is rounded on the way is
//   - nothing of a bf16 query; a fp32 query is three bf16 numbers (24 bits), whose products are added in fp32;
//   - the weights of V: two bf16 numbers (16 bits) for bf16 results, three for fp32;
//   - with positions within the cache the turned key, formed in fp32: two bf16 numbers for bf16 queries, three for fp32.
//
// A workgroup owns one (sequence, KV head, up to 16 of its query heads) and one of `nsplit` slices of the valid entries, its waves blocks of 32
// entries in turn.  Rows go straight from memory into the registers in which they are converted: 16 rows of a block by 4 lane groups,
// (d = 128) 16 bytes a lane, so that a lane has whole blocks of 32 dimensions and one scale; the order of dimensions along a contraction is free,
// and the query's operand follows it.  Rows of a block are requested while the one before it is worked on.  V has to be transposed for the second
// contraction: its converted rows pass through 8 KB of LDS per wave, read back with ds_read_b64_tr_b16.
//
// Operand layouts of 16x16x32 and the order of a block's rows as in decode_wide.hip: row 4g+i of score tile t is row 8g+4t+i of the block, so
// that a lane group's scores are the k-slots that it holds of the weights as B operand.
#include "common.h"
#include "decode_common.h"
#include "fp4.h"
#include "mfma_common.h"
#include "rotary.h"

namespace sepattn {

namespace {

constexpr int kRows = 32;      // entries per block
constexpr int kColumns = 16;   // query heads of a workgroup

__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// XOR permutation of the 16-byte chunks of a V row in LDS (row = 8a + 4t + i): conflict-free for the rows' writes and for transposed reads
template <int D>
__device__ inline int chunk_swizzle(int row) {
    const int i = row & 3, a = row >> 3;
    if (D == 128) return (i << 1) | ((a & 1) << 3) | (a >> 1);
    return (i & 2) | ((a & 1) << 2) | (a >> 1);
}

// maximum / sum over the four lane groups (lanes l, l^16, l^32, l^48)
__device__ inline float groups_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float groups_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// x as a sum of PARTS bf16 numbers: all but the last cut off, so that what they leave is exact
template <int PARTS>
__device__ inline void split_bf16(const f32x8 &x, bf16x8 (&part)[PARTS]) {
    f32x8 rest = x;
#pragma unroll
    for (int i = 0; i < PARTS - 1; ++i) {
        u32x4 packed;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const uint32_t lo = __float_as_uint(rest[e]), hi = __float_as_uint(rest[e + 1]);
            packed[e / 2] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
            rest[e] -= __uint_as_float(lo & 0xFFFF0000u);
            rest[e + 1] -= __uint_as_float(hi & 0xFFFF0000u);
        }
        part[i] = as_bf16x8(packed);
    }
    part[PARTS - 1] = __builtin_convertvector(rest, bf16x8);
}

template <typename T>
struct Precision;
template <>
struct Precision<uint16_t> {
    static constexpr int kQuery = 1, kWeights = 2, kTurned = 2;
};
template <>
struct Precision<float> {
    static constexpr int kQuery = 3, kWeights = 3, kTurned = 3;
};

template <int D>
using RowCodes = uint32_t __attribute__((ext_vector_type(D / 32)));  // a lane's part of a row: D / 4 values

// one output, and lse where it is wanted, from the sums relative to 2^M; no entries: 0 and -inf.  (Entries whose scores are all -inf: NaN and -inf.)
template <typename T>
__device__ inline void finish(int entries, float M, float sum, float o, T *out, float *lse) {
    const float val = entries == 0 ? 0.f : o / sum;
    *out = narrowed<T>(val);
    if (lse) *lse = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2_f;
}

template <typename T, int D, bool ROPE, int NW>
__global__ __launch_bounds__(64 * NW, 2) void decode_fp4_kernel(sepkv_params p, int G, int n_pos, const T *__restrict__ q, Fp4Cache cache,
                                                                 const int32_t *__restrict__ sizes, const float *__restrict__ rope,
                                                                 float *__restrict__ part, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int KSTEPS = D / 32, KS2 = KSTEPS / 2, DB = D / 16;
    constexpr int QP = Precision<T>::kQuery, WP = Precision<T>::kWeights, KP = ROPE ? Precision<T>::kTurned : 1;
    constexpr int PF = D + 2;  // record: max (log2 domain), sum, D unnormalised outputs
    constexpr int RF = D + 4;  // the same in LDS, in whole 16-byte pieces
    constexpr int STAGE = kColumns * RF * 4 > kRows * D * 2 ? kColumns * RF * 4 : kRows * D * 2;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[NW][STAGE];  // V rows of every wave's block; at the end the waves' records

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int nsplit = gridDim.x, split = blockIdx.x, chunks = (G + kColumns - 1) / kColumns;
    const int kv = blockIdx.y / chunks, first = (blockIdx.y % chunks) * kColumns, sq = blockIdx.z;
    const int heads = min(G - first, kColumns), h0 = kv * G + first;
    const long head = (long)sq * p.Hkv + kv;
    const uint8_t *Kc = cache.Kc + head * p.c * (D / 2), *Vc = cache.Vc + head * p.c * (D / 2);
    const Fp4Scales<D> *Ks = reinterpret_cast<const Fp4Scales<D> *>(cache.Ks) + head * p.c,
                       *Vs = reinterpret_cast<const Fp4Scales<D> *>(cache.Vs) + head * p.c;
    const CacheMap cm = cache_map(p, sizes + SEPKV_SIZES_COLS * sq);
    const int nv = cm.n_init + cm.n_sep + cm.n_past + cm.n_loc;
    const int nb = (nv + kRows - 1) / kRows, per = (nb + nsplit - 1) / nsplit * kRows;
    const int e0 = min(split * per, nv), e1 = min(nv, e0 + per);

    // first dimension of this lane's fragment ks: whole rows by the four lane groups; with ROPE both members of every pair are one lane's
    auto dim_of = [&](int ks) { return ROPE ? (ks < KS2 ? 0 : D / 2) + (D / 8) * g + 8 * (ks % KS2) : (D / 4) * g + 8 * ks; };
    bf16x8 query[KSTEPS][QP];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
        const T *src = q + ((long)sq * p.Hq + h0 + min(col, heads - 1)) * D + dim_of(ks);
        if constexpr (sizeof(T) == 2) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(src);
            query[ks][0] = as_bf16x8(col < heads ? x : u32x4{0u, 0u, 0u, 0u});
        } else {
            f32x8 x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = col < heads ? src[e] : 0.f;
            split_bf16<QP>(x, query[ks]);
        }
    }

    const int krow = 8 * (col >> 2) + (col & 3);  // this lane's rows of a block: krow, krow + 4
    struct Rows {
        RowCodes<D> k[2], v[2];
        uint32_t ks[2], vs[2];
    };
    auto request = [&](int eb, Rows &r) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t slot = decode_slot_of(cm, min(eb + krow + 4 * t, e1 - 1));  // entries past the end: the last one (masked)
            const uint8_t *k = Kc + slot * (D / 2), *v = Vc + slot * (D / 2) + g * (D / 8);
            if constexpr (ROPE) {  // D / 8 values of each half
                using Half = uint32_t __attribute__((ext_vector_type(KS2)));
                const Half a = __builtin_nontemporal_load(reinterpret_cast<const Half *>(k + g * (D / 16))),
                           b = __builtin_nontemporal_load(reinterpret_cast<const Half *>(k + D / 4 + g * (D / 16)));
#pragma unroll
                for (int ks = 0; ks < KS2; ++ks) r.k[t][ks] = a[ks], r.k[t][ks + KS2] = b[ks];
            } else {
                r.k[t] = __builtin_nontemporal_load(reinterpret_cast<const RowCodes<D> *>(k + g * (D / 8)));
            }
            r.v[t] = __builtin_nontemporal_load(reinterpret_cast<const RowCodes<D> *>(v));
            r.ks[t] = __builtin_nontemporal_load(Ks + slot), r.vs[t] = __builtin_nontemporal_load(Vs + slot);
        }
    };

    // cos / sin of the lane's two rows' places within a block
    float rc[2][KS2][8], rs[2][KS2][8];
    if constexpr (ROPE) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float *row = rope + (long)min(krow + 4 * t, n_pos - 1) * D + (D / 8) * g;
#pragma unroll
            for (int ks = 0; ks < KS2; ++ks)
#pragma unroll
                for (int e = 0; e < 8; ++e) rc[t][ks][e] = row[8 * ks + e], rs[t][ks][e] = row[D / 2 + 8 * ks + e];
        }
    }

    const uint32_t v_lds = lds_addr(&smem[wave][0]);
    const int vrow = 8 * g + (col >> 2);  // transposed reads: rows vrow, vrow + 4, columns 16 db + 4 (col % 4)
    const uint32_t kswz = chunk_swizzle<D>(krow), vswz = chunk_swizzle<D>(vrow);  // the same for rows + 4
    const uint32_t vwrite = v_lds + krow * D * 2, vread = v_lds + vrow * D * 2 + ((col & 1) << 3);
    const float sl2 = p.scale * kLog2e_f;
    f32x4 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    int eb = e0 + wave * kRows;
    Rows now, next;
    if (eb < e1) request(eb, now);
    for (; eb < e1; eb += NW * kRows, now = next) {
        if (eb + NW * kRows < e1) request(eb + NW * kRows, next);
        // ---- scores
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if constexpr (ROPE) {
            const float *base = rope + (long)(nv - 1 - eb) * D + (D / 8) * g;
#pragma unroll
            for (int ks = 0; ks < KS2; ++ks) {
                float bc[8], bs[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) bc[e] = base[8 * ks + e], bs[e] = base[D / 2 + 8 * ks + e];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float x[8], y[8];
                    fp4_to_f32(now.k[t][ks], fp4_scale(now.ks[t], D == 128 ? g >> 1 : 0), x);
                    fp4_to_f32(now.k[t][ks + KS2], fp4_scale(now.ks[t], D == 128 ? 2 + (g >> 1) : 1), y);
                    f32x8 u, v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {  // R(-distance): the distance is that of the block's first entry minus the row's place
                        const float c = fmaf(bs[e], rs[t][ks][e], bc[e] * rc[t][ks][e]), sn = fmaf(-bc[e], rs[t][ks][e], bs[e] * rc[t][ks][e]);
                        u[e] = fmaf(y[e], sn, x[e] * c);
                        v[e] = fmaf(-x[e], sn, y[e] * c);
                    }
                    bf16x8 ku[KP], kv_[KP];
                    split_bf16<KP>(u, ku);
                    split_bf16<KP>(v, kv_);
#pragma unroll
                    for (int i = 0; i < KP; ++i)
#pragma unroll
                        for (int j = 0; j < QP; ++j)
                            if (i + j < (KP > QP ? KP : QP)) {  // the products of two small parts are below the last one's rounding
                                s[t] = mfma16(ku[i], query[ks][j], s[t]);
                                s[t] = mfma16(kv_[i], query[ks + KS2][j], s[t]);
                            }
                }
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 a = __builtin_bit_cast(bf16x8, fp4_to_bf16(now.k[t][ks], fp4_scale(now.ks[t], D == 128 ? g : g >> 1)));
#pragma unroll
                    for (int j = 0; j < QP; ++j) s[t] = mfma16(a, query[ks][j], s[t]);
                }
        }
        // ---- V rows into LDS
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                const fp4_bf16x8 v = fp4_to_bf16(now.v[t][ks], fp4_scale(now.vs[t], D == 128 ? g : g >> 1));
                lds_write_b128_at(vwrite + 4 * t * D * 2 + (((uint32_t)(KSTEPS * g + ks) ^ kswz) << 4), __builtin_bit_cast(f32x4, v));
            }
        // ---- weights
        float x[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};  // rows 8g .. 8g+7 of the block
        const int n_valid = e1 - eb;
        if (n_valid < kRows) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 8 * g + i < n_valid ? x[i] : -INFINITY;
        }
        const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))) * sl2;
        // the running maximum is raised only where a weight would pass 2^8: with fp32 sums a common factor costs nothing
        if (__builtin_amdgcn_ballot_w64(top > m_run + 8.f)) {
            const float m_new = fmaxf(m_run, groups_max(top));
            const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= alpha;
            m_run = m_new;
        }
        const float shift = m_run == -INFINITY ? 0.f : -m_run;
        f32x8 pr;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            pr[i] = __builtin_amdgcn_exp2f(fmaf(x[i], sl2, shift));
            l_run += pr[i];
        }
        bf16x8 w[WP];
        split_bf16<WP>(pr, w);
        // ---- output
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const bf16x8 v = lds_read_tr_at(vread + (((uint32_t)(2 * db + ((col & 3) >> 1)) ^ vswz) << 4), 4 * D * 2);
#pragma unroll
            for (int i = 0; i < WP; ++i) acc[db] = mfma16(v, w[i], acc[db]);
        }
    }

    // ---- the waves' states: D outputs, max, sum of a head
    const float l_tot = groups_sum(l_run);
    if (l_tot != l_tot) m_run = 0.f;  // a NaN has to reach the sum even if there is no finite score
    if (col < heads) {
        float *r = reinterpret_cast<float *>(&smem[wave][0]) + col * RF;
        if (g == 0) *reinterpret_cast<float2 *>(r + D) = float2{m_run, l_tot};
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(r + 16 * db + 4 * g) = acc[db];
    }
    __syncthreads();
    for (int item = tid; item < heads * D; item += 64 * NW) {
        const int h = item / D, c = item % D;
        float M = -INFINITY, lsum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, reinterpret_cast<const float *>(&smem[w][0])[h * RF + D]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float *r = reinterpret_cast<const float *>(&smem[w][0]) + h * RF;
            const float wgt = r[D] == -INFINITY ? 0.f : exp2f(r[D] - M);
            lsum = fmaf(wgt, r[D + 1], lsum);
            o = fmaf(wgt, r[c], o);
        }
        const long sh = (long)sq * p.Hq + h0 + h;
        if (nsplit == 1) {
            finish<T>(nv, M, lsum, o, out + sh * D + c, lse && c == 0 ? lse + sh : nullptr);
        } else {
            float *rec = part + (sh * nsplit + split) * PF;
            rec[2 + c] = o;
            if (c == 0) rec[0] = M, rec[1] = lsum;
        }
    }
}

// the slices' records of a (sequence, query head)
template <typename T, int D>
__global__ void merge_fp4_kernel(sepkv_params p, int nsplit, const int32_t *__restrict__ sizes, const float *__restrict__ part, T *__restrict__ out,
                                 float *__restrict__ lse) {
    constexpr int PF = D + 2;
    const long sh = blockIdx.x;
    const CacheMap cm = cache_map(p, sizes + SEPKV_SIZES_COLS * (sh / p.Hq));
    const int c = threadIdx.x;
    const float *r = part + sh * nsplit * PF;
    float M = -INFINITY, lsum = 0.f, o = 0.f;
    for (int k = 0; k < nsplit; ++k) M = fmaxf(M, r[k * PF]);
    for (int k = 0; k < nsplit; ++k) {
        const float *rec = r + k * PF;
        const float wgt = rec[0] == -INFINITY ? 0.f : exp2f(rec[0] - M);
        lsum = fmaf(wgt, rec[1], lsum);
        o = fmaf(wgt, rec[2 + c], o);
    }
    finish<T>(cm.n_init + cm.n_sep + cm.n_past + cm.n_loc, M, lsum, o, out + sh * D + c, lse && c == 0 ? lse + sh : nullptr);
}

int chunks_of(const sepkv_params &p) { return (p.Hq / p.Hkv + kColumns - 1) / kColumns; }

int slices_of(const sepkv_params &p, int units) {
    const long pairs = (long)p.S * p.Hkv * chunks_of(p), fit = 2L * units / pairs;
    const int nb = (p.c + kRows - 1) / kRows;
    long n = (nb + 7) / 8;
    if (n > fit) n = fit;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace

size_t decode_fp4_workspace(const sepkv_params &p) {
    return align_up((size_t)p.S * p.Hq * slices_of(p, compute_units()) * (p.d + 2) * sizeof(float), 256);
}

int launch_decode_fp4(const sepkv_params &p, const void *q, const Fp4Cache &cache, const int32_t *sizes, const float *rope, int n_pos, void *out,
                      float *lse, void *ws, hipStream_t st) {
    const int G = p.Hq / p.Hkv, nsplit = slices_of(p, compute_units());
    float *part = static_cast<float *>(ws);
    constexpr int NW = 8;
    auto go = [&](auto T_, auto D_, auto ROPE_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        {
            ProfScope prof(SEPATTN_K_DECODE_SPLIT, st);
            hipLaunchKernelGGL((decode_fp4_kernel<T, D, decltype(ROPE_)::value, NW>), dim3(nsplit, p.Hkv * chunks_of(p), p.S), dim3(64 * NW), 0, st, p, G,
                               n_pos, static_cast<const T *>(q), cache, sizes, rope, part, static_cast<T *>(out), lse);
        }
        if (nsplit == 1) return launch_status();
        if (hipGetLastError() != hipSuccess) return (int)SEPATTN_ERR_HIP;
        ProfScope prof(SEPATTN_K_DECODE_MERGE, st);
        hipLaunchKernelGGL((merge_fp4_kernel<T, D>), dim3(p.S * p.Hq), dim3(D), 0, st, p, nsplit, sizes, part, static_cast<T *>(out), lse);
        return launch_status();
    };
    auto with = [&](auto T_, auto D_) { return rope ? go(T_, D_, std::true_type{}) : go(T_, D_, std::false_type{}); };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (p.dtype == SEPATTN_BF16) return p.d == 64 ? with(uint16_t{}, D64{}) : with(uint16_t{}, D128{});
    return p.d == 64 ? with(float{}, D64{}) : with(float{}, D128{});
}

}  // namespace sepattn
