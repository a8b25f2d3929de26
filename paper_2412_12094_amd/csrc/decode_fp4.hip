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
// What bounds it, d = 128, bf16, 32 query heads on 8 KV heads.  Long caches: memory.  4 sequences of up to 53019 entries, 137 MB in 26.8 us, 5.1 TB/s, and
// 4.6 for the merge launch.  Shorter ones: vector instructions and the start.  A block is 190 of them (64 convert, 24 split the weights), with positions
// 640: 128 form the angles, 128 turn, 192 split the turned keys.  A wave alone on its SIMD needs 1.8 us for a block with positions, three together 1.2
// each, so kResident is as much as fits without a spill: a spilled register is waited for with every load before it.  32 sequences of 1 to 3277
// entries, 60 MB, 17.9 us; with positions 28.9.  The other half of both is the start (launch, slice, first rows: 6 us) and the sum of the slices (4).
// The remainder of a cut number as one dot product of bf16 pairs instead of a mask and a subtraction took 72 instructions out of the 640 and changed no
// time, nor did a second block on its way (d = 64: 17.4 -> 18.9).  The second halves of turned keys as fp32 products (16x16x4) instead of two parts: 96
// instructions fewer, 29.8 -> 34.8: eight products that wait for each other.
//
// Operand layouts of 16x16x32 and the order of a block's rows as in decode_wide.hip: row 4g+i of score tile t is row 8g+4t+i of the block, so
// that a lane group's scores are the k-slots that it holds of the weights as B operand.
#include "common.h"
#include "decode_common.h"
#include "decode_fp4.h"
#include "fp4.h"
#include "mfma_common.h"
#include "rotary.h"

namespace sepattn {

namespace {

// waves per SIMD that the registers have to leave room for
template <typename T, int D, bool ROPE>
constexpr int kResident = sizeof(T) == 2 ? (ROPE && D == 128 ? 3 : 4) : (D == 128 ? (ROPE ? 2 : 3) : (ROPE ? 3 : 4));
constexpr int kWaves = kMxWaves, kRows = kMxRows, kColumns = kMxColumns, kMostSlices = kMxMostSlices;
// a cache line for each word in which slices are counted: side by side, 8 sequences of up to 8192 entries took 18.3 us instead of 14.2, with positions 28.3
// instead of 24.5
constexpr int kWordPitch = 128;
__host__ __device__ inline size_t words_bytes(long pairs) { return align_up((size_t)pairs * kWordPitch, 256); }

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

// of another lane of the same sixteen: row_ror 8 (0x128) and 4 (0x124), quad_perm [2, 3, 0, 1] (0x4E) and [1, 0, 3, 2] (0xB1)
template <int CTRL>
__device__ inline float dpp_of(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
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

// Weights are 2^(x sl2 - m) by one fma, with m the rounded product of the largest x.  What that rounding left is in every exponent, up to half a step of m:
// a common factor, which costs nothing until it leaves fp32 (m = 2^31: steps of 256).  From here on the products are rounded as m is.
constexpr float kFarMaximum = 16777216.f;  // 2^24, steps of 2
__device__ inline float rounded_product(float x, float y) {
#pragma clang fp contract(off)
    const float z = x * y;
    return z;
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

// The valid entries as runs of consecutive slots: entry e of a run sits in slot e + off, up to `end`.  All scalar.
struct Runs {
    int n1, n2, nv, sep_end, win_end, sep_off, win_off, s, wcap;
    __device__ Runs(const CacheMap &m)
        : n1(m.n_init), n2(m.n_init + m.n_sep), nv(m.n_init + m.n_sep + m.n_past + m.n_loc), s(m.s), wcap(m.wcap) {
        sep_off = m.a + m.sep_head - n1, win_off = m.a + m.s + m.win_head - n2;
        sep_end = min(n1 + m.s - m.sep_head, n2), win_end = min(n2 + m.wcap - m.win_head, nv);  // where the rings wrap
    }
    // the run of entry e (the same in all lanes)
    __device__ int find(int e, int &off) const {
        off = 0;
        int end = n1;
        if (e >= n1) off = sep_off, end = sep_end;
        if (e >= sep_end && e >= n1) off = sep_off - s, end = n2;
        if (e >= n2) off = win_off, end = win_end;
        if (e >= win_end && e >= n2) off = win_off - wcap, end = nv;
        return end;
    }
    // slot of entry e (of the lane's own)
    __device__ int slot(int e) const {
        int off = e >= sep_end ? sep_off - s : sep_off;
        off = e < n1 ? 0 : off;
        const int w = e >= win_end ? win_off - wcap : win_off;
        return e + (e >= n2 ? w : off);
    }
};

// A slice, which every workgroup finds by itself from the sizes, a sequence per lane (MxPlan, decode_fp4.h).
struct Slice {
    int sq, index, count, before;  // sequence, which of its slices, how many it has (0: there is no such slice), slices of the sequences in front of it
    CacheMap map;
};
// sums over the lanes up to this one
__device__ inline int lanes_sum(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15, 31: of a row to the next, of two to the last two
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}
__device__ inline int blocks_of(const CacheMap &m) { return (m.n_init + m.n_sep + m.n_past + m.n_loc + kRows - 1) / kRows; }
// slice number `want`; `want` < 0: the first one of sequence -1 - want
__device__ inline Slice slice_of(const sepkv_params &p, const MxPlan &plan, const int32_t *__restrict__ sizes, int want) {
    if (plan.most == 1) {
        if (want >= p.S) return {0, 0, 0, 0, {}};
        const int sq = want < 0 ? -1 - want : want;
        return {sq, 0, 1, sq, cache_map(p, sizes + SEPKV_SIZES_COLS * sq)};
    }
    if (p.S == 1) {
        const CacheMap m = cache_map(p, sizes);
        const int nb = blocks_of(m), n = __builtin_amdgcn_readfirstlane(mx_slices(plan, nb, reciprocal(mx_share(plan, nb))));
        return {0, max(want, 0), want < n ? n : 0, 0, m};
    }
    const int lane = threadIdx.x & 63;
    CacheMap m;
    int total = 0, before = 0;
    for (int s0 = (p.S - 1) & ~63; s0 >= 0; s0 -= 64) {  // (the first ones last: theirs are at hand then)
        m = cache_map(p, sizes + SEPKV_SIZES_COLS * min(s0 + lane, p.S - 1));
        total += s0 + lane < p.S ? blocks_of(m) : 0;
    }
    const float per_share = reciprocal(mx_share(plan, __builtin_amdgcn_readlane(lanes_sum(total), 63)));
    for (int s0 = 0;; s0 += 64) {
        const int n = s0 + lane < p.S ? mx_slices(plan, blocks_of(m), per_share) : 0, upto = lanes_sum(n), front = before + upto - n;
        const uint64_t found = __builtin_amdgcn_ballot_w64(want < 0 ? s0 + lane == -1 - want : want >= front && want < front + n);
        if (found) {
            const int l = __builtin_ctzll(found);
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
            return {s0 + l, max(want - of(front), 0), of(n), of(front),
                    {of(m.n_init), of(m.n_sep), of(m.n_past), of(m.n_loc), of(m.sep_head), of(m.win_head), p.a, p.s, m.wcap}};
        }
        if (s0 + 64 >= p.S) return {0, 0, 0, 0, m};
        before += __builtin_amdgcn_readlane(upto, 63);
        m = cache_map(p, sizes + SEPKV_SIZES_COLS * min(s0 + 64 + lane, p.S - 1));
    }
}

__device__ inline Slice find_slice(const sepkv_params &p, const MxPlan &plan, const int32_t *__restrict__ sizes, int want) {
    const Slice x = slice_of(p, plan, sizes, want);
    auto s = [](int v) { return __builtin_amdgcn_readfirstlane(v); };  // (the same in all lanes, which the compiler does not see)
    return {s(x.sq), s(x.index), s(x.count), s(x.before),
            {s(x.map.n_init), s(x.map.n_sep), s(x.map.n_past), s(x.map.n_loc), s(x.map.sep_head), s(x.map.win_head), p.a, p.s, p.c - p.a - p.s}};
}

template <int D>
constexpr int kMergeParts = 256 / (D / 2);  // threads of the merge launch that share two columns

// ADD: the slices of a sequence are added by the workgroup that finishes last.  Otherwise, where there are several, they are left to a merge launch.
template <typename T, int D, bool ROPE, bool ADD>
__global__ __launch_bounds__(64 * kWaves, (kResident<T, D, ROPE>)) void decode_fp4_kernel(
    sepkv_params p, MxPlan plan, int G, int n_pos, const T *__restrict__ q, Fp4Cache cache, const int32_t *__restrict__ sizes, const float *__restrict__ rope,
    uint64_t one, char *__restrict__ ws, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int KSTEPS = D / 32, KS2 = KSTEPS / 2, DB = D / 16, NW = kWaves;
    constexpr int QP = Precision<T>::kQuery, WP = Precision<T>::kWeights, KP = ROPE ? Precision<T>::kTurned : 1;
    constexpr int PF = D + 2;  // record: max (log2 domain), sum, D unnormalised outputs
    constexpr int RF = D + 4;  // the same in LDS, in whole 16-byte pieces
    constexpr int STAGE = kColumns * RF * 4 > kRows * D * 2 ? kColumns * RF * 4 : kRows * D * 2;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[NW][STAGE];  // V rows of every wave's block; at the end the waves' records
    __shared__ __attribute__((aligned(16))) float base_s[ROPE ? NW : 1][2][ROPE ? D : 4];  // table rows of every wave's block

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    // the table's rows 0 .. 31, which pass through LDS below: on their way while the slice is found
    constexpr int CH = D / 4, TABLE = ROPE ? kRows * CH / (64 * NW) : 1;
    f32x4 table[TABLE];
    if constexpr (ROPE) {
#pragma unroll
        for (int n = 0; n < TABLE; ++n) {
            const int i = tid + n * 64 * NW, r = i / CH;
            table[n] = *reinterpret_cast<const f32x4 *>(rope + (long)min(r, n_pos - 1) * D + (i % CH) * 4);
        }
    }
    const int chunks = (G + kColumns - 1) / kColumns, kv = blockIdx.x / chunks, first = (blockIdx.x % chunks) * kColumns;
    const Slice slice = find_slice(p, plan, sizes, blockIdx.y);
    if (slice.count == 0) return;
    const int sq = slice.sq, nsplit = slice.count, split = slice.index;
    const int heads = min(G - first, kColumns), h0 = kv * G + first;
    const long head = (long)sq * p.Hkv + kv;
    const uint8_t *Kc = cache.Kc + head * p.c * (D / 2), *Vc = cache.Vc + head * p.c * (D / 2);
    const uint8_t *Ks = cache.Ks + head * p.c * (D / 32), *Vs = cache.Vs + head * p.c * (D / 32);
    const Runs runs(slice.map);
    const int nv = runs.nv, nb = (nv + kRows - 1) / kRows;
    // as even as can be: the first ones have a block more
    const int each = nsplit == 1 ? nb : __builtin_amdgcn_readfirstlane(small_quotient(nb, reciprocal(nsplit))), more = nb - each * nsplit;
    const int e0 = min((split * each + min(split, more)) * kRows, nv), e1 = min(e0 + (each + (split < more)) * kRows, nv);

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

    typedef const __attribute__((address_space(1))) char *GlobalBytes;
    auto turns = (GlobalBytes)rope;
    asm volatile("" : "+s"(turns));  // (known as never written, its first loads would be moved behind the barriers)
    const int krow = 8 * (col >> 2) + (col & 3);  // this lane's rows of a block: krow, krow + 4
    struct Rows {
        RowCodes<D> k[2], v[2];
        Fp4Scales<D> ks[2], vs[2];  // (as they are loaded: widened here, the half words of d = 64 would be waited for at once)
        float base[2][ROPE ? D / 64 : 1];  // value(s) lane, lane + 64 of the table rows of the distances of entries 0 and 4 of the block
    };
    // slots of the lane's rows of a block; entries past the end: the last one (masked)
    int run_end = -1, run_off = 0;
    auto find_slots = [&](int eb, uint32_t (&slot)[2]) __attribute__((always_inline)) {
        if (eb >= run_end) run_end = min(runs.find(eb, run_off), e1);
        if (eb + kRows <= run_end) {  // one run of slots
            slot[0] = eb + run_off + krow;
            slot[1] = slot[0] + 4;
        } else {
            slot[0] = runs.slot(min(eb + krow, e1 - 1));
            slot[1] = runs.slot(min(eb + krow + 4, e1 - 1));
        }
    };
    auto request_keys = [&](Rows &rows, int eb, const uint32_t (&slot)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t off = slot[t] * (D / 2) + g * (ROPE ? D / 16 : D / 8);  // (c d / 2 < 2^29)
            if constexpr (ROPE) {  // D / 8 values of each half
                using Half = uint32_t __attribute__((ext_vector_type(KS2)));
                const Half a = __builtin_nontemporal_load(reinterpret_cast<const Half *>(Kc + (size_t)off)),
                           b = __builtin_nontemporal_load(reinterpret_cast<const Half *>(Kc + (size_t)(off + D / 4)));
#pragma unroll
                for (int ks = 0; ks < KS2; ++ks) rows.k[t][ks] = a[ks], rows.k[t][ks + KS2] = b[ks];
#pragma unroll
                for (int i = 0; i < D / 64; ++i)  // (4 c d < 2^32; beyond the end: masked)
                    rows.base[t][i] = *(const __attribute__((address_space(1))) float *)(turns + (size_t)((uint32_t)(max(nv - 1 - eb - 4 * t, 0) * D + 64 * i + lane) * 4u));
            } else {
                rows.k[t] = __builtin_nontemporal_load(reinterpret_cast<const RowCodes<D> *>(Kc + (size_t)off));
            }
            rows.ks[t] = __builtin_nontemporal_load(reinterpret_cast<const Fp4Scales<D> *>(Ks + (size_t)(slot[t] * (D / 32))));
        }
    };
    auto request_values = [&](Rows &rows, const uint32_t (&slot)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            rows.v[t] = __builtin_nontemporal_load(reinterpret_cast<const RowCodes<D> *>(Vc + (size_t)(slot[t] * (D / 2) + g * (D / 8))));
            rows.vs[t] = __builtin_nontemporal_load(reinterpret_cast<const Fp4Scales<D> *>(Vs + (size_t)(slot[t] * (D / 32))));
        }
    };

    int eb = e0 + wave * kRows;
    // cos / sin of the place of the lane's row krow within a block (that of row krow + 4 is the same behind entry 4): the table's rows 0 .. 31 pass through
    // LDS, where the V stages lie later, with the 16-byte chunks of a row permuted (row by row from memory, an instruction is 64 pieces of 16 bytes)
    float rc[KS2][8], rs[KS2][8];
    constexpr int STEP = NW * kRows;
    Rows rows;
    auto request_first = [&] {  // (of any slot where the wave has no block: behind a branch, as below, these loads would be waited for with all before)
        uint32_t slot[2];
        find_slots(eb, slot);
        slot[0] = min(slot[0], (uint32_t)p.c - 1u), slot[1] = min(slot[1], (uint32_t)p.c - 1u);  // a sequence without entries has none to repeat
        request_keys(rows, eb, slot);
        __builtin_amdgcn_sched_barrier(0);  // in the loop's order: else it waits for what the first round has on its way
        request_values(rows, slot);
        __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (ROPE) {
        static_assert(kRows * D * 4 <= NW * STAGE, "the table's rows fit the stages");
        request_first();
        const uint32_t t_lds = lds_addr(&smem[0][0]);
#pragma unroll
        for (int n = 0; n < TABLE; ++n) {
            const int i = tid + n * 64 * NW, r = i / CH;
            lds_write_b128_at(t_lds + r * D * 4 + (((uint32_t)(i % CH) ^ chunk_swizzle<128>(r)) << 4), table[n]);
        }
        auto barrier = [] {  // of LDS alone: a __syncthreads would also wait for the rows
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        barrier();
#pragma unroll
        for (int ks = 0; ks < KS2; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t row = t_lds + krow * D * 4, chunk = ((D / 8) * g + 8 * ks + 4 * h) / 4, swz = chunk_swizzle<128>(krow);
                const f32x4 c = lds_read_f32x4_at(row + ((chunk ^ swz) << 4)), sn = lds_read_f32x4_at(row + (((D / 8 + chunk) ^ swz) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) rc[ks][4 * h + e] = c[e], rs[ks][4 * h + e] = sn[e];
            }
        barrier();
    } else {
        request_first();
    }

    const uint32_t v_lds = lds_addr(&smem[wave][0]), b_lds = lds_addr(&base_s[ROPE ? wave : 0][0][0]);
    const int vrow = 8 * g + (col >> 2);  // transposed reads: rows vrow, vrow + 4, columns 16 db + 4 (col % 4)
    const uint32_t kswz = chunk_swizzle<D>(krow), vswz = chunk_swizzle<D>(vrow);  // the same for rows + 4
    // Stages start at multiples of 256 bytes, so that the permuted chunk is an XOR into the address: one instruction per access in the loop (kept there by
    // the empty statements), not a register per access
    static_assert(STAGE % 256 == 0, "");
    uint32_t vwrite = v_lds + krow * D * 2 + (((uint32_t)(KSTEPS * g) ^ kswz) << 4);
    uint32_t vread = v_lds + vrow * D * 2 + ((col & 1) << 3) + ((((uint32_t)(col & 3) >> 1) ^ vswz) << 4);
    const float sl2 = p.scale * kLog2e_f;
    f32x4 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    for (; eb < e1; eb += STEP) {
        // (requested in any case, beyond the end as the last entry again: behind a branch the compiler could not count the loads, and would wait for all)
        uint32_t next[2];
        find_slots(eb + STEP, next);
        // ---- scores
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if constexpr (ROPE) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < D / 64; ++i) base_s[wave][t][64 * i + lane] = rows.base[t][i];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ks = 0; ks < KS2; ++ks) {
                    f32x4 bc[2], bs[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bc[h] = lds_read_f32x4_at(b_lds + (t * D + (D / 8) * g + 8 * ks + 4 * h) * 4);
                        bs[h] = lds_read_f32x4_at(b_lds + (t * D + D / 2 + (D / 8) * g + 8 * ks + 4 * h) * 4);
                    }
                    float x[8], y[8];
                    fp4_to_f32(rows.k[t][ks], fp4_scale(rows.ks[t], D == 128 ? g >> 1 : 0), x);
                    fp4_to_f32(rows.k[t][ks + KS2], fp4_scale(rows.ks[t], D == 128 ? 2 + (g >> 1) : 1), y);
                    f32x8 u, v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {  // R(-distance): the distance is that of the block's entry 0 (4) minus the row's place behind it
                        const float c0 = bc[e >> 2][e & 3], s0 = bs[e >> 2][e & 3];
                        const float c = fmaf(s0, rs[ks][e], c0 * rc[ks][e]), sn = fmaf(-c0, rs[ks][e], s0 * rc[ks][e]);
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
                    __builtin_amdgcn_sched_barrier(0);  // one piece at a time: their values together do not leave room for three waves
                }
        } else {
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 a = __builtin_bit_cast(bf16x8, fp4_to_bf16(rows.k[t][ks], fp4_scale(rows.ks[t], D == 128 ? g : g >> 1)));
#pragma unroll
                    for (int j = 0; j < QP; ++j) s[t] = mfma16(a, query[ks][j], s[t]);
                }
        }
        __builtin_amdgcn_sched_barrier(0);
        request_keys(rows, eb + STEP, next);
        // ---- V rows into LDS
        asm volatile("" : "+v"(vwrite), "+v"(vread));
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                const fp4_bf16x8 v = fp4_to_bf16(rows.v[t][ks], fp4_scale(rows.vs[t], D == 128 ? g : g >> 1));
                lds_write_b128_at((vwrite ^ (uint32_t)(ks << 4)) + 4 * t * D * 2, __builtin_bit_cast(f32x4, v));
            }
        __builtin_amdgcn_sched_barrier(0);
        request_values(rows, next);
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
        float factor = sl2, shift = m_run == -INFINITY ? 0.f : -m_run;
        if (__builtin_amdgcn_ballot_w64(fabsf(shift) >= kFarMaximum)) {
            const bool far = fabsf(shift) >= kFarMaximum;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = far ? rounded_product(x[i], sl2) + shift : x[i];
            factor = far ? 1.f : factor, shift = far ? 0.f : shift;
        }
        f32x8 pr;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            pr[i] = __builtin_amdgcn_exp2f(fmaf(x[i], factor, shift));
            l_run += pr[i];
        }
        bf16x8 w[WP];
        split_bf16<WP>(pr, w);
        // ---- output, by four independent sums at a time (32 sequences 18.6 -> 17.9 us: one after the other, a product waits for the one before)
        constexpr int VB = 4;
#pragma unroll
        for (int db = 0; db < DB; db += VB) {
            bf16x8 v[VB];
#pragma unroll
            for (int x = 0; x < VB; ++x) v[x] = lds_read_tr_at(vread ^ (uint32_t)((db + x) << 5), 4 * D * 2);
#pragma unroll
            for (int i = 0; i < WP; ++i)
#pragma unroll
                for (int x = 0; x < VB; ++x) acc[db + x] = mfma16(v[x], w[i], acc[db + x]);
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
    // the word in which this pair's slices are counted, and the records behind all words
    const long pair = head * chunks + first / kColumns;
    uint64_t *const arrived = reinterpret_cast<uint64_t *>(ws + pair * kWordPitch);
    float *const recs = reinterpret_cast<float *>(ws + words_bytes((long)p.S * p.Hkv * chunks)) + ((long)slice.before * p.Hq + h0 * nsplit) * PF;
    uint64_t seen = 0;
    if (ADD && nsplit > 1) {
        if (tid == 0) seen = arrival_seen(arrived);
    }
    for (int item = tid; item < heads * (D / 2); item += 64 * NW) {  // two columns per thread
        const int h = item / (D / 2), c2 = item % (D / 2);
        float2 ml[NW], o[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float *r = reinterpret_cast<const float *>(&smem[w][0]) + h * RF;
            ml[w] = *reinterpret_cast<const float2 *>(r + D), o[w] = *reinterpret_cast<const float2 *>(r + 2 * c2);
        }
        float M = -INFINITY, lsum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[w].x);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float wgt = ml[w].x == -INFINITY ? 0.f : exp2f(ml[w].x - M);
            lsum = fmaf(wgt, ml[w].y, lsum), o0 = fmaf(wgt, o[w].x, o0), o1 = fmaf(wgt, o[w].y, o1);
        }
        const long sh = (long)sq * p.Hq + h0 + h;
        if (nsplit == 1) {
            finish<T>(nv, M, lsum, o0, out + sh * D + 2 * c2, nullptr);
            finish<T>(nv, M, lsum, o1, out + sh * D + 2 * c2 + 1, lse && c2 == 0 ? lse + sh : nullptr);
        } else {
            float *rec = recs + (h * nsplit + split) * PF;
            if constexpr (ADD) {
                publish(rec + 2 + 2 * c2, float2{o0, o1});
                if (c2 == 0) publish(rec, float2{M, lsum});
            } else {
                *reinterpret_cast<float2 *>(rec + 2 + 2 * c2) = float2{o0, o1};
                if (c2 == 0) *reinterpret_cast<float2 *>(rec) = float2{M, lsum};
            }
        }
    }
    if (!ADD || nsplit == 1) return;

    // ---- the workgroup that finishes last adds the slices' records, in slice order, whichever it is
    __shared__ int last_s;
    if (tid == 0) arrival_ready(arrived, seen, one, nsplit);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part of the record is where every XCD sees it
    __syncthreads();
    if (tid == 0) last_s = arrives_last(arrived, one, nsplit);
    __syncthreads();
    if (!last_s) return;
    if (tid == 0) arrival_reset(arrived);
    for (int item = tid; item < heads * (D / 2); item += 64 * NW) {
        const int h = item / (D / 2), c2 = item % (D / 2);
        const float *rec = recs + h * nsplit * PF;
        float2 ml[kMxMostAdded], o[kMxMostAdded];
#pragma unroll
        for (int k = 0; k < kMxMostAdded; ++k)
            if (k < nsplit) ml[k] = fetch_published(rec + k * PF), o[k] = fetch_published(rec + k * PF + 2 + 2 * c2);
        // every sum in the order in which merge_fp4_kernel forms it: captured calls, which that kernel finishes, give the same bits
        float M = -INFINITY, wgt[kMxMostAdded], sum[kMxMostAdded], o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int k = 0; k < kMxMostAdded; ++k)
            if (k < nsplit) M = fmaxf(M, ml[k].x);
#pragma unroll
        for (int k = 0; k < kMxMostAdded; ++k) {
            wgt[k] = k >= nsplit || ml[k].x == -INFINITY ? 0.f : exp2f(ml[k].x - M);
            sum[k] = k < nsplit ? wgt[k] * ml[k].y : 0.f;
        }
#pragma unroll
        for (int x = kMxMostAdded / 2; x > 0; x /= 2)
#pragma unroll
            for (int k = 0; k < x; ++k) sum[k] += sum[k + x];
        const float lsum = sum[0];
#pragma unroll
        for (int i = 0; i < kMergeParts<D>; ++i) {
            float a0 = 0.f, a1 = 0.f;
#pragma unroll
            for (int k = i; k < kMxMostAdded; k += kMergeParts<D>)
                if (k < nsplit) a0 = fmaf(wgt[k], o[k].x, a0), a1 = fmaf(wgt[k], o[k].y, a1);
            o0 += a0, o1 += a1;
        }
        const long sh = (long)sq * p.Hq + h0 + h;
        finish<T>(nv, M, lsum, o0, out + sh * D + 2 * c2, nullptr);
        finish<T>(nv, M, lsum, o1, out + sh * D + 2 * c2 + 1, lse && c2 == 0 ? lse + sh : nullptr);
    }
}

// The slices' records of a (sequence, query head), where there are several.  Thread k of the first wave has slice k's maximum and sum (there are at most
// 64), all of them its weight through LDS; the records are requested before that is known.
template <typename T, int D>
__global__ __launch_bounds__(256) void merge_fp4_kernel(sepkv_params p, MxPlan plan, const int32_t *__restrict__ sizes, const float *__restrict__ part,
                                                         T *__restrict__ out, float *__restrict__ lse) {
    constexpr int PF = D + 2, PARTS = kMergeParts<D>, N = kMostSlices / PARTS;  // a thread: two columns, every PARTS-th slice
    __shared__ float weight[kMostSlices], sums[PARTS][D];
    __shared__ float2 state;
    const long sh = blockIdx.x;
    const int sq = sh / p.Hq, h = sh - (long)sq * p.Hq;
    const Slice slice = find_slice(p, plan, sizes, -1 - sq);
    const int nsplit = slice.count;
    if (nsplit == 1) return;
    const int c2 = threadIdx.x % (D / 2), which = threadIdx.x / (D / 2);
    const float *r = part + ((long)slice.before * p.Hq + h * nsplit) * PF;
    float2 o[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int k = which + n * PARTS;
        o[n] = k < nsplit ? *reinterpret_cast<const float2 *>(r + k * PF + 2 + 2 * c2) : float2{0.f, 0.f};
    }
    if (threadIdx.x < 64) {
        const int k = threadIdx.x;
        const float2 ml = k < nsplit ? *reinterpret_cast<const float2 *>(r + k * PF) : float2{-INFINITY, 0.f};
        float M = groups_max(ml.x);  // over lanes 16, 32, 8, 4, 2 and 1 apart
        M = fmaxf(M, dpp_of<0x128>(M)), M = fmaxf(M, dpp_of<0x124>(M)), M = fmaxf(M, dpp_of<0x4E>(M)), M = fmaxf(M, dpp_of<0xB1>(M));
        const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        float sum = groups_sum(w * ml.y);
        sum += dpp_of<0x128>(sum), sum += dpp_of<0x124>(sum), sum += dpp_of<0x4E>(sum), sum += dpp_of<0xB1>(sum);
        weight[k] = w;
        if (k == 0) state = float2{M, sum};
    }
    __syncthreads();
    float o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const float w = weight[which + n * PARTS];
        o0 = fmaf(w, o[n].x, o0), o1 = fmaf(w, o[n].y, o1);
    }
    sums[which][2 * c2] = o0, sums[which][2 * c2 + 1] = o1;
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= D) return;
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) total += sums[i][c];
    finish<T>(1, state.x, state.y, total, out + sh * D + c, lse && c == 0 ? lse + sh : nullptr);  // (without entries there is one slice)
}

}  // namespace

size_t decode_fp4_workspace(const sepkv_params &p) {
    return words_bytes((long)p.S * p.Hkv * mx_chunks(p)) + align_up(mx_records(p, mx_shape(p, compute_units())) * (p.d + 2) * sizeof(float), 256);
}

int launch_decode_fp4(const sepkv_params &p, const void *q, const Fp4Cache &cache, const int32_t *sizes, const float *rope, int n_pos, void *out,
                      float *lse, void *ws, hipStream_t st) {
    const int G = p.Hq / p.Hkv, chunks = mx_chunks(p);
    const MxShape shape = mx_shape(p, compute_units());
    const bool add = shape.add && !being_captured(st);  // else a merge launch adds the slices
    const uint64_t one = add ? launch_number() : 0;
    auto go = [&](auto T_, auto D_, auto ROPE_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        auto launch = [&](auto ADD_) {
            ProfScope prof(SEPATTN_K_DECODE_SPLIT, st);
            hipLaunchKernelGGL((decode_fp4_kernel<T, D, decltype(ROPE_)::value, decltype(ADD_)::value>), dim3(p.Hkv * chunks, shape.slices),
                               dim3(64 * kWaves), 0, st, p, shape.plan, G, n_pos, static_cast<const T *>(q), cache, sizes, rope, one, static_cast<char *>(ws),
                               static_cast<T *>(out), lse);
        };
        add ? launch(std::true_type{}) : launch(std::false_type{});
        if (shape.plan.most == 1 || add) return launch_status();
        if (hipGetLastError() != hipSuccess) return (int)SEPATTN_ERR_HIP;
        ProfScope prof(SEPATTN_K_DECODE_MERGE, st);
        hipLaunchKernelGGL((merge_fp4_kernel<T, D>), dim3(p.S * p.Hq), dim3(256), 0, st, p, shape.plan, sizes,
                           reinterpret_cast<const float *>(static_cast<char *>(ws) + words_bytes((long)p.S * p.Hkv * chunks)), static_cast<T *>(out), lse);
        return launch_status();
    };
    auto with = [&](auto T_, auto D_) { return rope ? go(T_, D_, std::true_type{}) : go(T_, D_, std::false_type{}); };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (p.dtype == SEPATTN_BF16) return p.d == 64 ? with(uint16_t{}, D64{}) : with(uint16_t{}, D128{});
    return p.d == 64 ? with(float{}, D64{}) : with(float{}, D128{});
}

}  // namespace sepattn
