// Single-query attention behind shared prompts (Sec. 3.2 "Generation", Sec. 3.3): every sequence attends to the entries of the
// prefix cache that it shares with others and to those of its own cache.
//
// Softmax over the two sets is softmax over each, joined by maximum and sum, so the work is cut into
//   - the prefixes: all query heads of all sequences of a prefix that read one KV head are the rows of ONE product with its
//     keys and values, which are read once for all of them (per chunk of rows) and not once per sequence;
//   - the own caches, as sepattn_decode does (one slice of a cache per workgroup), in the same launch;
//   - the sum of the slices' records (maximum, sum, unnormalised output), in a second launch.
// What it cannot do without is to read every cache once, and 4 d operations per (query head, entry): with R rows on a KV head an entry's 4 d
// bytes feed 4 d R operations, so that from about 260 rows on the matrix units would bound it, below that the memory.
// Measured, 32/8 heads, d = 128, bf16, microseconds of the first launch + the second (bytes of the caches at the rate of a large copy):
//   2 sequences behind 600 entries                                   6.7 + 3.4 (1.2; launches and round trips)
//   32 sequences behind 8192 entries, 128 rows per KV head, turned  27 + 4.8 (18.7; 3.0 TB/s over both)
//   48 sequences behind 65536 entries, 192 rows per KV head          84 to 89 + 7.0 (72; 3.9 TB/s, 570 TFLOP/s)
// (In one launch, the last slice of a row adding its records: 12.8 for the first, in two 9.5 a call; four round trips past the L2 in sequence.)
#include "common.h"
#include "decode_common.h"
#include "decode_shared.h"
#include "mfma_common.h"

#include <algorithm>

namespace sepattn {

namespace {

constexpr int kShThreads = 256, kShWaves = 4;  // of the fp32 kernel and of the sum

// records of the prefixes' slices, [sequence][head][slice]: max (log2 domain), sum, 2 unused, D unnormalised outputs
template <int D>
constexpr int kShRecord = D + 4;

struct PrefixArgs {
    sepkv_params p, pp;
    int gq, nsplit;  // query heads per KV head, slices
    const void *q, *Kp, *Vp;
    const int32_t *sizes, *prefix_sizes, *group_start, *group_seq;
    const float *rope;
    int n_pos;
    float *part;
};

// A chunk of ROWS rows of one prefix; chunks are numbered over all prefixes.
struct Chunk {
    int prefix, row0, rows, first;  // first row of the chunk; rows of the prefix and its first entry in group_seq
};
template <int ROWS>
__device__ inline bool find_chunk(const PrefixArgs &x, int chunk, Chunk &c) {
    const int lane = threadIdx.x % kWave, G = x.pp.S;
    for (int g0 = 0; g0 < G; g0 += kWave) {
        const int g = min(g0 + lane, G - 1);
        const int s0 = min(max(x.group_start[g], 0), x.p.S), s1 = min(max(x.group_start[g + 1], s0), x.p.S);
        const int rows = (s1 - s0) * x.gq, n = g0 + lane < G ? (rows + ROWS - 1) / ROWS : 0;
        int upto = n;
#pragma unroll
        for (int o = 1; o < kWave; o *= 2) {
            const int other = __shfl_up(upto, o);
            if (lane >= o) upto += other;
        }
        const uint64_t beyond = __ballot(upto > chunk);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            c.prefix = __builtin_amdgcn_readfirstlane(g0 + at);
            c.row0 = __builtin_amdgcn_readfirstlane((chunk - __shfl(upto - n, at)) * ROWS);
            c.rows = __builtin_amdgcn_readfirstlane(__shfl(rows, at));
            c.first = __builtin_amdgcn_readfirstlane(__shfl(s0, at));
            return true;
        }
        chunk -= __builtin_amdgcn_readfirstlane(__shfl(upto, kWave - 1));
    }
    return false;
}

// entries [e0, e1) of a slice; false if it has none
__device__ inline bool slice_of(int entries, int nsplit, int split, int &e0, int &e1) {
    const int nb = (entries + kShBlock - 1) / kShBlock, per = (nb + nsplit - 1) / nsplit * kShBlock;
    e0 = __builtin_amdgcn_readfirstlane(min(split * per, entries));
    e1 = __builtin_amdgcn_readfirstlane(min(entries, e0 + per));
    return e0 < e1;
}
// the record of a slice without an entry: its outputs are not looked at
__device__ inline void mark_empty(float *record) { *reinterpret_cast<float2 *>(record) = float2{-INFINITY, 0.f}; }
// the map of one cache, which is the same in every lane, in scalar registers
__device__ inline CacheMap uniform_map(const sepkv_params &p, const int32_t *__restrict__ sizes, long cache) {
    CacheMap m = cache_map(p, sizes + SEPKV_SIZES_COLS * cache);
    for (int *x : {&m.n_init, &m.n_sep, &m.n_past, &m.n_loc, &m.sep_head, &m.win_head}) *x = __builtin_amdgcn_readfirstlane(*x);
    return m;
}
__device__ inline int entries_of(const CacheMap &m) { return m.n_init + m.n_sep + m.n_past + m.n_loc; }

// (sequence, head within the KV head's) of a row; rows past the last one repeat it
__device__ inline void row_of(const PrefixArgs &x, const Chunk &c, int r, int &seq, int &head) {
    r = min(r, c.rows - 1);
    const int member = r / x.gq;
    head = r - member * x.gq;
    seq = min(max(x.group_seq[c.first + member], 0), x.p.S - 1);
}
// position of a sequence's query: behind the prefix's entries and its own
__device__ inline int query_position(const PrefixArgs &x, int seq, int prefix_entries) {
    return min(max(prefix_entries + entries_of(cache_map(x.p, x.sizes + SEPKV_SIZES_COLS * seq)) - 1, 0), x.n_pos - 1);
}

// What a workgroup has to do.  Workgroups 0 .. n_prefix_groups - 1: (KV head, chunk of rows, slice of the prefix); the others: (KV head, sequence and
// chunk of 16 heads, slice of its own cache).  KV heads run fastest, so that with eight of them the workgroups that read the same rows are on
// one XCD.
struct SharedArgs {
    PrefixArgs x;
    const void *Kc, *Vc;
    float *own_part;
    int n_prefix_groups, chunks, n_own, head_chunks;
};
template <typename T>
struct SliceWork {
    CacheMap cm;
    int entries, e0, e1;  // of the cache, of the slice
    int kv, split;
    Chunk c;              // a prefix's
    int seq, head0;       // an own cache's: first head of the chunk, within the KV head's
    const T *K, *V;
};
// One row of the product: its query, the query's position (turned queries), where the slice's record goes (nullptr for a column without a row)
template <typename T>
struct SliceRow {
    const T *q;
    int position;
    float *record;
};
template <int D, bool ROPE, typename T>
__device__ __forceinline__ SliceRow<T> prefix_row(const SharedArgs &a, const SliceWork<T> &w, int block, int col) {
    const PrefixArgs &x = a.x;
    const int r = w.c.row0 + block * 16 + col;
    int seq, head;
    row_of(x, w.c, r, seq, head);
    const long row = (long)seq * x.p.Hq + w.kv * x.gq + head;
    return {static_cast<const T *>(x.q) + row * D, ROPE ? query_position(x, seq, w.entries) : 0,
            r < w.c.rows ? x.part + (row * x.nsplit + w.split) * kShRecord<D> : nullptr};
}
template <int D, typename T>
__device__ __forceinline__ SliceRow<T> own_row(const SharedArgs &a, const SliceWork<T> &w, int col) {
    const PrefixArgs &x = a.x;
    const int head = w.head0 + col;
    const long row = (long)w.seq * x.p.Hq + w.kv * x.gq + min(head, x.gq - 1);
    return {static_cast<const T *>(x.q) + row * D, 0, head < x.gq ? a.own_part + (row * a.n_own + w.split) * kShRecord<D> : nullptr};
}
// false: nothing to do (a slice without an entry has been marked as such)
template <int D, int ROWS, bool ROPE, typename T>
__device__ __forceinline__ bool prefix_work(const SharedArgs &a, int id, SliceWork<T> &w) {
    const PrefixArgs &x = a.x;
    const int Hkv = x.p.Hkv, chunk = id / Hkv % a.chunks;
    w.kv = id % Hkv, w.split = id / Hkv / a.chunks;
    if (!find_chunk<ROWS>(x, chunk, w.c)) return false;
    w.cm = uniform_map(x.pp, x.prefix_sizes, w.c.prefix);
    w.entries = entries_of(w.cm);
    if (!slice_of(w.entries, x.nsplit, w.split, w.e0, w.e1)) {
        if (threadIdx.x < ROWS)
            if (float *r = prefix_row<D, false>(a, w, threadIdx.x / 16, threadIdx.x % 16).record) mark_empty(r);
        return false;
    }
    const long head0 = ((long)w.c.prefix * Hkv + w.kv) * (long)x.pp.c * D;
    w.K = static_cast<const T *>(x.Kp) + head0, w.V = static_cast<const T *>(x.Vp) + head0;
    return true;
}
template <int D, typename T>
__device__ __forceinline__ bool own_work(const SharedArgs &a, int id, SliceWork<T> &w) {
    const PrefixArgs &x = a.x;
    const int Hkv = x.p.Hkv;
    w.kv = id % Hkv, w.head0 = id / Hkv % a.head_chunks * 16, w.seq = id / Hkv / a.head_chunks % x.p.S, w.split = id / Hkv / a.head_chunks / x.p.S;
    w.cm = uniform_map(x.p, x.sizes, w.seq);
    w.entries = entries_of(w.cm);
    if (!slice_of(w.entries, a.n_own, w.split, w.e0, w.e1)) {
        if (threadIdx.x < 16)
            if (float *r = own_row<D>(a, w, threadIdx.x).record) mark_empty(r);
        return false;
    }
    const long head0 = ((long)w.seq * Hkv + w.kv) * (long)x.p.c * D;
    w.K = static_cast<const T *>(a.Kc) + head0, w.V = static_cast<const T *>(a.Vc) + head0;
    return true;
}
// What to subtract in the exponent for a maximum: a row none of whose scores is above minus infinity has weights 0, not NaN.
__device__ inline float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// The states of NW waves that had the same 16 rows, [wave][row][record] in LDS, added in wave order and written; two columns per thread.
template <int D, int NW, typename Rows>
__device__ __forceinline__ void add_wave_states(const float *states, const Rows &rows, int block) {
    constexpr int REC = kShRecord<D>;
    for (int item = threadIdx.x; item < 16 * (D / 2); item += 64 * NW) {
        const int row = item / (D / 2), c2 = item % (D / 2);
        float *const to = rows(block, row).record;
        if (!to) continue;
        float M = -INFINITY, lsum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, states[(w * 16 + row) * REC]);
        const float base = base_of(M);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float *x = states + (w * 16 + row) * REC;
            const float wgt = __builtin_amdgcn_exp2f(x[0] - base);
            lsum = fmaf(wgt, x[1], lsum);
            o0 = fmaf(wgt, x[4 + 2 * c2], o0);
            o1 = fmaf(wgt, x[5 + 2 * c2], o1);
        }
        *reinterpret_cast<float2 *>(to + 4 + 2 * c2) = float2{o0, o1};
        if (c2 == 0) *reinterpret_cast<float2 *>(to) = float2{M, lsum};
    }
}

// ---- bf16 ------------------------------------------------------------------------------------------
// NW waves: rows (queries that read one KV head) against a slice of one cache, in blocks of 32 keys.  Operands as in
// decode_wide.hip (v_mfma_f32_16x16x32_bf16, the cache rows as A, 16 queries as the columns of B, score tile t's row 4g+i the block's row
// 8g+4t+i, so that a lane's probabilities are its operand of the second product); a wave has NB such column blocks, for which it
// reads the cache's fragments from LDS once.
//   SPLIT_ROWS: four waves have different rows (64 NB per workgroup) and share a ring of four stages of 32 rows of K and V: three tiles are
//     on their way, one barrier per tile.  NW = 8: two such groups, which take the slice's blocks in turn, so that a SIMD has two waves of one
//     workgroup and the slices, with their records, are half as many as with two workgroups of four per compute unit.
//   otherwise: the waves have the same 16 NB rows and take the blocks in turn, each with a stage of its own, whose K half is refilled
//     as soon as its fragments are in registers and the V half one step later; no barrier in the loop.
// The groups' or waves' states meet in LDS.
// Weights.  Their sum is formed in fp32 from the weights as they are.  For the second product they are the sum of two bf16 numbers (15 bits or more) where the
// waves share their rows: the product of the second ones finds room there (2 sequences behind 600 entries 9.4 us, with one number 9.4; 32 rows, 8192
// entries 18.7 and 18.4, 32768 entries 32.2 and 32.0).  SPLIT_ROWS: one bf16 number, 2^-8 of it at most, as in the other bf16 kernels, since there the second
// product is paid for in full (128 rows, 8192 entries 28.1 and 27.0, turned 31.0 and 29.7; 192 rows, 65536 entries 104 and 85, turned 144 and 122).  The
// output's distance to 64 bits is 1.66e-3 of its size with two numbers (its own rounding) and 2.35e-3 with one.
// KROPE (own caches): keys are turned by their distance to the query, as in decode_wide.hip.  LO (prefixes): the query is turned by its
// position.  Either is then the sum of two bf16 numbers, 16 bits of mantissa, and the scores are two products: rounded to one
// number, lse would be off by 1e-3.
template <int D, int NW>
constexpr int kShLds = NW * 2 * kShBlock * D;  // elements: a stage of K and V per wave

__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// XOR permutation of the 16-byte chunks of row 8a + 4t + i: see decode_wide.hip
template <int D>
__device__ inline int sh_swz(int row) {
    const int i = row & 3, a = row >> 3;
    if (D == 128) return (i << 1) | ((a & 1) << 3) | (a >> 1);
    return (i & 2) | ((a & 1) << 2) | (a >> 1);
}
// over the four lane groups
__device__ inline float groups_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float groups_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
template <int N>
__device__ inline void wait_loads() {
    static_assert(N == 0 || N == 4 || N == 5 || N == 6 || N == 8 || N == 9 || N == 12, "");
    if constexpr (N == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (N == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    if constexpr (N == 5) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
    if constexpr (N == 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
    if constexpr (N == 12) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
    if constexpr (N == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    if constexpr (N == 9) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
}
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ inline void barrier() {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wint-to-pointer-cast"
__device__ inline f32x4 lds_read_f4(uint32_t addr) { return *(const f32x4 __attribute__((address_space(3))) *)addr; }
#pragma clang diagnostic pop

// decode_slot_of without branches
__device__ inline int slot_of(const CacheMap &m, int e) {
    const int k = e - m.n_init, u = k - m.n_sep;
    const int sep = m.sep_head + k, win = m.win_head + u;
    const int in_sep = m.a + (sep >= m.s ? sep - m.s : sep), in_win = m.a + m.s + (win >= m.wcap ? win - m.wcap : win);
    return k < 0 ? e : u < 0 ? in_sep : in_win;
}

// slot of entry e, and the first entry behind e that does not lie in the slots next to it
__device__ inline void run_of(const CacheMap &m, int e, int &slot, int &end) {
    slot = slot_of(m, e);
    const int k = e - m.n_init, u = k - m.n_sep;
    const int sep = min(m.n_sep, m.s - m.sep_head), win = min(m.n_past + m.n_loc, m.wcap - m.win_head);  // entries in front of the rings' wraps
    end = k < 0 ? m.n_init : u < 0 ? m.n_init + (k < sep ? sep : m.n_sep) : m.n_init + m.n_sep + (u < win ? win : m.n_past + m.n_loc);
}

// a bf16 number and what it leaves of the sum of the two
__device__ inline void split_hi_lo(const f32x8 &x, bf16x8 &hi, bf16x8 &lo) {
    hi = __builtin_convertvector(x, bf16x8);
    lo = __builtin_convertvector(x - __builtin_convertvector(hi, f32x8), bf16x8);
}

// Weights as the sum of two bf16 numbers.  The first is the last one below the weight, so that the second is positive as well and an infinite
// value times either has the same sign.
__device__ inline void split_weights(const f32x8 &p, bf16x8 &hi, bf16x8 &lo) {
    f32x8 rest;
    u32x4 first;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t below[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            below[j] = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * i + j]), 1u);
            rest[2 * i + j] = p[2 * i + j] - __uint_as_float(below[j] & 0xFFFF0000u);
        }
        first[i] = __builtin_amdgcn_perm(below[1], below[0], 0x07060302u);
    }
    hi = as_bf16x8(first);
    lo = __builtin_convertvector(rest, bf16x8);
}

// rows: SliceRow of (column block, column)
template <int D, int NW, int NB, bool SPLIT_ROWS, bool KROPE, bool LO, typename Rows>
__device__ __forceinline__ void shared_body(const CacheMap &cm, const uint16_t *__restrict__ Kh, const uint16_t *__restrict__ Vh, int e0, int e1,
                                            int last /* KROPE: position of the query within the cache */, const float *__restrict__ rope,
                                            int n_pos, float sl2, uint16_t (&smem)[kShLds<D, NW>], float (&base_s)[NW][2][128], const Rows &rows) {
    static_assert(!KROPE || (NB == 1 && !SPLIT_ROWS && !LO), "");
    constexpr int CH = D / 8, RPL = 64 / CH;                         // 16-byte chunks per row, rows per wave-wide load
    constexpr int RW = 4, KG = NW / RW;                       // SPLIT_ROWS: waves per group, groups
    constexpr int NLD = kShBlock / RPL / (SPLIT_ROWS ? RW : 1);  // a wave's loads per block and tensor
    constexpr int KSTEPS = D / 32, KS2 = KSTEPS / 2, DB = D / 16, TILE = kShBlock * D;
    constexpr int STAGES = 4;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, g = lane >> 4, rw = wave % RW, kg = wave / RW;

    // queries; a turned one in two parts
    bf16x8 qhi[NB][KSTEPS], qlo[LO ? NB : 1][LO ? KSTEPS : 1];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const SliceRow<uint16_t> r = rows(SPLIT_ROWS ? rw * NB + nb : nb, col);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) qhi[nb][ks] = as_bf16x8(*reinterpret_cast<const u32x4 *>(r.q + 32 * ks + 8 * g));
        if constexpr (LO) {
            const float *row = rope + (long)r.position * D + 8 * g;
#pragma unroll
            for (int ks = 0; ks < KS2; ++ks) {
                const f32x8 u = __builtin_convertvector(qhi[nb][ks], f32x8), v = __builtin_convertvector(qhi[nb][ks + KS2], f32x8);
                f32x8 x, y;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 cs = *reinterpret_cast<const f32x4 *>(row + 32 * ks + 4 * h), sn = *reinterpret_cast<const f32x4 *>(row + D / 2 + 32 * ks + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[4 * h + e] = fmaf(u[4 * h + e], cs[e], -(v[4 * h + e] * sn[e]));
                        y[4 * h + e] = fmaf(v[4 * h + e], cs[e], u[4 * h + e] * sn[e]);
                    }
                }
                split_hi_lo(x, qhi[nb][ks], qlo[nb][ks]);
                split_hi_lo(y, qhi[nb][ks + KS2], qlo[nb][ks + KS2]);
            }
        }
    }

    // The queries have arrived: without this the compiler waits for them, and with them for every row on its way, in each round of the loop.
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) asm volatile("" : "+v"(qhi[nb][ks]));

    // loads: the wave's share of block eb's K or V rows into a stage; entries past the end: the last one (masked)
    const int my_pc = lane % CH, my_sub = lane / CH;
    const uint32_t lds0 = lds_addr(&smem[0]);
    const int stage_row0 = SPLIT_ROWS ? rw * (kShBlock / RW) : 0;  // first of the rows that this wave loads
    // Where a block's rows lie: nearly always in one run of slots, whose lanes' offsets never change; else a slot per row.
    uint32_t run_off[NLD];
#pragma unroll
    for (int u = 0; u < NLD; ++u) {
        const int r = stage_row0 + u * RPL + my_sub;
        run_off[u] = (uint32_t)(r * D * 2) + (uint32_t)((my_pc ^ sh_swz<D>(r)) * 16);
    }
    struct Place {
        int first;          // slot that the offsets count from
        uint32_t off[NLD];
    };
    int run_slot = 0, run_e = 0, run_end = 0;  // entry run_e lies in run_slot, those from there to run_end behind it
    auto place = [&](int eb) __attribute__((always_inline)) {
        Place at;
        if (eb + kShBlock <= run_end) {
            at.first = run_slot + (eb - run_e);
#pragma unroll
            for (int u = 0; u < NLD; ++u) at.off[u] = run_off[u];
        } else {
            at.first = 0;
#pragma unroll
            for (int u = 0; u < NLD; ++u) {
                const int r = stage_row0 + u * RPL + my_sub;
                at.off[u] = (uint32_t)slot_of(cm, min(eb + r, e1 - 1)) * (uint32_t)(D * 2) + (uint32_t)((my_pc ^ sh_swz<D>(r)) * 16);
            }
            run_e = min(eb + kShBlock, e1);
            run_of(cm, run_e, run_slot, run_end);
            run_end = min(run_end, e1);
        }
        return at;
    };
    auto load_rows = [&](const uint16_t *from, const Place &at, uint32_t stage) __attribute__((always_inline)) {
        from += (long)__builtin_amdgcn_readfirstlane(at.first) * D;
        static_for<NLD>([&](auto U) {
            const uint32_t to = stage + (stage_row0 + U * RPL) * D * 2;
            if constexpr (SPLIT_ROWS) dma_to_lds_16(from, at.off[U], to);  // the other chunks of rows read them as well
            else dma_to_lds_16_nt(from, at.off[U], to);
        });
    };
    auto k_stage = [&](int i) { return lds0 + (uint32_t)(i * 2 * TILE * 2); };
    auto v_stage = [&](int i) { return lds0 + (uint32_t)((i * 2 + 1) * TILE * 2); };

    f32x4 oacc[NB][DB];
    float m_run[NB], l_run[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m_run[nb] = -INFINITY, l_run[nb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // this lane's fragments in a stage: K row 8 (col/4) + col%4 (+ 4t), chunk 4 ks + g; V rows 8g + col/4 (+ 4), columns 16 db + 4 (col%4)
    const int krow = 8 * (col >> 2) + (col & 3), vrow = 8 * g + (col >> 2);
    const uint32_t kswz = sh_swz<D>(krow), vswz = sh_swz<D>(vrow);
    const uint32_t koff = krow * D * 2, voff = vrow * D * 2 + ((col & 1) << 3);

    auto key_fragment = [&](uint32_t stage, int t, int ks) __attribute__((always_inline)) {
        return lds_read_b128_at(stage + koff + 4 * t * D * 2 + (((uint32_t)(4 * ks + g) ^ kswz) << 4));
    };
    auto value_fragment = [&](uint32_t stage, int db) __attribute__((always_inline)) {
        return lds_read_tr_at(stage + voff + (((uint32_t)(2 * db + ((col & 3) >> 1)) ^ vswz) << 4), 4 * D * 2);
    };
    // Scores of column block nb -> its probabilities against the maximum so far.  That one is raised only where a lane's probabilities sum to
    // more than 2^8 (or there is none yet): a sum in fp32 and a product of bf16 numbers are as exact with a factor, and looking for every
    // block's maximum is a third of the vector instructions.  Entries past the slice's end: minus infinity.
    constexpr float kMost = 256.f;
    auto exponentials = [&](const f32x4 (&s)[2], int nb, f32x8 &p) __attribute__((always_inline)) {
        float psum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], sl2, -m_run[nb]));
            psum += p[i];
        }
        return psum;
    };
    auto mask_tail = [&](f32x4 (&s)[2], int n_valid) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = 8 * g + i < n_valid ? s[i >> 2][i & 3] : -INFINITY;
    };
    // Rows past the end repeat the last entry's: its weight there is 0, but an infinite value times 0 would be NaN, so their values count as zeros:
    // fragments, or, in front of them, the stage's rows (every wave that reads it clears them before its own reads)
    auto clear_tail = [&](bf16x8 (&va)[DB], int n_valid) __attribute__((always_inline)) {
        u32x4 keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = (8 * g + 2 * i < n_valid ? 0xFFFFu : 0u) | (8 * g + 2 * i + 1 < n_valid ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int db = 0; db < DB; ++db) va[db] = as_bf16x8(__builtin_bit_cast(u32x4, va[db]) & keep);
    };
    auto clear_rows = [&](uint32_t stage, int n_valid) __attribute__((always_inline)) {
#pragma unroll 1
        for (int chunk = n_valid * CH + lane; chunk < kShBlock * CH; chunk += 64) lds_write_b128_at(stage + chunk * 16, f32x4{0.f, 0.f, 0.f, 0.f});
        wait_lds();
    };
    auto raise = [&](const f32x4 (&s)[2], int nb, f32x8 &p) __attribute__((always_inline)) {
        float m = s[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) m = fmaxf(m, s[i >> 2][i & 3]);
        m = fmaxf(m_run[nb], groups_max(m) * sl2);
        const float base = base_of(m), alpha = __builtin_amdgcn_exp2f(m_run[nb] - base);
        m_run[nb] = base;
        l_run[nb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[nb][db] *= alpha;
        const float psum = exponentials(s, nb, p), all = groups_sum(psum);
        if (m == -INFINITY && all == all) m_run[nb] = m;  // no score above minus infinity; if they were NaN the sums are now, and the record counts
        return psum;
    };

    if constexpr (SPLIT_ROWS) {
        const int blocks = ((e1 - e0 + kShBlock - 1) / kShBlock + KG - 1) / KG;  // of a group
        const int stage0 = kg * STAGES;
        // Where the registers allow it, a wave reads a tile's K fragments one tile ahead and its V fragments in front of the exponentials, so
        // that neither is waited for; K then runs one tile ahead of V through the ring.  (Blocks past the end are loaded as
        // well, the last row over and over: the number of loads on their way stays the same.)
        constexpr bool AHEAD = D == 64 || NB * (LO ? 2 : 1) <= 2, EARLY_V = D == 64 || NB <= 2;
        auto where = [&](int i) __attribute__((always_inline)) { return place(e0 + (i * KG + kg) * kShBlock); };
        auto request_k = [&](int i, const Place &at) __attribute__((always_inline)) { load_rows(Kh, at, k_stage(stage0 + i % STAGES)); };
        auto request_v = [&](int i, const Place &at) __attribute__((always_inline)) { load_rows(Vh, at, v_stage(stage0 + i % STAGES)); };
        bf16x8 ka[2][KSTEPS];
        auto read_keys = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) ka[t][ks] = key_fragment(k_stage(stage0 + i % STAGES), t, ks);
        };
        Place at = where(0);
        request_k(0, at);
        if constexpr (!AHEAD) request_v(0, at);
        for (int i = 1; i < STAGES - (AHEAD ? 0 : 1); ++i) {
            const Place next = where(i);
            request_k(i, next);
            request_v(AHEAD ? i - 1 : i, AHEAD ? at : next);
            at = next;
        }
        if constexpr (AHEAD) {
            wait_loads<2 * NLD *(STAGES - 1)>();
            barrier();
            read_keys(0);
        }
        for (int i = 0; i < blocks; ++i) {
            wait_loads<2 * NLD *(STAGES - 2)>();
            if constexpr (AHEAD) wait_lds();
            barrier();  // everyone's part of V tile i and of K tile i (AHEAD: i + 1) has landed, and everyone has read what lay where the next ones go
            const int n_valid = e1 - e0 - (i * KG + kg) * kShBlock;
            const uint32_t k_at = k_stage(stage0 + i % STAGES), v_at = v_stage(stage0 + i % STAGES);
            // (else two steps' fragments in front of their use, which the scheduling fences keep there)
            constexpr int EARLY = 2;
            auto read_step = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < 2; ++t) ka[t][ks] = key_fragment(k_at, t, ks);
            };
            if constexpr (!AHEAD) {
#pragma unroll
                for (int ks = 0; ks < EARLY; ++ks) read_step(ks);
                __builtin_amdgcn_sched_barrier(0);
            }
            {
                const Place next = where(i + STAGES - (AHEAD ? 0 : 1));
                request_k(i + STAGES - (AHEAD ? 0 : 1), next);
                request_v(i + STAGES - 1, AHEAD ? at : next);
                at = next;
            }
            if (n_valid > 0) {  // (the second group's last block may be past the end)
                f32x4 s[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                static_for<KSTEPS>([&](auto KS) __attribute__((always_inline)) {
                    constexpr int ks = KS;
                    if constexpr (!AHEAD && ks + EARLY < KSTEPS) {
                        read_step(ks + EARLY);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            s[nb][t] = mfma16(ka[t][ks], qhi[nb][ks], s[nb][t]);
                            if constexpr (LO) s[nb][t] = mfma16(ka[t][ks], qlo[nb][ks], s[nb][t]);
                        }
                });
                auto tail = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mask_tail(s[nb], n_valid);
                };
                if constexpr (!EARLY_V) {
                    if (n_valid < kShBlock) {
                        tail();
                        clear_rows(v_at, n_valid);
                    }
                }
                bf16x8 va[DB];
#pragma unroll
                for (int db = 0; db < (EARLY_V ? DB : EARLY); ++db) va[db] = value_fragment(v_at, db);
                if constexpr (AHEAD) read_keys(i + 1);
                if constexpr (!EARLY_V) __builtin_amdgcn_sched_barrier(0);
                if constexpr (EARLY_V) {
                    if (n_valid < kShBlock) {
                        tail();
                        clear_tail(va, n_valid);
                    }
                }
                f32x8 p[NB];
                float psum[NB];
                bool over = false;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    psum[nb] = exponentials(s[nb], nb, p[nb]);
                    over |= !(psum[nb] <= kMost);
                }
                if (__builtin_amdgcn_ballot_w64(over) != 0ull) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) psum[nb] = raise(s[nb], nb, p[nb]);
                }
                bf16x8 pb[NB];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    l_run[nb] += psum[nb];
                    pb[nb] = __builtin_convertvector(p[nb], bf16x8);
                }
                static_for<DB>([&](auto DBI) __attribute__((always_inline)) {
                    constexpr int db = DBI;
                    if constexpr (!EARLY_V && db + EARLY < DB) {
                        va[db + EARLY] = value_fragment(v_at, db + EARLY);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) oacc[nb][db] = mfma16(va[db], pb[nb], oacc[nb][db]);
                    if constexpr (!EARLY_V) __builtin_amdgcn_sched_barrier(0);
                });
            }
            if constexpr (!AHEAD) wait_lds();
        }
        wait_loads<0>();
        // ---- the second group's states meet the first's
        constexpr int REC = kShRecord<D>;
        static_assert(KG == 1 || KG == 2 && RW * NB * 16 * REC * sizeof(float) <= kShLds<D, NW> * sizeof(uint16_t), "");
        float *const red = reinterpret_cast<float *>(&smem[0]) + (rw * NB * 16 + col) * REC;
        if constexpr (KG > 1) __syncthreads();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            l_run[nb] = groups_sum(l_run[nb]);
            if (KG == 1 || kg == 0) continue;
            float *const r = red + nb * 16 * REC;
            if (g == 0) *reinterpret_cast<float2 *>(r) = float2{m_run[nb], l_run[nb]};
#pragma unroll
            for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(r + 4 + 16 * db + 4 * g) = oacc[nb][db];
        }
        if constexpr (KG > 1) {
            __syncthreads();
            if (kg > 0) return;
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float *const to = rows(rw * NB + nb, col).record;
            if (!to) continue;
            if constexpr (KG == 1) {
                if (g == 0) *reinterpret_cast<float2 *>(to) = float2{m_run[nb], l_run[nb]};
#pragma unroll
                for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(to + 4 + 16 * db + 4 * g) = oacc[nb][db];
                continue;
            }
            const float *r = red + nb * 16 * REC;
            const float2 ml = *reinterpret_cast<const float2 *>(r);
            const float M = fmaxf(m_run[nb], ml.x), base = base_of(M);
            const float mine = __builtin_amdgcn_exp2f(m_run[nb] - base), other = __builtin_amdgcn_exp2f(ml.x - base);
            if (g == 0) *reinterpret_cast<float2 *>(to) = float2{M, fmaf(other, ml.y, mine * l_run[nb])};
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const f32x4 o = *reinterpret_cast<const f32x4 *>(r + 4 + 16 * db + 4 * g);
                f32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = fmaf(other, o[i], mine * oacc[nb][db][i]);
                *reinterpret_cast<f32x4 *>(to + 4 + 16 * db + 4 * g) = v;
            }
        }
    } else {
        const uint32_t ks_ = k_stage(wave), vs_ = v_stage(wave), bs_ = lds_addr(&base_s[wave][0][0]), ts_ = lds0;
        Place at;
        auto request_keys = [&](int eb, int par) __attribute__((always_inline)) {
            at = place(eb);
            if constexpr (KROPE) {  // the table row of the first entry's distance
                if (lane < D / 4) dma_to_lds_16(rope + (long)min(last - eb, n_pos - 1) * D, lane * 16, bs_ + par * D * 4);
            }
            load_rows(Kh, at, ks_);
        };
        int eb = e0 + wave * kShBlock;
        const bool some = eb < e1;
        // cos / sin of the lane's two rows krow + 4t within a block: table rows 0 .. 31, through LDS, over the V stages of the first waves
        f32x4 rc[2][KS2][2], rs[2][KS2][2];
        if constexpr (KROPE) {
            constexpr int TCH = D / 4, TRPL = 64 / TCH, TLD = kShBlock / TRPL / NW;
            static_assert(TLD >= 1 && TLD * TRPL * NW == kShBlock, "");
            // (where row r goes: the V stages lie apart; half a stage holds 16 rows at either d)
            auto table_row = [&](int r) { return v_stage(r >> 4) + (uint32_t)((r & 15) * D * 4); };
            static_assert(16 * D * 4 <= 2 * TILE, "");
            static_for<TLD>([&](auto U) {
                const int r0 = (wave * TLD + U) * TRPL, r = r0 + lane / TCH;
                dma_to_lds_16(rope, (uint32_t)(min(r, n_pos - 1) * D * 4) + (uint32_t)(((lane % TCH) ^ sh_swz<128>(r)) * 16), table_row(r0));
            });
            if (some) {
                request_keys(eb, 0);
                wait_loads<NLD + 1>();
            } else {
                wait_loads<0>();
            }
            barrier();
            const uint32_t tswz = sh_swz<128>(krow);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ks = 0; ks < KS2; ++ks)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t row = table_row(krow + 4 * t);
                        rc[t][ks][h] = lds_read_f4(row + (((uint32_t)(8 * ks + 2 * g + h) ^ tswz) << 4));
                        rs[t][ks][h] = lds_read_f4(row + (((uint32_t)(D / 8 + 8 * ks + 2 * g + h) ^ tswz) << 4));
                    }
            wait_lds();
            barrier();
            if (some) load_rows(Vh, at, vs_);
        } else if (some) {
            request_keys(eb, 0);
            load_rows(Vh, at, vs_);
        }
        for (int par = 0; eb < e1; eb += NW * kShBlock, par ^= 1) {
            const bool more = eb + NW * kShBlock < e1;
            const int n_valid = e1 - eb;
            wait_loads<NLD>();  // the K rows; the V rows may be in flight
            bf16x8 ka[2][KSTEPS];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks) ka[t][ks] = key_fragment(ks_, t, ks);
            f32x4 bc[KS2][2], bs[KS2][2];
            if constexpr (KROPE) {
#pragma unroll
                for (int ks = 0; ks < KS2; ++ks)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bc[ks][h] = lds_read_f4(bs_ + par * D * 4 + (8 * ks + 2 * g + h) * 16);
                        bs[ks][h] = lds_read_f4(bs_ + par * D * 4 + (D / 8 + 8 * ks + 2 * g + h) * 16);
                    }
            }
            if (more) {
                wait_lds();
                request_keys(eb + NW * kShBlock, par ^ 1);
            }
            f32x4 s[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (KROPE) {
                // R(-distance): (x, y) -> (x cos + y sin, y cos - x sin), dimension i with i + D/2; row r's distance is that of the
                // block's first entry minus r
#pragma unroll
                for (int ks = 0; ks < KS2; ++ks)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const f32x8 x = __builtin_convertvector(ka[t][ks], f32x8), y = __builtin_convertvector(ka[t][ks + KS2], f32x8);
                        f32x8 u, v;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float c0 = bc[ks][e >> 2][e & 3], s0 = bs[ks][e >> 2][e & 3];
                            const float cr = rc[t][ks][e >> 2][e & 3], sr = rs[t][ks][e >> 2][e & 3];
                            const float c = fmaf(s0, sr, c0 * cr), sn = fmaf(-c0, sr, s0 * cr);
                            u[e] = fmaf(y[e], sn, x[e] * c);
                            v[e] = fmaf(-x[e], sn, y[e] * c);
                        }
                        bf16x8 lo;
                        split_hi_lo(u, ka[t][ks], lo);
                        s[0][t] = mfma16(lo, qhi[0][ks], s[0][t]);
                        split_hi_lo(v, ka[t][ks + KS2], lo);
                        s[0][t] = mfma16(lo, qhi[0][ks + KS2], s[0][t]);
                    }
            }
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        s[nb][t] = mfma16(ka[t][ks], qhi[nb][ks], s[nb][t]);
                        if constexpr (LO) s[nb][t] = mfma16(ka[t][ks], qlo[nb][ks], s[nb][t]);
                    }
            if (more) wait_loads<NLD + (KROPE ? 1 : 0)>();  // the V rows (only the next block's K rows are in flight)
            else wait_loads<0>();
            bf16x8 va[DB];
#pragma unroll
            for (int db = 0; db < DB; ++db) va[db] = value_fragment(vs_, db);
            if (more) {
                wait_lds();
                load_rows(Vh, at, vs_);
            }
            if (n_valid < kShBlock) {
                clear_tail(va, n_valid);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mask_tail(s[nb], n_valid);
            }
            bf16x8 pb[NB], pl[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                f32x8 p;
                float psum = exponentials(s[nb], nb, p);
                if (__builtin_amdgcn_ballot_w64(!(psum <= kMost)) != 0ull) psum = raise(s[nb], nb, p);
                l_run[nb] += psum;
                split_weights(p, pb[nb], pl[nb]);
            }
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) oacc[nb][db] = mfma16(va[db], pb[nb], oacc[nb][db]);
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) oacc[nb][db] = mfma16(va[db], pl[nb], oacc[nb][db]);
        }
        // ---- the waves' states meet in LDS, one column block after the other; a thread adds two columns of a row
        constexpr int REC = kShRecord<D>;
        static_assert(NW * 16 * REC * sizeof(float) <= kShLds<D, NW> * sizeof(uint16_t), "");
        float *red = reinterpret_cast<float *>(&smem[0]);  // [wave][row][REC]
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float l = groups_sum(l_run[nb]);
            __syncthreads();
            float *r = red + (wave * 16 + col) * REC;
            if (g == 0) *reinterpret_cast<float2 *>(r) = float2{m_run[nb], l};
#pragma unroll
            for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(r + 4 + 16 * db + 4 * g) = oacc[nb][db];
            __syncthreads();
            add_wave_states<D, NW>(red, rows, nb);
        }
    }
}

template <int D, int NW, int NB, bool SPLIT_ROWS, bool ROPE>
__global__ __launch_bounds__(64 * NW, 8 / NW) void shared_decode_kernel(SharedArgs a) {
    __shared__ __attribute__((aligned(1024))) uint16_t smem[kShLds<D, NW>];
    __shared__ __attribute__((aligned(1024))) float base_s[NW][2][128];
    const PrefixArgs &x = a.x;
    const float sl2 = x.p.scale * kLog2e_f;
    SliceWork<uint16_t> w;
    if ((int)blockIdx.x < a.n_prefix_groups) {
        if (!prefix_work<D, (SPLIT_ROWS ? 4 : 1) * 16 * NB, ROPE>(a, blockIdx.x, w)) return;
        shared_body<D, NW, NB, SPLIT_ROWS, false, ROPE>(w.cm, w.K, w.V, w.e0, w.e1, 0, x.rope, x.n_pos, sl2, smem, base_s,
                                                        [&](int block, int col) { return prefix_row<D, ROPE>(a, w, block, col); });
    } else {
        if (!own_work<D>(a, blockIdx.x - a.n_prefix_groups, w)) return;
        shared_body<D, NW, 1, false, ROPE, false>(w.cm, w.K, w.V, w.e0, w.e1, w.entries - 1, x.rope, x.n_pos, sl2, smem, base_s,
                                                  [&](int, int col) { return own_row<D>(a, w, col); });
    }
}

// ---- fp32 ------------------------------------------------------------------------------------------
// The same division into prefixes and own caches with fp32 operands, v_mfma_f32_16x16x4_f32.  Four waves, tiles of 64 keys in LDS; the next tile's
// rows are on their way in registers meanwhile.  SPLIT_ROWS: each wave has 16 rows of its own and takes every key; otherwise all
// have the same 16 rows and a quarter of the tile's keys each, and their states meet in LDS.
// Lane l, group g = l / 16.  Scores: A = K, row l%16 = key, B = queries, column l%16; the four k-slots of step 4 S + i are dimensions 16 S + 4 g + i,
// so that a lane's operands are pieces of 16 bytes.  C: column l%16 = query, rows 4 g + i = keys.  Output: O^T += V^T P^T, the k-slots
// of step i are keys 4 g + i, which the lane group holds.
// KROPE (own caches): a key is turned by its distance to the query on its way into LDS, by the thread that holds both of a pair.
// The fp32 matrix rate is a sixteenth of bf16's, and this type is there to check a bf16 run against: 11 sequences of up to 150 entries behind three prefixes
// of up to 250 (12/12 heads, d = 64, turned) take 9.2 us and 3.2 for the sum, most of it launches and round trips (bytes: 2.2).
// Where there is more to read it stays far from the memory's rate: 41 sequences of 32/8 heads, d = 64, behind 2209 entries 34 us (17), 8 of d = 128 behind 8192
// 41 (19): tiles through registers, two barriers per 64 keys, V from LDS four bytes at a time.
typedef float f4 __attribute__((ext_vector_type(4)));
constexpr int kFpKeys = 64;
template <int D>
constexpr int kFpPitch = D + 4;  // floats per row in LDS

template <int D, bool SPLIT_ROWS, bool KROPE, bool LO, typename Rows>
__device__ __forceinline__ void shared_fp32_body(const CacheMap &cm, const float *__restrict__ Kh, const float *__restrict__ Vh, int e0, int e1, int last,
                                                 const float *__restrict__ rope, int n_pos, float sl2, float (&smem)[2 * kFpKeys * kFpPitch<D>],
                                                 const Rows &rows) {
    constexpr int PITCH = kFpPitch<D>, REC = kShRecord<D>, ITEMS = kFpKeys * (D / 8) / kShThreads;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane & 15, g = lane >> 4;
    float *const ks = smem, *const vs = smem + kFpKeys * PITCH;
    f4 q[D / 16];
    {
        const auto r = rows(SPLIT_ROWS ? wave : 0, col);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q[s] = *reinterpret_cast<const f4 *>(r.q + 16 * s + 4 * g);
        if constexpr (LO) {
            const float *row = rope + (long)r.position * D + 4 * g;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const f4 cs = *reinterpret_cast<const f4 *>(row + 16 * s), sn = *reinterpret_cast<const f4 *>(row + D / 2 + 16 * s);
                const f4 u = q[s], v = q[s + D / 32];
                q[s] = u * cs - v * sn;
                q[s + D / 32] = v * cs + u * sn;
            }
        }
    }
    // a thread's pieces of a tile: columns pc .. pc + 3 and their partners D/2 on
    f4 kr[ITEMS][2], vr[ITEMS][2], cs[KROPE ? ITEMS : 1], sn[KROPE ? ITEMS : 1];
    auto fetch = [&](int eb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = threadIdx.x + i * kShThreads, pc = item % (D / 8) * 4, e = min(eb + item / (D / 8), e1 - 1);
            const long off = (long)slot_of(cm, e) * D + pc;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                kr[i][h] = *reinterpret_cast<const f4 *>(Kh + off + h * (D / 2));
                vr[i][h] = *reinterpret_cast<const f4 *>(Vh + off + h * (D / 2));
            }
            if constexpr (KROPE) {
                const float *row = rope + (long)min(last - e, n_pos - 1) * D + pc;
                cs[i] = *reinterpret_cast<const f4 *>(row);
                sn[i] = *reinterpret_cast<const f4 *>(row + D / 2);
            }
        }
    };
    auto stage = [&](int eb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = threadIdx.x + i * kShThreads, at = item / (D / 8) * PITCH + item % (D / 8) * 4;
            if (eb + item / (D / 8) >= e1) vr[i][0] = vr[i][1] = f4{0.f, 0.f, 0.f, 0.f};  // (0 times an infinity of the last entry, which is there, would be NaN)
            f4 x = kr[i][0], y = kr[i][1];
            if constexpr (KROPE) {  // R(-distance)
                x = kr[i][0] * cs[i] + kr[i][1] * sn[i];
                y = kr[i][1] * cs[i] - kr[i][0] * sn[i];
            }
            *reinterpret_cast<f4 *>(ks + at) = x;
            *reinterpret_cast<f4 *>(ks + at + D / 2) = y;
            *reinterpret_cast<f4 *>(vs + at) = vr[i][0];
            *reinterpret_cast<f4 *>(vs + at + D / 2) = vr[i][1];
        }
    };
    f4 o[D / 16];
#pragma unroll
    for (int db = 0; db < D / 16; ++db) o[db] = f4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    fetch(e0);
    for (int eb = e0; eb < e1; eb += kFpKeys) {
        __syncthreads();
        stage(eb);
        __syncthreads();
        if (eb + kFpKeys < e1) fetch(eb + kFpKeys);
#pragma unroll 1
        for (int blk = SPLIT_ROWS ? 0 : wave; blk < (SPLIT_ROWS ? kFpKeys / 16 : wave + 1); ++blk) {
            const int n_valid = e1 - eb - 16 * blk;
            if (n_valid <= 0) break;
            const float *const kb = ks + 16 * blk * PITCH, *const vb = vs + 16 * blk * PITCH;
            f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < D / 16; ++st) {
                const f4 k = *reinterpret_cast<const f4 *>(kb + col * PITCH + 16 * st + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[st][i], s, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = 4 * g + i < n_valid ? s[i] * sl2 : -INFINITY;
            const float m_new = fmaxf(m, groups_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
            const float base = base_of(m_new), alpha = exp2f(m - base);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] = exp2f(s[i] - base);
                sum += s[i];
            }
            m = m_new;
            if (m_new == -INFINITY) m = groups_sum(sum) == 0.f ? m_new : base;  // scores that are NaN: the sums are now, and the record counts
            l = l * alpha + sum;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                o[db] *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(vb[(4 * g + i) * PITCH + 16 * db + col], s[i], o[db], 0, 0, 0);
            }
        }
    }
    l = groups_sum(l);
    if constexpr (SPLIT_ROWS) {
        float *const to = rows(wave, col).record;
        if (!to) return;
        if (g == 0) *reinterpret_cast<float2 *>(to) = float2{m, l};
#pragma unroll
        for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f4 *>(to + 4 + 16 * db + 4 * g) = o[db];
    } else {
        static_assert(kShWaves * 16 * REC <= 2 * kFpKeys * PITCH, "the waves' states fit the tiles");
        __syncthreads();
        float *const r = smem + (wave * 16 + col) * REC;
        if (g == 0) *reinterpret_cast<float2 *>(r) = float2{m, l};
#pragma unroll
        for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f4 *>(r + 4 + 16 * db + 4 * g) = o[db];
        __syncthreads();
        add_wave_states<D, kShWaves>(smem, rows, 0);
    }
}

template <int D, bool SPLIT_ROWS, bool ROPE>
__global__ __launch_bounds__(kShThreads, 2) void shared_decode_fp32_kernel(SharedArgs a) {
    constexpr int ROWS = (SPLIT_ROWS ? kShWaves : 1) * 16;
    __shared__ __attribute__((aligned(16))) float smem[2 * kFpKeys * kFpPitch<D>];
    const PrefixArgs &x = a.x;
    const float sl2 = x.p.scale * kLog2e_f;
    SliceWork<float> w;
    if ((int)blockIdx.x < a.n_prefix_groups) {
        if (!prefix_work<D, ROWS, ROPE>(a, blockIdx.x, w)) return;
        shared_fp32_body<D, SPLIT_ROWS, false, ROPE>(w.cm, w.K, w.V, w.e0, w.e1, 0, x.rope, x.n_pos, sl2, smem, [&](int block, int col) { return prefix_row<D, ROPE>(a, w, block, col); });
    } else {
        if (!own_work<D>(a, blockIdx.x - a.n_prefix_groups, w)) return;
        shared_fp32_body<D, false, ROPE, false>(w.cm, w.K, w.V, w.e0, w.e1, w.entries - 1, x.rope, x.n_pos, sl2, smem, [&](int, int col) { return own_row<D>(a, w, col); });
    }
}

// ---- the slices' sum ------------------------------------------------------------------------------
// WPR waves per (sequence, head), prefix slices first, then the own cache's; wave w takes slices w, w + WPR, ... of both, eight records in one
// round trip, and the waves' sums are added in wave order.  Nothing but the records has to be read for that (a slice without an entry
// says so in its own; those of a prefix that the sequence does not have are skipped), so that the kernel is one round trip and its
// launch: 3.3 us for a few rows, 4.7 for 1024 rows of 14 records, 7.0 for 1536 rows of 28.
template <typename T, int D, int WPR>
__global__ __launch_bounds__(kShThreads) void shared_merge_kernel(sepkv_params p, int n_prefixes, int n_prefix, int n_own,
                                                                  const int32_t *__restrict__ prefix_of, const float *__restrict__ prefix_part,
                                                                  const float *__restrict__ own_part, T *__restrict__ out, float *__restrict__ lse) {
    constexpr int REC = kShRecord<D>, C = D / kWave, NR = 8;
    __shared__ float state[WPR][D + 2];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), w0 = WPR == 1 ? 0 : wave;
    const int head = WPR == 1 ? blockIdx.x * kShWaves + wave : blockIdx.x, seq = blockIdx.y;
    if (head >= p.Hq) return;
    const long row = (long)seq * p.Hq + head;
    const int of = prefix_of[seq];
    const int total = n_prefix + n_own;
    const float *pre = prefix_part + row * n_prefix * REC, *own = own_part + row * n_own * REC;
    float M = -INFINITY, l = 0.f, o[C] = {};
    for (int k0 = w0; k0 < total; k0 += WPR * NR) {
        float m[NR], ls[NR], os[NR][C];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int k = min(k0 + WPR * i, total - 1);  // past the last one: that again, with weight 0
            const float *r = k < n_prefix ? pre + k * REC : own + (k - n_prefix) * REC, *v = r + 4 + C * lane;
            const float2 ml = *reinterpret_cast<const float2 *>(r);
            m[i] = ml.x, ls[i] = ml.y;
#pragma unroll
            for (int j = 0; j < C; ++j) os[i][j] = v[j];
        }
        const bool shares = of >= 0 && of < n_prefixes;
        float Mn = M;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int k = k0 + WPR * i;
            if (k >= total || (k < n_prefix && !shares)) m[i] = -INFINITY;
            Mn = fmaxf(Mn, m[i]);
        }
        if (Mn == -INFINITY) continue;  // slices without an entry
        const float keep = exp2f(M - Mn);
        M = Mn;
        l *= keep;
#pragma unroll
        for (int j = 0; j < C; ++j) o[j] *= keep;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const bool used = m[i] != -INFINITY;  // (else the rest of the record is whatever the memory held)
            const float w = used ? exp2f(m[i] - M) : 0.f;
            l = fmaf(w, used ? ls[i] : 0.f, l);
#pragma unroll
            for (int j = 0; j < C; ++j) o[j] = fmaf(w, used ? os[i][j] : 0.f, o[j]);
        }
    }
    auto write = [&](int c, float v, float lsum) {
        v = lsum == 0.f ? 0.f : v / lsum;  // (NaN stays NaN)
        if constexpr (sizeof(T) == 2) out[row * D + c] = decode_f32_to_bf16(v);
        else out[row * D + c] = v;
        if (lse && c == 0) lse[row] = lsum == 0.f ? -INFINITY : (M + log2f(lsum)) * kLn2_f;
    };
    if constexpr (WPR == 1) {
#pragma unroll
        for (int j = 0; j < C; ++j) write(C * lane + j, o[j], l);
        return;
    }
    if (lane == 0) state[wave][D] = M, state[wave][D + 1] = l;
#pragma unroll
    for (int j = 0; j < C; ++j) state[wave][C * lane + j] = o[j];
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= D) return;
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < WPR; ++w) M = fmaxf(M, state[w][D]);
    float lsum = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < WPR; ++w) {
        const float wgt = state[w][D] == -INFINITY ? 0.f : exp2f(state[w][D] - M);
        lsum = fmaf(wgt, state[w][D + 1], lsum);
        v = fmaf(wgt, state[w][c], v);
    }
    write(c, v, lsum);
}

}  // namespace

size_t decode_shared_workspace(const sepkv_params &p, const sepkv_params &pp) {
    size_t most = 0;
    for (const bool rope : {false, true}) {  // one size for calls with and without positions
        const SharedShape s = shared_shape(p, pp, rope);
        most = std::max(most, prefix_record_bytes(p, s) + own_record_bytes(p, s));
    }
    return most;
}

int launch_decode_shared(const SharedDecode &x, hipStream_t st) {
    const SharedShape s = shared_shape(x.p, x.pp, x.rope != nullptr);
    float *const own_part = x.part + prefix_record_bytes(x.p, s) / sizeof(float);
    const int gq = x.p.Hq / x.p.Hkv;
    const PrefixArgs a = {x.p, x.pp, gq, s.n_prefix, x.q, x.Kp, x.Vp, x.sizes, x.prefix_sizes, x.group_start, x.group_seq,
                          x.rope, x.n_pos, x.part};
    const dim3 block(kShThreads);
    {
        const int head_chunks = (gq + 15) / 16;
        const long n_prefix_groups = (long)x.p.Hkv * s.chunks * s.n_prefix, n = n_prefix_groups + (long)x.p.Hkv * head_chunks * x.p.S * s.n_own;
        if (n > 0x7FFFFFFFL) return SEPATTN_ERR_SHAPE;
        const SharedArgs all = {a, x.Kc, x.Vc, own_part, (int)n_prefix_groups, s.chunks, s.n_own, head_chunks};
        ProfScope prof(SEPATTN_K_DECODE_SPLIT, st);
        auto fp32 = [&](auto D_, auto ROWS_) {
            constexpr int D = decltype(D_)::value;
            constexpr bool ROWS = decltype(ROWS_)::value != 0;
            if (x.rope) hipLaunchKernelGGL((shared_decode_fp32_kernel<D, ROWS, true>), dim3((unsigned)n), block, 0, st, all);
            else hipLaunchKernelGGL((shared_decode_fp32_kernel<D, ROWS, false>), dim3((unsigned)n), block, 0, st, all);
        };
        auto go = [&](auto D_, auto NW_, auto NB_, auto ROWS_, auto ROPE_) {
            constexpr int D = decltype(D_)::value, NW = decltype(NW_)::value, NB = decltype(NB_)::value;
            constexpr bool ROWS = decltype(ROWS_)::value != 0, ROPE = decltype(ROPE_)::value != 0;
            hipLaunchKernelGGL((shared_decode_kernel<D, NW, NB, ROWS, ROPE>), dim3((unsigned)n), dim3(64 * NW), 0, st, all);
        };
        using N1 = IntC<1>;
        using N2 = IntC<2>;
        using N3 = IntC<3>;
        using W4 = IntC<4>;
        using W8 = IntC<8>;
        auto shape = [&](auto D_, auto ROPE_) {
            constexpr int D = decltype(D_)::value;
            constexpr bool ROPE = decltype(ROPE_)::value != 0;
            if (!s.split_rows) return s.nb == 1 ? go(D_, W4{}, N1{}, IntC<0>{}, ROPE_) : go(D_, W4{}, N2{}, IntC<0>{}, ROPE_);
            if constexpr (D == 128 && !ROPE)
                if (s.waves == 8) return s.nb == 2 ? go(D_, W8{}, N2{}, N1{}, ROPE_) : go(D_, W8{}, N3{}, N1{}, ROPE_);
            if constexpr (D == 64 || !ROPE)
                if (s.nb == 3) return go(D_, W4{}, N3{}, N1{}, ROPE_);
            s.nb == 1 ? go(D_, W4{}, N1{}, N1{}, ROPE_) : go(D_, W4{}, N2{}, N1{}, ROPE_);
        };
        if (x.p.dtype == SEPATTN_FP32) {
            if (x.p.d == 64) s.split_rows ? fp32(IntC<64>{}, N1{}) : fp32(IntC<64>{}, IntC<0>{});
            else s.split_rows ? fp32(IntC<128>{}, N1{}) : fp32(IntC<128>{}, IntC<0>{});
        } else if (x.p.d == 64) x.rope ? shape(IntC<64>{}, N1{}) : shape(IntC<64>{}, IntC<0>{});
        else x.rope ? shape(IntC<128>{}, N1{}) : shape(IntC<128>{}, IntC<0>{});
        const int rc = launch_status();
        if (rc != SEPATTN_OK) return rc;
    }
    ProfScope prof(SEPATTN_K_DECODE_MERGE, st);
    auto go = [&](auto T_, auto D_) {
        using T = decltype(T_);
        constexpr int D = decltype(D_)::value;
        auto rows = [&](auto WPR_) {
            constexpr int WPR = decltype(WPR_)::value;
            const dim3 grid(WPR == 1 ? (x.p.Hq + kShWaves - 1) / kShWaves : x.p.Hq, x.p.S);
            hipLaunchKernelGGL((shared_merge_kernel<T, D, WPR>), grid, block, 0, st, x.p, x.pp.S, s.n_prefix, s.n_own, x.prefix_of, x.part,
                               own_part, static_cast<T *>(x.out), x.lse);
        };
        // one round trip of one wave where the records are few (128 sequences behind 2048 entries: 51.3 us a call, with four waves per row 55.8)
        s.n_prefix + s.n_own <= 8 ? rows(IntC<1>{}) : rows(IntC<kShWaves>{});
    };
    if (x.p.dtype == SEPATTN_BF16) x.p.d == 64 ? go(uint16_t{}, IntC<64>{}) : go(uint16_t{}, IntC<128>{});
    else x.p.d == 64 ? go(float{}, IntC<64>{}) : go(float{}, IntC<128>{});
    return launch_status();
}

}  // namespace sepattn
