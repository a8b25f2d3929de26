// Single-query attention behind shared prompts (Sec. 3.2 "Generation", Sec. 3.3): every sequence attends to the entries of the
// prefix cache that it shares with others and to those of its own cache.
//
// Softmax over the two sets is softmax over each, joined by maximum and sum, so the work is cut into
//   - the prefixes: all query heads of all sequences of a prefix that read one KV head are the rows of ONE product with its
//     keys and values, which are read once for all of them (per chunk of rows) and not once per sequence;
//   - the own caches, as sepattn_decode does (one slice of a cache per workgroup);
//   - the sum of the slices' records (maximum, sum, unnormalised output), one wave per (sequence, head).
#include "common.h"
#include "decode_common.h"
#include "mfma_common.h"

namespace sepattn {

namespace {

constexpr int kShThreads = 256, kShWaves = 4;
constexpr int kShBlock = 32;  // keys per block; slices are whole blocks

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

// What a workgroup has to do: chunk `blockIdx.y` of the rows of all prefixes, cut per prefix into chunks of ROWS.
struct Chunk {
    int prefix, row0, rows, first;  // first row of the chunk, rows and first entry in group_seq of the prefix
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
    e0 = min(split * per, entries);
    e1 = min(entries, e0 + per);
    return e0 < e1;
}
__device__ inline int slices_in_use(int entries, int nsplit) {
    const int nb = (entries + kShBlock - 1) / kShBlock, per = (nb + nsplit - 1) / nsplit;
    return per ? (nb + per - 1) / per : 0;
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

// ---- bf16 ------------------------------------------------------------------------------------------
// Four waves: RB row blocks of 32 rows, and KG = 4 / RB groups of waves that take the key tiles in turn.  The waves of a
// group share its stages of K and V rows in LDS (two, of TK keys).  Operands as in decode_mfma.hip: the cache rows are the A operand, a
// wave's 32 rows the columns of B, so a row's softmax state is in one lane pair.
// LO (turned queries): the query is the sum of two bf16 numbers, 16 bits of mantissa, and the scores are two products; rounded
// to one, lse would be off by 1e-3.
template <int D, int RB, bool LO>
__global__ __launch_bounds__(kShThreads, RB == 4 ? 2 : 1) void shared_prefix_kernel(PrefixArgs x) {
    constexpr int KG = kShWaves / RB, ROWS = 32 * RB, TK = RB == 1 ? 32 : 64;
    constexpr int CH = D / 8, RPL = 64 / CH;   // 16-byte chunks per cache row, rows per wave-wide load
    constexpr int NLD = TK / RB / RPL;         // such loads per wave, tensor and tile
    constexpr int KSTEPS = D / 16, KS2 = KSTEPS / 2, DB = D / 32, REC = kShRecord<D>;
    __shared__ __attribute__((aligned(1024))) uint16_t smem[KG][2][2][TK * D];  // [group][stage][K, V]

    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int rb = wave % RB, kg = wave / RB, col = lane & 31, hh = lane >> 5;
    const int kv = blockIdx.x, split = blockIdx.z;
    Chunk c;
    if (!find_chunk<ROWS>(x, blockIdx.y, c)) return;
    const CacheMap cm = cache_map(x.pp, x.prefix_sizes + SEPKV_SIZES_COLS * c.prefix);
    const int np = entries_of(cm);
    int e0, e1;
    if (!slice_of(np, x.nsplit, split, e0, e1)) return;
    const uint16_t *Kh = static_cast<const uint16_t *>(x.Kp) + ((long)c.prefix * x.p.Hkv + kv) * (long)x.pp.c * D;
    const uint16_t *Vh = static_cast<const uint16_t *>(x.Vp) + ((long)c.prefix * x.p.Hkv + kv) * (long)x.pp.c * D;

    const int tiles = (e1 - e0 + TK - 1) / TK, steps = (tiles + KG - 1) / KG;
    const int my_pc = lane % CH, my_sub = lane / CH;
    auto issue = [&](int step) {
        const int eb = e0 + (step * KG + kg) * TK;
        static_for<NLD>([&](auto U) {
            const int r = (rb * NLD + U) * RPL + my_sub;
            const uint32_t off = (uint32_t)decode_slot_of(cm, min(eb + r, e1 - 1)) * (uint32_t)(D * 2);
            dma_to_lds_16(Kh, off + swz_chunk<kSwzRow, D>(my_pc, r) * 16, lds_addr(&smem[kg][step & 1][0][(rb * NLD + U) * RPL * D]));
            dma_to_lds_16(Vh, off + swz_chunk<kSwzTr, D>(my_pc, r) * 16, lds_addr(&smem[kg][step & 1][1][(rb * NLD + U) * RPL * D]));
        });
    };

    // queries: B operand, column = row of the chunk
    int seq, head;
    row_of(x, c, c.row0 + rb * 32 + col, seq, head);
    const uint16_t *qrow = static_cast<const uint16_t *>(x.q) + ((long)seq * x.p.Hq + kv * x.gq + head) * D + 8 * hh;
    bf16x8 qhi[KSTEPS], qlo[LO ? KSTEPS : 1];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qhi[ks] = as_bf16x8(*reinterpret_cast<const u32x4 *>(qrow + 16 * ks));
    if constexpr (LO) {
        const float *row = x.rope + (long)query_position(x, seq, np) * D + 8 * hh;
#pragma unroll
        for (int ks = 0; ks < KS2; ++ks) {
            const f32x8 u = __builtin_convertvector(qhi[ks], f32x8), v = __builtin_convertvector(qhi[ks + KS2], f32x8);
            f32x8 cs, sn, a, b;
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = row[16 * ks + e], sn[e] = row[D / 2 + 16 * ks + e];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = fmaf(u[e], cs[e], -(v[e] * sn[e]));
                b[e] = fmaf(v[e], cs[e], u[e] * sn[e]);
            }
            qhi[ks] = __builtin_convertvector(a, bf16x8);
            qhi[ks + KS2] = __builtin_convertvector(b, bf16x8);
            qlo[ks] = __builtin_convertvector(a - __builtin_convertvector(qhi[ks], f32x8), bf16x8);
            qlo[ks + KS2] = __builtin_convertvector(b - __builtin_convertvector(qhi[ks + KS2], f32x8), bf16x8);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loop counts its own loads only
    issue(0);

    const float sl2 = x.p.scale * kLog2e_f;
    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    const int a_row = pi_row(col);

    for (int step = 0; step < steps; ++step) {
        if (step + 1 < steps) {
            issue(step + 1);
            static_assert(2 * NLD == 16 || 2 * NLD == 8 || 2 * NLD == 4, "wait counts are written for d = 64 and 128");
            if constexpr (2 * NLD == 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
            if constexpr (2 * NLD == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
            if constexpr (2 * NLD == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        if constexpr (RB > 1) {
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
        const uint16_t *Kst = smem[kg][step & 1][0], *Vst = smem[kg][step & 1][1];
        const int eb = e0 + (step * KG + kg) * TK;
#pragma unroll
        for (int blk = 0; blk < TK / 32; ++blk) {
            const int n_valid = e1 - (eb + 32 * blk);
            if (n_valid <= 0) continue;
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                const bf16x8 ka = lds_read_a_swz<kSwzRow, D>(Kst + 32 * blk * D, a_row, 2 * ks + hh);
                s = mfma_bf16(ka, qhi[ks], s);
                if constexpr (LO) s = mfma_bf16(ka, qlo[ks], s);
            }
            if (n_valid < 32) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (rho_row(hh, i) >= n_valid) s[i] = -INFINITY;
            }
            float m_loc = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) m_loc = fmaxf(m_loc, s[i]);
            const float m_new = fmaxf(m_run, pair_max(m_loc * sl2));  // finite: key 0 of the block is valid
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            float psum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -m_new));
                psum += s[i];
            }
            l_run = l_run * alpha + psum;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0ull) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
            }
            const bf16x8 p0 = pack_bf16x8(s, 0), p1 = pack_bf16x8(s, 8);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                oacc[db] = mfma_bf16(lds_read_a_tr_swz<kSwzTr, D>(Vst + 32 * blk * D, 0, db * 32, lane), p0, oacc[db]);
                oacc[db] = mfma_bf16(lds_read_a_tr_swz<kSwzTr, D>(Vst + 32 * blk * D, 16, db * 32, lane), p1, oacc[db]);
            }
        }
        // everyone has read the stage before the next step's loads overwrite it
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if constexpr (RB > 1) {
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
    }

    // ---- the key groups' states meet in LDS
    float l_tot = pair_sum(l_run);
    if constexpr (KG > 1) {
        __syncthreads();
        float *red = reinterpret_cast<float *>(smem);  // [row][group][REC]
        static_assert(sizeof(smem) >= sizeof(float) * ROWS * (KG - 1) * REC, "records fit the stages");
        if (kg > 0) {
            float *r = red + ((rb * 32 + col) * (KG - 1) + kg - 1) * REC;
            if (hh == 0) r[0] = m_run, r[1] = l_tot;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4 *>(r + 4 + db * 32 + 8 * i + 4 * hh) = f32x4{oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
        }
        __syncthreads();
        if (kg > 0) return;
        const float *r = red + (rb * 32 + col) * (KG - 1) * REC;
        float M = m_run;
#pragma unroll
        for (int k = 0; k < KG - 1; ++k) M = fmaxf(M, r[k * REC]);
        const float own = __builtin_amdgcn_exp2f(m_run - M);  // group 0 has the slice's first tile: m_run is finite
        l_tot *= own;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[db][i] *= own;
#pragma unroll
        for (int k = 0; k < KG - 1; ++k) {
            const float w = __builtin_amdgcn_exp2f(r[k * REC] - M);  // 0 for a group without a tile
            l_tot = fmaf(w, r[k * REC + 1], l_tot);
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(r + k * REC + 4 + db * 32 + 8 * i + 4 * hh);
#pragma unroll
                    for (int j = 0; j < 4; ++j) oacc[db][4 * i + j] = fmaf(w, v[j], oacc[db][4 * i + j]);
                }
        }
        m_run = M;
    }
    if (c.row0 + rb * 32 + col >= c.rows) return;
    float *r = x.part + (((long)seq * x.p.Hq + kv * x.gq + head) * x.nsplit + split) * REC;
    if (hh == 0) *reinterpret_cast<float2 *>(r) = float2{m_run, l_tot};
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4 *>(r + 4 + db * 32 + 8 * i + 4 * hh) = f32x4{oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
}

// ---- fp32 ------------------------------------------------------------------------------------------
// Four waves of 16 rows each, tiles of 32 keys in LDS, v_mfma_f32_16x16x4_f32 with fp32 operands.  Lane l, group g = l / 16.  Scores: A = K, row
// l%16 = key, B = queries, column l%16; the four k-slots of step 4 S + i are dimensions 16 S + 4 g + i, so that a lane's
// operands are pieces of 16 bytes.  C: column l%16 = query, rows 4 g + i = keys.  Output: O^T += V^T P^T, the k-slots of step i
// are keys 4 g + i, which the lane group holds.
typedef float f4 __attribute__((ext_vector_type(4)));
template <int D>
__global__ __launch_bounds__(kShThreads) void shared_prefix_fp32_kernel(PrefixArgs x) {
    constexpr int ROWS = 16 * kShWaves, TK = kShBlock, PITCH = D + 4, REC = kShRecord<D>;
    __shared__ __attribute__((aligned(16))) float ks[TK * PITCH], vs[TK * PITCH];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = lane & 15, g = lane >> 4;
    const int kv = blockIdx.x, split = blockIdx.z;
    Chunk c;
    if (!find_chunk<ROWS>(x, blockIdx.y, c)) return;
    const CacheMap cm = cache_map(x.pp, x.prefix_sizes + SEPKV_SIZES_COLS * c.prefix);
    const int np = entries_of(cm);
    int e0, e1;
    if (!slice_of(np, x.nsplit, split, e0, e1)) return;
    const float *Kh = static_cast<const float *>(x.Kp) + ((long)c.prefix * x.p.Hkv + kv) * (long)x.pp.c * D;
    const float *Vh = static_cast<const float *>(x.Vp) + ((long)c.prefix * x.p.Hkv + kv) * (long)x.pp.c * D;
    int seq, head;
    row_of(x, c, c.row0 + wave * 16 + col, seq, head);
    const float *qrow = static_cast<const float *>(x.q) + ((long)seq * x.p.Hq + kv * x.gq + head) * D + 4 * g;
    f4 q[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q[s] = *reinterpret_cast<const f4 *>(qrow + 16 * s);
    if (x.rope) {
        const float *row = x.rope + (long)query_position(x, seq, np) * D + 4 * g;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const f4 cs = *reinterpret_cast<const f4 *>(row + 16 * s), sn = *reinterpret_cast<const f4 *>(row + D / 2 + 16 * s);
            const f4 u = q[s], v = q[s + D / 32];
            q[s] = u * cs - v * sn;
            q[s + D / 32] = v * cs + u * sn;
        }
    }
    const float sl2 = x.p.scale * kLog2e_f;
    f4 o[D / 16];
#pragma unroll
    for (int db = 0; db < D / 16; ++db) o[db] = f4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (int eb = e0; eb < e1; eb += TK) {
        __syncthreads();
        for (int i = threadIdx.x; i < TK * (D / 4); i += kShThreads) {
            const int r = i / (D / 4), pc = i % (D / 4) * 4;
            const long off = (long)decode_slot_of(cm, min(eb + r, e1 - 1)) * D + pc;
            *reinterpret_cast<f4 *>(ks + r * PITCH + pc) = *reinterpret_cast<const f4 *>(Kh + off);
            *reinterpret_cast<f4 *>(vs + r * PITCH + pc) = *reinterpret_cast<const f4 *>(Vh + off);
        }
        __syncthreads();
#pragma unroll
        for (int blk = 0; blk < TK / 16; ++blk) {
            const int n_valid = e1 - eb - 16 * blk;
            if (n_valid <= 0) continue;
            f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < D / 16; ++st) {
                const f4 k = *reinterpret_cast<const f4 *>(ks + (16 * blk + col) * PITCH + 16 * st + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[st][i], s, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = 4 * g + i < n_valid ? s[i] * sl2 : -INFINITY;
            float m_new = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
            m_new = fmaxf(m_new, __shfl_xor(m_new, 16));
            m_new = fmaxf(m, fmaxf(m_new, __shfl_xor(m_new, 32)));  // finite: key 0 of the block is valid
            const float alpha = exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] = exp2f(s[i] - m);
                l += s[i];
            }
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                o[db] *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(vs[(16 * blk + 4 * g + i) * PITCH + 16 * db + col], s[i], o[db], 0, 0, 0);
            }
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (c.row0 + wave * 16 + col >= c.rows) return;
    float *r = x.part + (((long)seq * x.p.Hq + kv * x.gq + head) * x.nsplit + split) * REC;
    if (g == 0) r[0] = m, r[1] = l;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f4 *>(r + 4 + 16 * db + 4 * g) = o[db];
}

// ---- the slices' sum: one wave per (sequence, head), prefix slices first, then the own cache's, in order ------------
template <typename T, int D>
__global__ __launch_bounds__(kShThreads) void shared_merge_kernel(sepkv_params p, sepkv_params pp, int n_prefix, int n_own,
                                                                  const int32_t *__restrict__ prefix_sizes, const int32_t *__restrict__ prefix_of,
                                                                  const float *__restrict__ prefix_part, const float *__restrict__ own_part,
                                                                  T *__restrict__ out, float *__restrict__ lse) {
    constexpr int REC = kShRecord<D>, OWN = D + 2, C = D / kWave;
    const int lane = threadIdx.x % kWave;
    const long row = (long)blockIdx.x * kShWaves + threadIdx.x / kWave;
    if (row >= (long)p.S * p.Hq) return;
    const int of = prefix_of[row / p.Hq];
    const int np = of >= 0 && of < pp.S ? slices_in_use(entries_of(cache_map(pp, prefix_sizes + SEPKV_SIZES_COLS * of)), n_prefix) : 0;
    const int total = np + n_own;
    const float *pre = prefix_part + row * n_prefix * REC, *own = own_part + row * n_own * OWN;
    auto record = [&](int k) { return k < np ? pre + k * REC : own + (k - np) * OWN; };
    float M = -INFINITY;
    for (int k = lane; k < total; k += kWave) M = fmaxf(M, record(k)[0]);
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) M = fmaxf(M, __shfl_xor(M, o));
    float l = 0.f, o[C] = {};
    for (int k0 = 0; k0 < total; k0 += kWave) {
        const int n = min(kWave, total - k0);
        float w = 0.f, ml = 0.f;
        if (lane < n) {
            const float *r = record(k0 + lane);
            w = r[0] == -INFINITY ? 0.f : exp2f(r[0] - M);
            ml = r[1];
        }
        for (int k = 0; k < n; ++k) {
            const float wk = __shfl(w, k);
            const float *r = record(k0 + k) + (k0 + k < np ? 4 : 2) + C * lane;
            l = fmaf(wk, __shfl(ml, k), l);
#pragma unroll
            for (int i = 0; i < C; ++i) o[i] = fmaf(wk, r[i], o[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const float v = l > 0.f ? o[i] / l : 0.f;
        if constexpr (sizeof(T) == 2) out[row * D + C * lane + i] = decode_f32_to_bf16(v);
        else out[row * D + C * lane + i] = v;
    }
    if (lse && lane == 0) lse[row] = l > 0.f ? (M + log2f(l)) * kLn2_f : -INFINITY;
}

// ---- host ------------------------------------------------------------------------------------------
struct SharedShape {
    int rb;        // bf16: row blocks per workgroup
    int chunks;    // of rows, all prefixes together, at most
    int n_prefix;  // slices per prefix
    int n_own;     // slices per own cache
};
SharedShape shared_shape(const sepkv_params &p, const sepkv_params &pp) {
    SharedShape s;
    const long gq = p.Hq / p.Hkv, all = p.S * gq, per_prefix = (all + pp.S - 1) / pp.S;
    s.rb = per_prefix <= 32 ? 1 : per_prefix <= 64 ? 2 : 4;
    const long rows = p.dtype == SEPATTN_FP32 ? 64 : 32 * s.rb;
    s.chunks = (int)(pp.S == 1 ? (all + rows - 1) / rows : all / rows + (pp.S < p.S ? pp.S : p.S));
    const long nb = (pp.c + kShBlock - 1) / kShBlock, groups = (long)p.Hkv * s.chunks;
    long ns = (2L * compute_units() + groups - 1) / groups;
    if (ns > nb / 4) ns = nb / 4;
    s.n_prefix = (int)(ns < 1 ? 1 : ns > 64 ? 64 : ns);
    s.n_own = decode_record_slices(p);
    return s;
}
size_t prefix_record_bytes(const sepkv_params &p, const SharedShape &s) {
    return align_up((size_t)p.S * p.Hq * s.n_prefix * (p.d + 4) * sizeof(float), 256);
}

}  // namespace

size_t decode_shared_workspace(const sepkv_params &p, const sepkv_params &pp) {
    const SharedShape s = shared_shape(p, pp);
    return prefix_record_bytes(p, s) + align_up((size_t)p.S * p.Hq * s.n_own * (p.d + 2) * sizeof(float), 256);
}

int launch_decode_shared(const SharedDecode &x, hipStream_t st) {
    const SharedShape s = shared_shape(x.p, x.pp);
    float *const own_part = x.part + prefix_record_bytes(x.p, s) / sizeof(float);
    const PrefixArgs a = {x.p, x.pp, x.p.Hq / x.p.Hkv, s.n_prefix, x.q, x.Kp, x.Vp, x.sizes, x.prefix_sizes, x.group_start, x.group_seq,
                          x.rope, x.n_pos, x.part};
    const dim3 grid(x.p.Hkv, s.chunks, s.n_prefix), block(kShThreads);
    {
        ProfScope prof(SEPATTN_K_DECODE_SPLIT, st);
        auto go = [&](auto D_) {
            constexpr int D = decltype(D_)::value;
            if (x.p.dtype == SEPATTN_FP32) {
                hipLaunchKernelGGL((shared_prefix_fp32_kernel<D>), grid, block, 0, st, a);
                return;
            }
            auto rows = [&](auto RB_) {
                constexpr int RB = decltype(RB_)::value;
                if (x.rope) hipLaunchKernelGGL((shared_prefix_kernel<D, RB, true>), grid, block, 0, st, a);
                else hipLaunchKernelGGL((shared_prefix_kernel<D, RB, false>), grid, block, 0, st, a);
            };
            s.rb == 1 ? rows(IntC<1>{}) : s.rb == 2 ? rows(IntC<2>{}) : rows(IntC<4>{});
        };
        x.p.d == 64 ? go(IntC<64>{}) : go(IntC<128>{});
    }
    int rc = launch_status();
    if (rc != SEPATTN_OK) return rc;
    rc = launch_decode_records(x.p, s.n_own, x.q, x.Kc, x.Vc, x.sizes, x.rope, x.n_pos, own_part, st);
    if (rc != SEPATTN_OK) return rc;
    ProfScope prof(SEPATTN_K_DECODE_MERGE, st);
    const dim3 merge(((unsigned)(x.p.S * x.p.Hq) + kShWaves - 1) / kShWaves);
    auto go = [&](auto T_, auto D_) {
        using T = decltype(T_);
        hipLaunchKernelGGL((shared_merge_kernel<T, decltype(D_)::value>), merge, block, 0, st, x.p, x.pp, s.n_prefix, s.n_own, x.prefix_sizes,
                           x.prefix_of, x.part, own_part, static_cast<T *>(x.out), x.lse);
    };
    if (x.p.dtype == SEPATTN_BF16) x.p.d == 64 ? go(uint16_t{}, IntC<64>{}) : go(uint16_t{}, IntC<128>{});
    else x.p.d == 64 ? go(float{}, IntC<64>{}) : go(float{}, IntC<128>{});
    return launch_status();
}

}  // namespace sepattn
