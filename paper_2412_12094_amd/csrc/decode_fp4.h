// How a decode over the cache in 4 bits is cut into slices (decode_fp4.hip).  A header of its own so that a host program can check that they fit what is
// launched and what the workspace holds.
#pragma once

#include <algorithm>

#include "common.h"

namespace sepattn {

constexpr int kMxRows = 32;                   // entries per block; slices are whole blocks
constexpr int kMxColumns = 16;                // query heads of a workgroup
constexpr int kMxWaves = 4;                   // ... its waves
constexpr int kMxLeastBlocks = kMxWaves;      // of a slice
constexpr int kMxManyBlocks = 20;             // of a slice where there is more than one workgroup per compute unit
constexpr int kMxMostSlices = 64;             // of a sequence
constexpr int kMxMostAdded = 16;              // of a sequence whose slices the kernel itself adds
constexpr int kMxMostDivided = 512;           // sequences of a call in which they are cut

// How sequences are cut into slices.  Their lengths stand on the device, and those of a batch differ, so every workgroup finds its slice by itself.
// With T blocks in all sequences a slice has at most  share = max(kMxLeastBlocks, min(T / one, max(kMxManyBlocks, T / all)) + 1)  blocks, where `one`
// and `all` are the workgroups that one (KV head, 16 query heads) has if there is one per compute unit and if there are as many as it holds: more than one
// only where slices stay long enough to pay for being added.  A sequence of nb blocks has ceil(nb / share) slices, at least 1, at most `most`; they are
// numbered through all sequences and at most  all + S.  (most 1: the slices are the sequences.)
// Against as many slices for every sequence of the batch, chosen by the capacity (bf16, d = 128, 32 query heads on 8 KV heads; the kernel's loop as it was
// then): 32 sequences of 1 to 3277 entries 20.5 -> 18.8 us, with positions 36.5 -> 30.1; 8 of up to 8192 15.8 -> 14.5; 4 of up to 53019 29.7 -> 30.8, where
// memory was the bound and the search is on the way.  With positions and equal lengths of 1706 entries, one, two and three workgroups per unit took 29.8,
// 27.7 and 26.8 us.
//
// Batches of many sequences are cut less and less and in the end not at all: where `all` leaves no workgroup to spare (with 256 compute units from 182 sequences at
// 8 KV heads, 118 at 12, 38 at 32 on), and past kMxMostDivided.  Similar lengths fill the chip then.  One long sequence is walked by one workgroup per KV
// head: 32768 entries among 191 of 500 at 8 KV heads 196 us, where all of 500 take 25; among 149 others 50 and 26.
struct MxPlan {
    int most;
    float per_one, per_all;  // 1 / one, 1 / all
};
// `share` for `total` blocks (512 sequences: below 2^28; rounded in fp32, alike in every workgroup).  one <= all, so it is above total / all
__host__ __device__ inline int mx_share(const MxPlan &plan, int total) {
    const int one = (int)((float)total * plan.per_one), all = (int)((float)total * plan.per_all), many = all > kMxManyBlocks ? all : kMxManyBlocks;
    const int share = (one < many ? one : many) + 1;
    return share > kMxLeastBlocks ? share : kMxLeastBlocks;
}
// slices of a sequence of nb blocks (c d < 2^30, so nb < 2^19)
__host__ __device__ inline int mx_slices(const MxPlan &plan, int nb, float per_share) {
    const int n = 1 + small_quotient(nb > 0 ? nb - 1 : 0, per_share);
    return n < plan.most ? n : plan.most;
}

struct MxShape {
    MxPlan plan;
    int slices;  // there are no more, for one (KV head, 16 query heads)
    bool add;    // the kernel adds them itself
};
inline int mx_chunks(const sepkv_params &p) { return (p.Hq / p.Hkv + kMxColumns - 1) / kMxColumns; }
inline MxShape mx_shape(const sepkv_params &p, int units) {
    const int rows = p.Hkv * mx_chunks(p), nb = (p.c + kMxRows - 1) / kMxRows, row = std::min(p.Hq / p.Hkv, kMxColumns) * p.d;
    // Three workgroups per compute unit; cut lengths add about half a slice per sequence, or S at most.  The registers have room for three or four of every form
    // but one, fp32 with positions at d = 128, which has two: counted with two, 32 sequences of 1 to 3277 entries take 41 us instead of 43 there and 4 of up to
    // 53019 68 instead of 72, but 8 of up to 8192 30.1 instead of 29.2, and at d = 64, where three fit, 32 sequences 40.5 instead of 32.2.
    const int all = 3 * units / rows - std::min(p.S, 4 + p.S / 2), one = std::min(std::max(units / rows, 1), all);
    if (nb <= kMxLeastBlocks || all <= 0 || p.S > kMxMostDivided) return {{1, 0.f, 0.f}, p.S, false};
    // Added by the kernel or by a launch of its own (us, bf16, d = 128).  Rows of 512 floats, 4 query heads on each of 8 KV heads: 8 sequences of up to 8192
    // entries 14.2 by the kernel, 14.9 by a launch.  Of 1024, 8 on each: one sequence of 3332 slots 10.1 and 9.4, 8 level, 32 20.0 and 21.4: the smaller
    // calls decide.  With more than 256 blocks sixteen slices, which is all that the kernel adds, are too few: one sequence of 16384 slots 10.7 and
    // 9.8, of 32768 15.3 and 13.1 (of 8192 8.6 and 9.0).
    const bool add = kMxMostAdded * row <= 8192 && nb <= kMxMostAdded * kMxMostAdded;
    const int most = std::min((nb + kMxLeastBlocks - 1) / kMxLeastBlocks, add ? kMxMostAdded : kMxMostSlices);
    return {{most, 1.f / one, 1.f / all}, all + p.S, add};
}
// records in the workspace, each of a slice and a query head
inline size_t mx_records(const sepkv_params &p, const MxShape &x) { return x.plan.most == 1 ? 0 : (size_t)x.slices * p.Hq; }

}  // namespace sepattn
