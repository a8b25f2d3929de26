// How a decode behind shared prompts is cut: rows per workgroup, waves, slices (decode_shared.hip).  A header of its own so that a host program can
// say which kernel a call takes.
#pragma once

#include <algorithm>
#include <cmath>

#include "common.h"

namespace sepattn {

constexpr int kShBlock = 32;  // keys per block; slices are whole blocks

struct SharedShape {
    bool split_rows;  // bf16: what shared_body's waves share
    int nb;           // bf16: column blocks of a wave
    int waves;        // bf16: per workgroup
    int chunks;       // of rows, all prefixes together, at most
    int n_prefix;     // slices per prefix
    int n_own;        // slices per own cache
};
// From the capacities and from the mean number of rows per prefix place (the device alone knows how much of them is in use): a pool of G places of which
// few are used is cut as if the sequences were spread over all of them, into few rows a workgroup and few slices (48 sequences behind one prompt of 65536
// entries: 102 us with G = 1, 149 with 4, 394 with 8, 567 with 16; 32 behind 8192: 28, 39 with 4, 81 with 16).
// Figures: microseconds of a call, 32/8 heads, d = 128, bf16, without positions unless said, each line from one machine (two differ by up to 8 %); rows: of
// one KV head and prefix.
// Rows and waves.  Up to 32 rows every wave has all of them (18 us; cut by rows 18.5: 8 sequences behind 8192 entries); above, each wave its own:
//     64 rows, 8192 entries                              20.9 (23.5 with all of them in each wave)
//     192 rows, 65536 entries, 3 / 2 / 1 column blocks    85 / 107 / 102: an entry read from LDS serves more rows (best of several numbers of slices)
//     128 rows, 8192 entries,  2 / 1 column blocks        28.4 / 27.0, turned 33.2 / 31.2: slices of fewer than 20 steps
//   NW = 8 where a slice is long and there are many: 192 rows, 65536 entries 85 to 90 over 20 to 28 slices (4 waves, 32 to 48 slices: 90 to 99), 128 rows
//     69 (74); 8192 entries 29 (27.5).
// Slices.  `bytes_us`: what reading every cache once takes.  A prefix is cut so finely that a workgroup's walk through its slice, at `step` per
// 32 keys while the memory is busy, ends well before that, and at least so finely that half of the places that the chip has for workgroups
// are taken; finer, and a slice more costs a record per row, written and read again (192 rows, 65536 entries, 16 / 20 / 24 / 28 / 32 slices: 98 / 87 / 85 /
// 89 / 97, with the rule's 27 90; 128 rows, 8192 entries, turned, 8 / 12 / 16 / 20 of one column block: 32.4 / 31.4 / 32.1 / 43.3, with the rule's 13 31.2).  Turned
// queries, whose scores are two products, take longer per step, but so do the own caches beside them, and fewer slices pay: 96 rows, 20000 entries
// 35.0 (steps of 0.95 and 1.1: 39.6), 400 rows, 4096 entries 52.1 (56.7).  Where it misses the best of a sweep: 192 rows, 65536 entries, turned, two column
// blocks and 32 slices 127; 28 slices 121, one block and 20 slices 117.
inline SharedShape shared_shape(const sepkv_params &p, const sepkv_params &pp, bool rope) {
    SharedShape s = {};
    const long gq = p.Hq / p.Hkv, all = p.S * gq, per_prefix = (all + pp.S - 1) / pp.S, units = compute_units();
    const long nb = (pp.c + kShBlock - 1) / kShBlock, own_nb = (p.c + kShBlock - 1) / kShBlock;
    auto chunks_of = [&](long rows) { return pp.S == 1 ? (all + rows - 1) / rows : all / rows + (pp.S < p.S ? pp.S : p.S); };
    s.waves = 4;
    const bool fp32 = p.dtype == SEPATTN_FP32;
    const long slots = (p.d == 64 ? 3 : 2) * units, own_groups = (long)p.S * p.Hkv * ((gq + 15) / 16);
    const double own_rows = (double)p.S * p.c, prefix_rows = (double)pp.S * pp.c, bytes_us = (fp32 ? 8.0 : 4.0) * p.d * p.Hkv * (own_rows + prefix_rows) / 5.3e6;
    const double most_us = std::max(5.0, bytes_us * (0.4 + 0.5 * prefix_rows / (own_rows + prefix_rows)));
    auto cut = [&](double step) {
        const long groups = (long)p.Hkv * s.chunks, finest = std::clamp(nb / (fp32 ? 2 : nb > 64 ? 8 : 4), 1L, 64L), room = (slots - own_groups) / groups;
        long ns = std::max((long)std::ceil(nb * step * (p.d == 64 ? 0.6 : 1.0) / most_us - 0.25), (slots / 2 - own_groups) / groups);
        // no second round of workgroups for a few slices
        if (ns > room && room * 10 >= ns * 6) ns = room;
        else if (ns > slots / groups && slots / groups * 10 >= ns * 7) ns = slots / groups;
        return (int)std::clamp(ns, 1L, finest);
    };
    if (fp32) {
        s.split_rows = per_prefix > 16;
        s.chunks = (int)chunks_of(s.split_rows ? 64 : 16);
        s.n_prefix = cut(s.split_rows ? 1.9 : 0.5);
    } else if (per_prefix <= 32) {
        s.nb = per_prefix <= 16 ? 1 : 2;
        s.chunks = (int)chunks_of(16 * s.nb);
        s.n_prefix = cut(s.nb == 1 ? 0.35 : 0.45);
    } else {
        s.split_rows = true;
        static const double step[2][3] = {{0.75, 0.85, 1.05}, {0.7, 0.9, 0.}};
        s.nb = per_prefix <= 64 ? 1 : per_prefix <= 128 ? 2 : 3;
        // three column blocks where they waste no more rows than two (turned queries at d = 128 have no registers for them)
        if (s.nb == 3 && ((rope && p.d == 128) || (per_prefix + 191) / 192 * 3 > (per_prefix + 127) / 128 * 2)) s.nb = 2;
        for (;; --s.nb) {  // fewer rows per workgroup, and more workgroups, where a slice would be a few steps and there is room
            s.chunks = (int)chunks_of(64 * s.nb);
            s.n_prefix = cut(step[rope && p.d == 128][s.nb - 1]);
            if (s.nb == 1 || nb / s.n_prefix >= 20 || own_groups + (long)p.Hkv * ((all + 64 * s.nb - 1) / (64 * s.nb)) * s.n_prefix >= slots) break;
        }
        if (p.d == 128 && !rope && s.nb > 1 && s.n_prefix >= 24) {
            s.waves = 8;
            s.n_prefix = (s.n_prefix * 7 + 5) / 10;
        }
    }
    const long no = (slots / 2) / own_groups;
    s.n_own = (int)std::clamp(no, 1L, std::clamp(own_nb / 4, 1L, 64L));
    return s;
}
inline size_t prefix_record_bytes(const sepkv_params &p, const SharedShape &s) {
    return align_up((size_t)p.S * p.Hq * s.n_prefix * (p.d + 4) * sizeof(float), 256);
}
inline size_t own_record_bytes(const sepkv_params &p, const SharedShape &s) {
    return align_up((size_t)p.S * p.Hq * s.n_own * (p.d + 4) * sizeof(float), 256);
}

}  // namespace sepattn
