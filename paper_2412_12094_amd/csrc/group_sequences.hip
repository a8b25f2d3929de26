// The sequences of a batch listed by the prefix they share (plan of the shared decode, made once per batch).
//
// One wave per prefix g, and one more for the end: it walks through prefix_of[0 .. S), 1024 entries per round trip.  The number of entries
// with 0 <= prefix_of < g is where its own begin; those it finds are written in ascending order at begin + (how many before),
// counted with ballots.  Every wave reads the whole array (L2), no wave waits for another and nothing has to be cleared: G S / 64
// steps of a few instructions.  Up to 1024 sequences the entries stay in registers between the two walks (G = 12, S = 1000: 3.1 us, of
// which the launch is most; with 64 entries per round trip 8.0).
#include "common.h"

namespace sepattn {

namespace {

constexpr int kGroupWaves = 4;

__global__ __launch_bounds__(kWave * kGroupWaves) void group_sequences_kernel(const int32_t *__restrict__ prefix_of, int S, int G,
                                                                              int32_t *__restrict__ group_start, int32_t *__restrict__ group_seq) {
    const int g = blockIdx.x * kGroupWaves + threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (g > G) return;
    constexpr int N = 16;
    int of[N];
    auto read = [&](int s0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int s = s0 + i * kWave + lane;
            of[i] = s < S ? prefix_of[s] : -1;
        }
    };
    int begin = 0;
    for (int s0 = 0; s0 < S; s0 += N * kWave) {
        read(s0);
#pragma unroll
        for (int i = 0; i < N; ++i) begin += __builtin_popcountll(__ballot(of[i] >= 0 && of[i] < g));
    }
    if (lane == 0) group_start[g] = begin;
    if (g == G) {  // the entries behind the last prefix's
        for (int i = begin + lane; i < S; i += kWave) group_seq[i] = 0;
        return;
    }
    for (int s0 = 0; s0 < S; s0 += N * kWave) {
        if (S > N * kWave) read(s0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool mine = of[i] == g;
            const uint64_t all = __ballot(mine);
            if (mine) group_seq[begin + __builtin_popcountll(all & ((1ull << lane) - 1))] = s0 + i * kWave + lane;
            begin += __builtin_popcountll(all);
        }
    }
}

}  // namespace

int launch_group_sequences(const int32_t *prefix_of, int S, int G, int32_t *group_start, int32_t *group_seq, hipStream_t st) {
    hipLaunchKernelGGL(group_sequences_kernel, dim3(G / kGroupWaves + 1), dim3(kWave * kGroupWaves), 0, st, prefix_of, S, G, group_start,
                       group_seq);
    return launch_status();
}

}  // namespace sepattn
