// What the kernels of the shared-prefix attention have in common: sizes, addresses, where partial results lie.
#pragma once

#include "kernels.cuh"

namespace cass {

constexpr int kSaTok = 64;                               // positions of a tile of the streaming kernel
constexpr int kSaMaxSeq = 1024;

struct SharedAttn {
    int n_seq, rows, n_q, n_kv, group, d, prefix, capacity;
    int64_t q_seq, q_row, q_head, out_seq, out_row, out_head, p_pos, p_head, c_seq, c_pos, c_head;      // elements
    float scale_log2;                                    // scores are kept as powers of two
    const uint16_t *q, *kp, *vp, *kc, *vc;
    const int32_t* lens;
    // scratch.  A part: the unnormalised output, maximum and sum of up to `pairs` (row, query head) pairs over some positions.
    float *part_o, *part_m, *part_l;                     // [slot][pairs][d], [slot][pairs], [slot][pairs]
    float* scores;                                       // [sequence][query head x row in pair order][capacity], for the weights; or null
    // the streaming kernel's work
    int ctas, pairs;                                     // CTAs; pairs of a segment
    int p_groups, c_groups;                              // segments of pairs of the prefix (0: not this kernel's) and of a sequence
    // The prefix by the tensor-core kernel: the pairs of all sequences in tiles of 128.  Two tiles a CTA, `pre_n2` CTAs a head, its positions over
    // `pre_s2` CTAs: parts [split][head][CTA][256].  What is left over, one tile, over `pre_s1` (0: nothing is left): parts
    // [2 split + warpgroup][head][128], pre_at1 pairs further.
    float *pre_o, *pre_m, *pre_l;
    int pre_n2, pre_s2, pre_s1;
    int64_t pre_at1;
};
constexpr int kStTile = 128;                             // pairs and positions of a tile of that kernel

// Whether the tensor-core kernel can take this prefix, and over how many CTAs; the number of pairs that its parts hold.
bool shared_tc_usable(const SharedAttn& a);
int64_t shared_tc_plan(SharedAttn& a);

// Positions of sequence b's cache; -1: the sequence is not there.
__device__ __forceinline__ int shared_len(const SharedAttn& a, int b) {
    const int n = a.lens ? a.lens[b] : 0;
    return n < 0 ? -1 : min(n, a.capacity);
}

// The streaming kernel's segments are numbered: those of the prefix (group, head), then those of the sequences (sequence, group,
// head); their tiles form one list of T, worker w of W = min(T, CTAs) takes tiles w T / W to (w + 1) T / W (one at least), and its part
// of segment s goes to slot w + s (from one part to the next either number grows, so no two share a slot).
__device__ __forceinline__ int shared_workers(int64_t tiles, int ctas) { return (int)min(tiles, (int64_t)ctas); }
__device__ __forceinline__ int64_t shared_first_tile(int64_t tiles, int workers, int w) { return tiles * w / workers; }
__device__ __forceinline__ int shared_worker_of(int64_t tiles, int workers, int64_t t) { return (int)(((t + 1) * workers - 1) / tiles); }

int launch_shared_prefix_tc(const SharedAttn& a, int dtype, int32_t* d_status, cudaStream_t s);

}  // namespace cass
