// What the kernels of the shared-prefix attention have in common: sizes, addresses, where partial results lie.
#pragma once

#include <cuda_fp16.h>

#include "kernels.cuh"

namespace cass {

// ---- 16-bit types ----
template <int DT> struct SaType;
template <> struct SaType<CASS_BF16> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static constexpr uint32_t kExponent = 0x7F80u;
    static __device__ __forceinline__ float get(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ uint16_t put(float v) { return float_to_bf16_bits(v); }
};
template <> struct SaType<CASS_F16> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static constexpr uint32_t kExponent = 0x7C00u;
    static __device__ __forceinline__ float get(uint32_t v) { return __half2float(__ushort_as_half((uint16_t)v)); }
    static __device__ __forceinline__ uint16_t put(float v) { return __half_as_ushort(__float2half_rn(v)); }
};

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

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
    float* scores;                                       // [sequence][KV head][pair][score_stride], for the weights; or null
    int64_t score_stride;                                // the capacity, rounded up to 4
    // the streaming kernel's work
    int behind_tc;                                       // it is launched behind the tensor-core kernel, whose parts it does not need
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
// head); their tiles form one list of T, of which worker w of W = min(T, CTAs) takes those from w T / W on, and its part of segment s goes
// to slot w + s (from one part to the next either number grows, so no two share a slot).  (T / W + 1 tiles for the first T % W workers and
// T / W for the others sets neighbours the same distance apart: one cache of 32000 positions 29 -> 35 us.)
struct SaList {
    int p_tiles, p_total, seq_segs, p_segs, total, workers;
    uint64_t step;                                       // T / W in 2^-32
};
__device__ __forceinline__ SaList shared_list(const SharedAttn& a, int c_tiles) {      // c_tiles: tiles of all sequences' lengths
    SaList s;
    s.p_tiles = a.p_groups ? ceil_div(a.prefix, kSaTok) : 0;
    s.p_segs = a.p_groups * a.n_kv;
    s.seq_segs = a.c_groups * a.n_kv;
    s.p_total = s.p_tiles * s.p_segs;
    s.total = s.p_total + c_tiles * s.seq_segs;
    s.workers = max(min(s.total, a.ctas), 1);
    // long division, 16 bits at a time (the remainders are below the number of CTAs, below 2^16)
    const uint32_t W = (uint32_t)s.workers, each = (uint32_t)s.total / W, r0 = ((uint32_t)s.total - each * W) << 16, q1 = r0 / W, r1 = (r0 - q1 * W) << 16;
    s.step = ((uint64_t)each << 32) | (q1 << 16) | (r1 / W);
    return s;
}
__device__ __forceinline__ int shared_first_tile(const SaList& s, int w) { return w >= s.workers ? s.total : (int)(((uint64_t)(uint32_t)w * s.step) >> 32); }
__device__ __forceinline__ int shared_worker_of(const SaList& s, int t) {
    int w = min((int)__fdividef((float)t * (float)s.workers, (float)s.total), s.workers - 1);      // one off at most
    while (w > 0 && shared_first_tile(s, w) > t) --w;
    while (shared_first_tile(s, w + 1) <= t) ++w;
    return w;
}
constexpr int64_t kSaMaxTiles = 1 << 30;

// mt: tiles of 16 pairs that a CTA takes at a time, 1, 2 or 4 (1 beyond head size 128)
int launch_shared_stream_bf16(const SharedAttn& a, int mt, int32_t* d_status, cudaStream_t s);
int launch_shared_stream_f16(const SharedAttn& a, int mt, int32_t* d_status, cudaStream_t s);
int launch_shared_prefix_tc(const SharedAttn& a, int dtype, int32_t* d_status, cudaStream_t s);

}  // namespace cass
