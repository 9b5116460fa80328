// What the kernels of the shared-prefix attention have in common: sizes, addresses, where partial results lie.
#pragma once

#include <cuda_fp16.h>

#include "kernels.cuh"

namespace cass {

// ---- 16-bit types ----
// Numerators of the softmax are rounded to the type for the second product, half a step of each (2^-8 of it in bf16, 2^-11 in fp16): an output
// is off by less than such a step of the values' weighted sizes, as its own rounding is, and the products run at the 16-bit rate.  Their sums stay
// in 32 bits and are of the numerators before that.  fp16 has no exponents for a long flat tail behind a favoured position (below 2^-14 of the
// maximum its steps stay the same, below 2^-25 there is nothing), so its numerators are relative to 2^-lift of the base and reach 2^15, with
// the kernels' room for growth; parts carry the base so lowered as their maximum, and the merge needs not know.
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
    static constexpr float kGrowth = 8.f;                // powers of two that numerators may grow over their base before what was summed is rescaled
    static constexpr float kLift = 0.f;                  // of numerators that are rescaled at every new maximum
    static __device__ __forceinline__ float get(uint32_t v) { return __uint_as_float(v << 16); }
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
    static constexpr float kGrowth = 4.f;                // (with 8, and no lift: 64 sequences of 40 heads behind 32768 positions 90.3 us, so 92.8)
    static constexpr float kLift = 15.f;
    static __device__ __forceinline__ float get(uint32_t v) { return __half2float(__ushort_as_half((uint16_t)v)); }
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
    float* part_o;                                       // [slot][pairs][d]
    float2* part_ml;                                     // [slot][pairs]
    int2* slots;                                         // [segment]: the first and the last slot of the streaming kernel's parts
    int n_slots;                                         // that part_o and part_ml have
    float* scores;                                       // [sequence][KV head][pair][score_stride], for the weights; or null
    int64_t score_stride;                                // the capacity, rounded up to 4
    float* lse;                                          // [sequence][KV head][pair], in powers of two, for the weights
    // the streaming kernel's work
    int behind_tc;                                       // it is launched behind the tensor-core kernel, whose parts it does not need
    int ctas, pairs;                                     // spans at most (CTAs that fit the GPU, tiles that there can be); pairs of a segment, at most
    int p_groups, c_groups;                              // segments of pairs of the prefix (0: not this kernel's) and of a sequence
    // The prefix by the tensor-core kernel: the pairs of all sequences in tiles of 128.  Two tiles a CTA, `pre_n2` CTAs a head, its positions over
    // `pre_s2` CTAs: parts [split][head][CTA][256].  What is left over, one tile, over `pre_s1` (0: nothing is left): parts
    // [2 split + warpgroup][head][128], pre_at1 pairs further.
    float* pre_o;
    float2* pre_ml;
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
// head); their tiles form one list, cut into as many even spans as CTAs fit the GPU (a tile at least).  SMs do not get the same share of the
// memory's rate (of equal spans of one cache of 32000 positions the first ends 21 us after the start, the last 30), so a span is cut again: from
// 8 tiles on a quarter is left for later and a sixteenth of it (a tile at least) for last, from 4 on a quarter; below that it is one piece.
// The CTAs take first the large pieces, then, as they get free, the small ones.  (Small pieces at the list's end instead leave the last
// segment with hundreds of parts.)  Pieces are numbered along the list, and the part of piece u that lies in segment s goes to slot u + s (from
// one part to the next either number grows, so no two share a slot).
constexpr int kSaLevels = 3;
__host__ __device__ inline int shared_levels(int each) { return each >= 8 ? 3 : each >= 4 ? 2 : 1; }         // pieces of a span, none of them empty
struct SaList {
    int p_tiles, p_total, seq_segs, p_segs, total, spans, each, more, levels;
};
__device__ __forceinline__ SaList shared_list(const SharedAttn& a, int c_tiles) {      // c_tiles: tiles of all sequences' lengths
    SaList s;
    s.p_tiles = a.p_groups ? ceil_div(a.prefix, kSaTok) : 0;
    s.p_segs = a.p_groups * a.n_kv;
    s.seq_segs = a.c_groups * a.n_kv;
    s.p_total = s.p_tiles * s.p_segs;
    s.total = s.p_total + c_tiles * s.seq_segs;
    s.spans = max(min(s.total, a.ctas), 1);
    s.each = s.total / s.spans;
    s.more = s.total - s.each * s.spans;
    s.levels = shared_levels(s.each);
    return s;
}
__device__ __forceinline__ int shared_span(const SaList& s, int w) { return w >= s.spans ? s.total : w * s.each + w * s.more / s.spans; }      // w total / spans
__device__ __forceinline__ int shared_cut(const SaList& s, int tiles, int level) {       // tiles of a span before its piece `level`
    return level == 0 ? 0 : level >= s.levels ? tiles : level == 1 ? tiles - tiles / 4 : tiles - max(tiles / 16, 1);
}
// What the table says of a segment's parts; none, if it says what cannot be (the streaming kernel gave up before it wrote it).
__host__ __device__ __forceinline__ int2 shared_slots(int2 s, int n) { return s.x >= 0 && s.x <= s.y && s.y < n ? s : make_int2(0, -1); }
constexpr int64_t kSaMaxTiles = 1 << 30;

// CTAs of the streaming kernel that an SM holds.
constexpr int shared_stream_per_sm(int d, int mt) { return mt <= 2 && d <= 128 ? 2 : 1; }
// mt: tiles of 16 pairs that a CTA takes at a time, 1, 2 or 4 (1 beyond head size 128); levels: pieces of a span at most
int launch_shared_stream_bf16(const SharedAttn& a, int mt, int levels, int32_t* d_status, cudaStream_t s);
int launch_shared_stream_f16(const SharedAttn& a, int mt, int levels, int32_t* d_status, cudaStream_t s);
int launch_shared_prefix_tc(const SharedAttn& a, int dtype, int32_t* d_status, cudaStream_t s);

}  // namespace cass
