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
    int ctas, pairs;                                     // CTAs that fit the GPU; pairs of a segment, at most
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
// head); their tiles form one list of T, cut into units.  A CTA takes one unit after another, and a unit's part of segment s goes to slot
// unit + s (from one part to the next either number grows, so no two share a slot).  SMs do not get the same share of the memory's
// rate (of equal parts of one cache of 32000 positions the first ends 21 us after the start, the last 30), so the units shrink: the first
// 3/4 of the list in as many units as CTAs fit the GPU, then 3/16 and 1/16 likewise, a tile at least.
constexpr int kSaLevels = 3;
struct SaList {
    int p_tiles, p_total, seq_segs, p_segs, total, ctas;
    int tile[kSaLevels + 1], unit[kSaLevels + 1];        // first tile and first unit of every level, and the end
};
__host__ __device__ inline int shared_level_tile(int total, int level) {
    return level == 0 ? 0 : level == 1 ? (int)((int64_t)total * 3 / 4) : level == 2 ? (int)((int64_t)total * 15 / 16) : total;
}
__device__ __forceinline__ SaList shared_list(const SharedAttn& a, int c_tiles) {      // c_tiles: tiles of all sequences' lengths
    SaList s;
    s.p_tiles = a.p_groups ? ceil_div(a.prefix, kSaTok) : 0;
    s.p_segs = a.p_groups * a.n_kv;
    s.seq_segs = a.c_groups * a.n_kv;
    s.p_total = s.p_tiles * s.p_segs;
    s.total = s.p_total + c_tiles * s.seq_segs;
    s.ctas = a.ctas;
    s.tile[0] = s.unit[0] = 0;
#pragma unroll
    for (int i = 0; i < kSaLevels; ++i) {
        s.tile[i + 1] = shared_level_tile(s.total, i + 1);
        s.unit[i + 1] = s.unit[i] + min(s.tile[i + 1] - s.tile[i], a.ctas);
    }
    return s;
}
__device__ __forceinline__ int shared_first_tile(const SaList& s, int u) {             // of unit u, or the end
    int t0 = s.tile[0], t1 = s.tile[1], u0 = s.unit[0], u1 = s.unit[1];
#pragma unroll
    for (int i = 1; i < kSaLevels; ++i)
        if (u >= s.unit[i]) { t0 = s.tile[i]; t1 = s.tile[i + 1]; u0 = s.unit[i]; u1 = s.unit[i + 1]; }
    if (u >= s.unit[kSaLevels]) return s.total;
    const int w = u - u0;
    if (u1 - u0 < s.ctas) return t0 + w;                 // a tile each
    const int each = (t1 - t0) / s.ctas, more = t1 - t0 - each * s.ctas;
    return t0 + w * each + w * more / s.ctas;            // w (t1 - t0) / ctas
}
__device__ __forceinline__ int shared_unit_of(const SaList& s, int t) {                 // that tile t is in
    int t0 = s.tile[0], t1 = s.tile[1], u0 = s.unit[0], u1 = s.unit[1];
#pragma unroll
    for (int i = 1; i < kSaLevels; ++i)
        if (t >= s.tile[i]) { t0 = s.tile[i]; t1 = s.tile[i + 1]; u0 = s.unit[i]; u1 = s.unit[i + 1]; }
    const uint32_t n = (uint32_t)(u1 - u0), tiles = (uint32_t)(t1 - t0);
    if (n == tiles) return u0 + (t - t0);
    // the largest w with w tiles / n <= t - t0, rounded down: ((t - t0 + 1) n - 1) / tiles
    const uint64_t x = (uint64_t)(uint32_t)(t - t0 + 1) * n - 1;
    return u0 + (x >> 32 ? (int)(x / tiles) : (int)((uint32_t)x / tiles));
}
constexpr int64_t kSaMaxTiles = 1 << 30;

// CTAs of the streaming kernel that an SM holds.
constexpr int shared_stream_per_sm(int d, int mt) { return mt <= 2 && d <= 128 ? 2 : 1; }
// mt: tiles of 16 pairs that a CTA takes at a time, 1, 2 or 4 (1 beyond head size 128)
int launch_shared_stream_bf16(const SharedAttn& a, int mt, int units, int32_t* d_status, cudaStream_t s);
int launch_shared_stream_f16(const SharedAttn& a, int mt, int units, int32_t* d_status, cudaStream_t s);
int launch_shared_prefix_tc(const SharedAttn& a, int dtype, int32_t* d_status, cudaStream_t s);

}  // namespace cass
