// Attention of a batch behind a shared prefix.  All sequences' queries of a KV head form the rows of one product with the prefix,
// which is read once; every sequence's own cache is read by its own queries.  Both leave partial results (output, maximum, sum) that
// k_shared_merge joins; the weights that the caches' positions got follow from the scores, once the sums are known.
//
// k_shared_stream: tiles of 64 positions, K and V through a ring of asynchronous copies, both products by mma.sync (16 pairs of (row,
// query head) by 16 positions), softmax in registers with a running maximum.  What is bound by memory runs here: with up to 64 pairs
// a position's 512 bytes (head size 128) cost less time in the products than on the bus.  The positions of all segments form one list of
// tiles that the CTAs share evenly, whatever the lengths are; the lengths are read on the device.
#include <cuda_fp16.h>

#include "shared_attn.cuh"

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

__device__ __forceinline__ void cp16(void* dst, const void* src, bool there) {      // zeros where there is nothing
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm4_t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Byte of 16-byte vector c of a row in shared memory: eight rows' vectors of one column lie in different banks.
template <int D>
__device__ __forceinline__ uint32_t sa_at(int row, int c) {
    return (uint32_t)(row * D * 2 + ((D % 64 == 0 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4));
}

template <int D, int MT>
struct SaShape {
    static constexpr int warps = MT == 4 ? 8 : 4;
    static constexpr int groups = warps / MT;            // of positions: a warp takes 64 / groups of a tile's
    static constexpr int tok = kSaTok / groups;
    static constexpr int pairs = 16 * MT;
    static constexpr bool q_regs = D <= 128;             // Q in registers from a segment's first tile on
    static constexpr int stages = MT == 4 ? 5 : 3;
    static constexpr int q_bufs = q_regs ? stages - 1 : stages;      // segments that begin in the tiles under way
    static constexpr int stage_bytes = kSaTok * D * 2 * 2;
    static constexpr int q_bytes = pairs * D * 2;
    static constexpr int smem = stages * stage_bytes + q_bufs * q_bytes;
    static constexpr int per_sm = smem + 1024 + 512 <= 233472 / 2 ? 2 : 1;
    static_assert((groups - 1) * MT * 64 * D <= stage_bytes, "the joining of a segment's warps fits a stage");
};

// One segment of the list as a worker sees it.
struct SaSegment {
    int index, head, first, seq, n;                      // number; KV head; first pair; sequence (-1: prefix); positions
    int64_t begin, end;                                  // tiles of the list
};

template <int DT, int D, int MT>
__global__ void __launch_bounds__(SaShape<D, MT>::warps * 32) k_shared_stream(SharedAttn a) {
    using S = SaShape<D, MT>;
    using T = SaType<DT>;
    constexpr int kThreads = S::warps * 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t s_scan[S::warps];
    __shared__ float s_ml[S::groups][S::pairs][2];
    __shared__ int s_seq, s_before;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, mt = warp % MT, grp = warp / MT;
    uint8_t* sQ = smem + S::stages * S::stage_bytes;
    pdl_wait();
    pdl_early<2>();

    // ---- the list: tiles of the prefix, then of the sequences ----
    const int p_tiles = a.p_groups ? ceil_div(a.prefix, kSaTok) : 0, seq_segs = a.c_groups * a.n_kv, p_segs = a.p_groups * a.n_kv;
    const int64_t p_total = (int64_t)p_tiles * p_segs;
    constexpr int kPer = kSaMaxSeq / kThreads;   // sequences a thread counts, in order
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = tid * kPer + i;
        if (b < a.n_seq) mine += ceil_div(max(shared_len(a, b), 0), kSaTok);
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) s_scan[warp] = upto;
    if (tid == 0) { s_seq = a.n_seq; s_before = 0; }
    __syncthreads();
    int64_t c_tiles = 0, ahead = upto - mine;
#pragma unroll
    for (int w = 0; w < S::warps; ++w) {
        if (w < warp) ahead += s_scan[w];
        c_tiles += s_scan[w];
    }
    const int64_t total = p_total + c_tiles * seq_segs;
    const int workers = shared_workers(total, a.ctas);
    if ((int)blockIdx.x >= workers) return;
    const int64_t t0 = shared_first_tile(total, workers, blockIdx.x), t1 = shared_first_tile(total, workers, blockIdx.x + 1);
    // the sequence that the first tile falls into (if it is none of the prefix's), found by the thread that counted it
    if (t0 >= p_total) {
        const int64_t at = (t0 - p_total) / seq_segs;    // in tiles of sequences: a sequence's segments are equally long
        if (at >= ahead && at < ahead + mine) {
            int64_t before = ahead;
            for (int i = 0; i < kPer; ++i) {
                const int b = tid * kPer + i, n = b < a.n_seq ? ceil_div(max(shared_len(a, b), 0), kSaTok) : 0;
                if (at < before + n) { s_seq = b; s_before = (int)before; break; }
                before += n;
            }
        }
    }
    __syncthreads();

    auto first_of_seq = [&](SaSegment& g, int b, int64_t begin) {     // segment 0 of the first sequence >= b that has tiles
        int n = 0;
        for (; b < a.n_seq; ++b) {
            n = shared_len(a, b);
            if (n > 0) break;
        }
        g.seq = b; g.n = n; g.index = p_segs + b * seq_segs; g.head = 0; g.first = 0;
        g.begin = begin; g.end = begin + ceil_div(n, kSaTok);
    };
    auto next = [&](SaSegment& g) {
        if (++g.head == a.n_kv) { g.head = 0; g.first += S::pairs; }
        ++g.index;
        if (g.seq < 0) {
            if (g.index == p_segs) { first_of_seq(g, 0, g.end); return; }
        } else if ((g.index - p_segs) % seq_segs == 0) {
            first_of_seq(g, g.seq + 1, g.end);
            return;
        }
        const int64_t len = g.end - g.begin;
        g.begin = g.end;
        g.end += len;
    };
    SaSegment cur;
    if (t0 < p_total) {
        const int i = (int)(t0 / p_tiles);
        cur = {i, i % a.n_kv, i / a.n_kv * S::pairs, -1, a.prefix, (int64_t)i * p_tiles, (int64_t)(i + 1) * p_tiles};
    } else {
        first_of_seq(cur, s_seq, p_total + (int64_t)s_before * seq_segs);
        const int64_t len = cur.end - cur.begin;
        const int i = (int)((t0 - cur.begin) / len);     // its segment
        cur.index += i; cur.head = i % a.n_kv; cur.first = i / a.n_kv * S::pairs;
        cur.begin += i * len; cur.end += i * len;
    }

    // ---- copies: tile t of segment g into its stage, the segment's Q with the first of its tiles here ----
    SaSegment ld = cur;
    int ld_segs = 0;                                     // segments begun by the copies
    auto pairs_of = [&](const SaSegment& g) { return (g.seq < 0 ? a.n_seq : 1) * a.rows * a.group; };
    auto q_row = [&](const SaSegment& g, int p) {        // query of pair p of the segment's sequences
        const int r = p / a.group, hq = g.head * a.group + p - r * a.group;
        return a.q + (g.seq < 0 ? (int64_t)(r / a.rows) * a.q_seq + (int64_t)(r % a.rows) * a.q_row : (int64_t)g.seq * a.q_seq + (int64_t)r * a.q_row) +
               (int64_t)hq * a.q_head;
    };
    auto load = [&](int64_t t) {
        if (t < t1) {
            if (t >= ld.end) next(ld);
            if (t == t0 || t == ld.begin) {
                uint8_t* to = sQ + (ld_segs % S::q_bufs) * S::q_bytes;
                const int P = pairs_of(ld);
                for (int i = tid; i < S::pairs * (D / 8); i += kThreads) {
                    const int p = i / (D / 8), c = i % (D / 8);
                    const bool there = ld.first + p < P;
                    cp16(to + sa_at<D>(p, c), there ? q_row(ld, ld.first + p) + c * 8 : a.q, there);
                }
                ++ld_segs;
            }
            uint8_t* to = smem + (int)((t - t0) % S::stages) * S::stage_bytes;
            const int pos0 = (int)(t - ld.begin) * kSaTok;
            const uint16_t *k, *v;
            int64_t stride;
            if (ld.seq < 0) { k = a.kp + ld.head * a.p_head; v = a.vp + ld.head * a.p_head; stride = a.p_pos; }
            else {
                const int64_t o = ld.seq * a.c_seq + ld.head * a.c_head;
                k = a.kc + o; v = a.vc + o; stride = a.c_pos;
            }
#pragma unroll 4
            for (int i = tid; i < kSaTok * (D / 8); i += kThreads) {
                const int p = i / (D / 8), c = i % (D / 8);
                const bool there = pos0 + p < ld.n;
                const int64_t o = there ? (int64_t)(pos0 + p) * stride + c * 8 : 0;
                cp16(to + sa_at<D>(p, c), k + o, there);
                cp16(to + kSaTok * D * 2 + sa_at<D>(p, c), v + o, there);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < S::stages - 1; ++i) load(t0 + i);

    // ---- products ----
    float o[D / 8][4], m[2], l[2];
    uint32_t qf[S::q_regs ? D / 16 : 1][4];
    int lim[2], cur_segs = 0;                            // positions that this thread's two rows see
    const int row = lane >> 2, col = 2 * (lane & 3);
    for (int64_t t = t0; t < t1; ++t) {
        asm volatile("cp.async.wait_group %0;" ::"n"(S::stages - 2) : "memory");
        __syncthreads();
        const uint32_t sK = smem_u32(smem + (int)((t - t0) % S::stages) * S::stage_bytes), sV = sK + kSaTok * D * 2;
        if (t >= cur.end) { next(cur); ++cur_segs; }
        const uint32_t q_at = smem_u32(sQ + (cur_segs % S::q_bufs) * S::q_bytes);
        const int q_r = mt * 16 + (lane & 15), q_c = lane >> 4;
        if (t == t0 || t == cur.begin) {
            if (S::q_regs) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) ldm4(qf[k], q_at + sa_at<D>(q_r, 2 * k + q_c));
                __syncthreads();                         // its buffer may be filled again
            }
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[i] = -INFINITY;
                l[i] = 0.f;
                const int p = cur.first + mt * 16 + row + 8 * i;
                lim[i] = p >= pairs_of(cur) ? 0 : cur.seq < 0 ? a.prefix : cur.n - (a.rows - 1 - p / a.group);
            }
        }
        load(t + S::stages - 1);                         // into the stage that was read before the barrier
        const int pos0 = (int)(t - cur.begin) * kSaTok + grp * S::tok;         // this warp's first position
        float s[S::tok / 8][4];
#pragma unroll
        for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[j][i] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            uint32_t q[4];
            if (S::q_regs) {
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = qf[k][i];
            } else {
                ldm4(q, q_at + sa_at<D>(q_r, 2 * k + q_c));
            }
#pragma unroll
            for (int j = 0; j < S::tok / 16; ++j) {
                uint32_t b[4];                           // positions 0-7 and 8-15, eight dims each twice
                ldm4(b, sK + sa_at<D>(grp * S::tok + j * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
                T::mma(s[2 * j], q, b[0], b[1]);
                T::mma(s[2 * j + 1], q, b[2], b[3]);
            }
        }
        const bool cut = pos0 + S::tok > min(lim[0], lim[1]);
#pragma unroll
        for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[j][i] *= a.scale_log2;
                if (cut && pos0 + j * 8 + col + (i & 1) >= lim[i >> 1]) s[j][i] = -INFINITY;
            }
        if (a.scores && cur.seq >= 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = cur.first + mt * 16 + row + 8 * i;
                if (p >= a.rows * a.group) continue;
                float* to = a.scores + (((int64_t)cur.seq * a.n_kv + cur.head) * a.rows * a.group + p) * a.capacity;
#pragma unroll
                for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int pos = pos0 + j * 8 + col + e;
                        if (pos < cur.n) to[pos] = s[j][2 * i + e];
                    }
            }
        }
        float base[2], fix[2];
        bool grew = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x = m[i];
#pragma unroll
            for (int j = 0; j < S::tok / 8; ++j) x = fmaxf(x, fmaxf(s[j][2 * i], s[j][2 * i + 1]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            base[i] = x == -INFINITY ? 0.f : x;
            fix[i] = exp2_fast(m[i] - base[i]);
            grew |= x != m[i];
            m[i] = x;
        }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] *= fix[j >> 1];
            l[0] *= fix[0];
            l[1] *= fix[1];
        }
#pragma unroll
        for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[j][i] = exp2_fast(s[j][i] - base[i >> 1]);
                l[i >> 1] += s[j][i];
            }
        // Positions that some of the warp's rows do not see: what is no number in their V must not meet a 0 of P in the product.
        // It is taken out there and added, for the rows that see it, one by one.
        const int seen_by_all = cur.seq < 0 ? a.prefix : cur.n - (a.rows - 1);
        const bool guard = pos0 + S::tok > seen_by_all && pos0 < cur.n && a.rows > 1 && cur.seq >= 0;
#pragma unroll
        for (int j = 0; j < S::tok / 16; ++j) {
            const uint32_t p[4] = {T::pack(s[2 * j][0], s[2 * j][1]), T::pack(s[2 * j][2], s[2 * j][3]), T::pack(s[2 * j + 1][0], s[2 * j + 1][1]),
                                   T::pack(s[2 * j + 1][2], s[2 * j + 1][3])};
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                uint32_t b[4];                           // dims 0-7 (16 positions), dims 8-15
                ldm4_t(b, sV + sa_at<D>(grp * S::tok + j * 16 + (lane & 15), 2 * n + (lane >> 4)));
                if (guard) {
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if ((b[i] & T::kExponent) == T::kExponent) { b[i] &= 0xFFFF0000u; odd = true; }
                        if ((b[i] >> 16 & T::kExponent) == T::kExponent) { b[i] &= 0x0000FFFFu; odd = true; }
                    }
                    if (__any_sync(0xffffffffu, odd)) {
                        for (int k = 0; k < 16; ++k) {   // position by position; p of (row, k) is in lane 4 row + (k % 8) / 2
                            const int pos = pos0 + j * 16 + k, src = (lane & ~3) | ((k & 7) >> 1);
                            float x[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const float even = __shfl_sync(0xffffffffu, k < 8 ? s[2 * j][2 * i] : s[2 * j + 1][2 * i], src);
                                const float oddp = __shfl_sync(0xffffffffu, k < 8 ? s[2 * j][2 * i + 1] : s[2 * j + 1][2 * i + 1], src);
                                x[i] = (k & 1) ? oddp : even;
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t at = sV + sa_at<D>(grp * S::tok + j * 16 + k, 2 * n + h) + col * 2;
                                uint32_t w;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at));
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const uint32_t bits = e ? w >> 16 : w & 0xFFFFu;
                                    if ((bits & T::kExponent) != T::kExponent) continue;
#pragma unroll
                                    for (int i = 0; i < 2; ++i)
                                        if (pos < lim[i]) o[2 * n + h][2 * i + e] = fmaf(x[i], T::get(bits), o[2 * n + h][2 * i + e]);
                                }
                            }
                        }
                    }
                }
                T::mma(o[2 * n], p, b[0], b[1]);
                T::mma(o[2 * n + 1], p, b[2], b[3]);
            }
        }
        // ---- the segment's end, or the worker's: join the warps' positions, through the stage that was read last ----
        if (t + 1 == t1 || t + 1 == cur.end) {
            __syncthreads();
            float* box = reinterpret_cast<float*>(smem + (int)((t - t0) % S::stages) * S::stage_bytes);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                if ((lane & 3) == 0) {
                    s_ml[grp][mt * 16 + row + 8 * i][0] = m[i];
                    s_ml[grp][mt * 16 + row + 8 * i][1] = l[i];
                }
            }
            if (grp > 0) {
                float4* to = reinterpret_cast<float4*>(box) + ((grp - 1) * MT + mt) * (D / 8) * 32 + lane;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) to[i * 32] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
            }
            __syncthreads();
            if (grp == 0) {
                float all[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f}, w[S::groups][2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int p = mt * 16 + row + 8 * i;
#pragma unroll
                    for (int g = 0; g < S::groups; ++g) all[i] = fmaxf(all[i], s_ml[g][p][0]);
                    const float b = all[i] == -INFINITY ? 0.f : all[i];
#pragma unroll
                    for (int g = 0; g < S::groups; ++g) {
                        w[g][i] = exp2_fast(s_ml[g][p][0] - b);
                        sum[i] += w[g][i] * s_ml[g][p][1];
                    }
                }
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i][j] *= w[0][j >> 1];
#pragma unroll
                for (int g = 1; g < S::groups; ++g) {
                    const float4* from = reinterpret_cast<const float4*>(box) + ((g - 1) * MT + mt) * (D / 8) * 32 + lane;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        const float4 x = from[i * 32];
                        o[i][0] = fmaf(w[g][0], x.x, o[i][0]);
                        o[i][1] = fmaf(w[g][0], x.y, o[i][1]);
                        o[i][2] = fmaf(w[g][1], x.z, o[i][2]);
                        o[i][3] = fmaf(w[g][1], x.w, o[i][3]);
                    }
                }
                const int64_t slot = (int64_t)blockIdx.x + cur.index;
                const int P = min(pairs_of(cur) - cur.first, S::pairs);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int p = mt * 16 + row + 8 * i;
                    if (p >= P) continue;
                    float* to = a.part_o + (slot * a.pairs + p) * D + col;
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(to + j * 8) = make_float2(o[j][2 * i], o[j][2 * i + 1]);
                    if ((lane & 3) == 0) {
                        a.part_m[slot * a.pairs + p] = all[i];
                        a.part_l[slot * a.pairs + p] = sum[i];
                    }
                }
            }
        }
    }
}

// ---- joining the parts ----
constexpr int kSmThreads = 128, kSmWarps = kSmThreads / 32;
constexpr int kSmMaxParts = 4 * kSms;                // of a pair: at most every CTA's of either kernel, and two a CTA of the tensor-core kernel's
constexpr int kSmPos = 4 * kSmThreads;                   // positions of a weights block

// Where the parts of (sequence b, head, pair p of the sequence) lie: those of the prefix, then those of its cache, in order.
struct SaParts {
    int64_t pre0, pre_step, own0;                        // first place, distance of two, in pairs
    int n_pre, n_own, own_step;
    bool pre_tc;
    __device__ __forceinline__ int count() const { return n_pre + n_own; }
};

__device__ SaParts shared_parts(const SharedAttn& a, int seg_pairs, int b, int head, int p, int tiles_before, int64_t c_tiles, int n) {
    SaParts r{};
    const int p_tiles = a.p_groups ? ceil_div(a.prefix, kSaTok) : 0, seq_segs = a.c_groups * a.n_kv, p_segs = a.p_groups * a.n_kv;
    const int64_t p_total = (int64_t)p_tiles * p_segs, total = p_total + c_tiles * seq_segs;
    const int workers = shared_workers(total, a.ctas);
    const int P = a.rows * a.group, all = b * P + p;     // the pair among those of all sequences
    if (p_tiles) {
        const int s = all / seg_pairs * a.n_kv + head;
        const int w0 = shared_worker_of(total, workers, (int64_t)s * p_tiles), w1 = shared_worker_of(total, workers, (int64_t)(s + 1) * p_tiles - 1);
        r.pre0 = (int64_t)(w0 + s) * a.pairs + all % seg_pairs;
        r.pre_step = a.pairs;
        r.n_pre = w1 - w0 + 1;
    } else if (a.prefix) {
        const int cta = all / (2 * kStTile);
        r.pre_tc = true;
        if (cta < a.pre_n2) {
            r.pre0 = ((int64_t)head * a.pre_n2 + cta) * 2 * kStTile + all % (2 * kStTile);
            r.pre_step = (int64_t)a.n_kv * a.pre_n2 * 2 * kStTile;
            r.n_pre = a.pre_s2;
        } else {
            r.pre0 = a.pre_at1 + (int64_t)head * kStTile + all % (2 * kStTile);
            r.pre_step = (int64_t)a.n_kv * kStTile;
            r.n_pre = 2 * a.pre_s1;
        }
    }
    const int tiles = ceil_div(max(n, 0), kSaTok);
    if (tiles) {
        const int k = p / seg_pairs * a.n_kv + head;
        const int64_t first = p_total + (int64_t)tiles_before * seq_segs + (int64_t)k * tiles;
        const int w0 = shared_worker_of(total, workers, first), w1 = shared_worker_of(total, workers, first + tiles - 1);
        r.own0 = (int64_t)(w0 + p_segs + b * seq_segs + k) * a.pairs + p % seg_pairs;
        r.own_step = a.pairs;
        r.n_own = w1 - w0 + 1;
    }
    return r;
}

// grid: blocks of the (sequence, row, query head)s, WARPS warps each, then (with weights) one for every 512 positions of every (sequence, KV
// head).  A warp a pair where there are many pairs, four where there are few with many parts.
template <int DT, int WARPS>
__global__ void __launch_bounds__(kSmThreads) k_shared_merge(SharedAttn a, int seg_pairs, int pair_blocks, int pos_blocks, uint16_t* __restrict__ out,
                                                             float* __restrict__ lse, const float* weight_in, float* weight_out,
                                                             int32_t* __restrict__ d_status) {
    using T = SaType<DT>;
    __shared__ float s_w[kSmWarps][kSmMaxParts];
    __shared__ __align__(16) float s_o[kSmWarps][256];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_early<3>();
    const int P = a.rows * a.group;
    const bool weights = (int)blockIdx.x >= pair_blocks;
    int b, head, p = 0, r = 0, hq = 0, chunk = 0;
    if (weights) {
        int i = blockIdx.x - pair_blocks;
        chunk = i % pos_blocks; i /= pos_blocks;
        head = i % a.n_kv; b = i / a.n_kv;
    } else {
        const int i = blockIdx.x * (kSmWarps / WARPS) + warp / WARPS;
        hq = i % a.n_q; r = i / a.n_q % a.rows; b = i / a.n_q / a.rows;
        if (b >= a.n_seq) return;
        head = hq / a.group; p = r * a.group + hq % a.group;
    }
    const int n = shared_len(a, b);
    if (n < 0) return;                                   // the sequence is not there
    int before = 0, tiles = 0;
    for (int i = lane; i < a.n_seq; i += 32) {
        const int t = ceil_div(max(shared_len(a, i), 0), kSaTok);
        tiles += t;
        before += i < b ? t : 0;
    }
    before = __reduce_add_sync(0xffffffffu, before);
    tiles = __reduce_add_sync(0xffffffffu, tiles);

    // maximum of all parts and their sum relative to it, by a warp; w: the parts' factors, 2^(m - M)
    auto sums = [&](const SaParts& s, float* w, float& M, float& L) {
        const float *pm = s.pre_tc ? a.pre_m : a.part_m, *pl = s.pre_tc ? a.pre_l : a.part_l;
        const int count = s.count();
        float m0 = -INFINITY, l0 = 0.f;                  // of the first 32, one round trip
        auto load = [&](int i, float& m, float& l) {
            if (i < s.n_pre) { m = pm[s.pre0 + i * s.pre_step]; l = pl[s.pre0 + i * s.pre_step]; }
            else { const int64_t at = s.own0 + (int64_t)(i - s.n_pre) * s.own_step; m = a.part_m[at]; l = a.part_l[at]; }
        };
        if (lane < count) load(lane, m0, l0);
        M = m0;
        for (int i = lane + 32; i < count; i += 32) {
            float m, l;
            load(i, m, l);
            M = fmaxf(M, m);
        }
        M = warp_max(M);
        const float base = M == -INFINITY ? 0.f : M;
        const float f0 = exp2_fast(m0 - base);
        L = f0 * l0;
        if (w && lane < count) w[lane] = f0;
        for (int i = lane + 32; i < count; i += 32) {
            float m, l;
            load(i, m, l);
            const float f = exp2_fast(m - base);
            L += f * l;
            if (w) w[i] = f;
        }
        L = warp_sum(L);
        __syncwarp();
    };
    if (weights) {
        const int pos0 = chunk * kSmPos;
        const float* in = weight_in ? weight_in + ((int64_t)b * a.n_kv + head) * a.capacity : nullptr;
        float* to = weight_out + ((int64_t)b * a.n_kv + head) * a.capacity;
        float* s_lse = &s_w[0][0];
        if (pos0 < n) {
            for (int q = warp; q < P; q += kSmWarps) {
                float M, L;
                sums(shared_parts(a, seg_pairs, b, head, q, before, tiles, n), nullptr, M, L);
                if (lane == 0) s_lse[q] = M + log2f(L);
            }
            __syncthreads();
        }
        const float* from = a.scores + ((int64_t)b * a.n_kv + head) * P * a.capacity;
#pragma unroll
        for (int i = 0; i < kSmPos / kSmThreads; ++i) {
            const int pos = pos0 + i * kSmThreads + tid;
            if (pos >= a.capacity) break;
            float sum = 0.f;
            for (int q = 0; q < a.rows; ++q) {
                if (pos >= n - (a.rows - 1 - q)) continue;
                for (int g = 0; g < a.group; ++g) sum += exp2_fast(from[(int64_t)(q * a.group + g) * a.capacity + pos] - s_lse[q * a.group + g]);
            }
            if (pos < n || in != to) to[pos] = (in ? in[pos] : 0.f) + sum;
        }
        return;
    }
    if (p == 0 && head == 0 && warp % WARPS == 0 && lane == 0 && a.lens && a.lens[b] > a.capacity) atomicCAS(d_status, 0, CASS_ERR_CAPACITY);
    const SaParts s = shared_parts(a, seg_pairs, b, head, p, before, tiles, n);
    const int parts = s.count();
    float M, L, *w = s_w[warp];
    sums(s, w, M, L);                                    // each of the pair's warps for itself
    const float* po = s.pre_tc ? a.pre_o : a.part_o;
    const bool sees = a.prefix > 0 || n - (a.rows - 1 - r) > 0;
    uint16_t* to = out + (int64_t)b * a.out_seq + (int64_t)r * a.out_row + (int64_t)hq * a.out_head;
    auto put = [&](int c, float4 x) {
        const uint32_t lo = T::put(sees ? x.x / L : 0.f) | ((uint32_t)T::put(sees ? x.y / L : 0.f) << 16);
        const uint32_t hi = T::put(sees ? x.z / L : 0.f) | ((uint32_t)T::put(sees ? x.w / L : 0.f) << 16);
        *reinterpret_cast<uint2*>(to + c) = make_uint2(lo, hi);
    };
    for (int c = lane * 4; c < a.d; c += 128) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int i = warp % WARPS; i < parts; i += WARPS) {
            const float* from = i < s.n_pre ? po + (s.pre0 + i * s.pre_step) * a.d : a.part_o + (s.own0 + (int64_t)(i - s.n_pre) * s.own_step) * a.d;
            const float4 x = *reinterpret_cast<const float4*>(from + c);
            const float f = w[i];
            sum.x = fmaf(f, x.x, sum.x); sum.y = fmaf(f, x.y, sum.y); sum.z = fmaf(f, x.z, sum.z); sum.w = fmaf(f, x.w, sum.w);
        }
        if (WARPS == 1) put(c, sum);
        else *reinterpret_cast<float4*>(&s_o[warp][c]) = sum;
    }
    if (WARPS > 1) {
        __syncthreads();
        if (warp == 0)
            for (int c = lane * 4; c < a.d; c += 128) {
                float4 x = *reinterpret_cast<const float4*>(&s_o[0][c]);
#pragma unroll
                for (int i = 1; i < WARPS; ++i) {
                    const float4 y = *reinterpret_cast<const float4*>(&s_o[i][c]);
                    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                }
                put(c, x);
            }
    }
    if (lse && warp % WARPS == 0 && lane == 0) lse[((int64_t)b * a.rows + r) * a.n_q + hq] = sees ? (M + log2f(L)) * 0.693147180559945309f : -INFINITY;
}

// ---- host ----

struct SaPlan {
    SharedAttn a;
    int mt, per_sm;
    bool tc;
    size_t at_o, at_m, at_l, at_scores, at_pre_o, at_pre_m, at_pre_l, bytes;
};

constexpr int kSmManyPairs = 4 * kSms;                   // joined by a warp each
constexpr int kSaStreamPairs = 64;                       // pairs behind a prefix up to which it is streamed

static bool head_dim_ok(int d) { return d == 32 || d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }

static int shared_plan(const cass_cache_geom* c, const cass_shared_attn* t, bool with_weights, SaPlan* plan) {
    if (!c || !t || !cache_geom_ok(*c, true)) return CASS_ERR_INVALID_ARG;
    if (t->rows < 1 || t->n_q_heads < 1 || t->prefix_len < 0 || t->n_q_heads % c->n_kv_heads) return CASS_ERR_INVALID_ARG;
    if (!(t->scale >= 0.f) || t->scale > 3e38f) return CASS_ERR_INVALID_ARG;
    const int64_t in[] = {t->q_seq, t->q_row, t->q_head, t->out_seq, t->out_row, t->out_head, t->prefix_pos_stride, t->prefix_head_stride};
    for (int64_t s : in)
        if (s < 0 || s % 8 || s > ((int64_t)1 << 46)) return CASS_ERR_INVALID_ARG;
    if ((t->prefix_len > 1 && t->prefix_pos_stride < c->head_dim) || (t->prefix_len && c->n_kv_heads > 1 && t->prefix_head_stride < c->head_dim))
        return CASS_ERR_INVALID_ARG;
    // the output's heads lie apart, as rows of a cache do: (sequence, row, head) by its strides
    cass_cache_geom o = *c;
    o.n_kv_heads = t->n_q_heads; o.capacity = t->rows; o.seq_stride = t->out_seq; o.pos_stride = t->out_row; o.head_stride = t->out_head;
    if (!cache_geom_ok(o, false)) return CASS_ERR_INVALID_ARG;
    const int group = t->n_q_heads / c->n_kv_heads;
    if (!head_dim_ok(c->head_dim) || group > 16 || t->rows > kMaxVerifyRows || c->n_seq > kSaMaxSeq || t->n_q_heads > 1024) return CASS_ERR_UNSUPPORTED;
    SharedAttn& a = plan->a;
    a = SharedAttn{};
    a.n_seq = c->n_seq; a.rows = t->rows; a.n_q = t->n_q_heads; a.n_kv = c->n_kv_heads; a.group = group; a.d = c->head_dim;
    a.prefix = t->prefix_len; a.capacity = c->capacity;
    a.q_seq = t->q_seq; a.q_row = t->q_row; a.q_head = t->q_head;
    a.out_seq = t->out_seq; a.out_row = t->out_row; a.out_head = t->out_head;
    a.p_pos = t->prefix_pos_stride; a.p_head = t->prefix_head_stride;
    a.c_seq = c->seq_stride; a.c_pos = c->pos_stride; a.c_head = c->head_stride;
    a.scale_log2 = (t->scale > 0.f ? t->scale : 1.0f / sqrtf((float)a.d)) * 1.44269504088896341f;
    const int P = a.rows * group, all = a.n_seq * P;     // pairs of a sequence, of all
    plan->tc = a.prefix && all > kSaStreamPairs && shared_tc_usable(a);
    const int most = a.prefix && !plan->tc ? (all > P ? all : P) : P;
    plan->mt = a.d > 128 || most <= 16 ? 1 : most <= 32 ? 2 : 4;
    const int seg = 16 * plan->mt;
    a.pairs = most < seg ? most : seg;
    a.p_groups = a.prefix && !plan->tc ? ceil_div(all, seg) : 0;
    a.c_groups = ceil_div(P, seg);
    plan->per_sm = plan->mt == 4 || a.d > 128 ? 1 : 2;
    a.ctas = kSms * plan->per_sm;
    size_t off = 0;
    auto take = [&](size_t b) { const size_t o2 = off; off = align_up(off + b, 256); return o2; };
    const size_t slots = (size_t)a.ctas + (size_t)a.n_kv * ((size_t)a.p_groups + (size_t)a.n_seq * a.c_groups);
    plan->at_o = take(slots * a.pairs * a.d * 4);
    plan->at_m = take(slots * a.pairs * 4);
    plan->at_l = take(slots * a.pairs * 4);
    const size_t pre = plan->tc ? (size_t)shared_tc_plan(a) : 0;
    plan->at_pre_o = take(pre * a.d * 4);
    plan->at_pre_m = take(pre * 4);
    plan->at_pre_l = take(pre * 4);
    plan->at_scores = take(with_weights ? (size_t)a.n_seq * a.n_q * a.rows * a.capacity * 4 : 0);
    plan->bytes = off < 256 ? 256 : off;
    return CASS_OK;
}

template <int DT, int D, int MT>
static int run_stream(const SharedAttn& a, cudaStream_t s) {
    using S = SaShape<D, MT>;
    CASS_ALLOW_SMEM(k_shared_stream<DT, D, MT>);
    CASS_PDL_LAUNCH((k_shared_stream<DT, D, MT>), dim3(a.ctas), dim3(S::warps * 32), (size_t)S::smem, s, a);
    return CASS_OK;
}

template <int DT, int D>
static int run_stream_d(const SharedAttn& a, int mt, cudaStream_t s) {
    if (mt == 1) return run_stream<DT, D, 1>(a, s);
    if constexpr (D <= 128) {
        if (mt == 2) return run_stream<DT, D, 2>(a, s);
        if (mt == 4) return run_stream<DT, D, 4>(a, s);
    }
    return CASS_ERR_UNSUPPORTED;
}

template <int DT>
static int run_shared(const SaPlan& plan, uint16_t* out, float* lse, const float* weight_in, float* weight_out, int32_t* d_status, cudaStream_t s) {
    const SharedAttn& a = plan.a;
    int rc = plan.tc ? launch_shared_prefix_tc(a, DT, d_status, s) : CASS_OK;
    if (rc) return rc;
    rc = CASS_ERR_UNSUPPORTED;
    switch (a.d) {
        case 32: rc = run_stream_d<DT, 32>(a, plan.mt, s); break;
        case 64: rc = run_stream_d<DT, 64>(a, plan.mt, s); break;
        case 96: rc = run_stream_d<DT, 96>(a, plan.mt, s); break;
        case 128: rc = run_stream_d<DT, 128>(a, plan.mt, s); break;
        case 192: rc = run_stream_d<DT, 192>(a, plan.mt, s); break;
        case 256: rc = run_stream_d<DT, 256>(a, plan.mt, s); break;
    }
    if (rc) return rc;
    const int pos_blocks = weight_out ? ceil_div(a.capacity, kSmPos) : 0;
    const int64_t pairs = (int64_t)a.n_seq * a.rows * a.n_q;
    const bool many = pairs >= kSmManyPairs;
    const int64_t pair_blocks = many ? (pairs + kSmWarps - 1) / kSmWarps : pairs, blocks = pair_blocks + (int64_t)a.n_seq * a.n_kv * pos_blocks;
    if (blocks > 0x7FFFFFFF) return CASS_ERR_UNSUPPORTED;
    if (many)
        CASS_PDL_LAUNCH((k_shared_merge<DT, 1>), dim3((unsigned)blocks), dim3(kSmThreads), 0, s, a, 16 * plan.mt, (int)pair_blocks, pos_blocks, out, lse,
                        weight_in, weight_out, d_status);
    else
        CASS_PDL_LAUNCH((k_shared_merge<DT, kSmWarps>), dim3((unsigned)blocks), dim3(kSmThreads), 0, s, a, 16 * plan.mt, (int)pair_blocks, pos_blocks, out,
                        lse, weight_in, weight_out, d_status);
    return CASS_OK;
}

}  // namespace cass

using namespace cass;

extern "C" size_t cass_shared_prefix_scratch_bytes(const cass_cache_geom* cache, const cass_shared_attn* attn, int with_weights) {
    SaPlan plan;
    return shared_plan(cache, attn, with_weights != 0, &plan) ? 0 : plan.bytes;
}

extern "C" int cass_shared_prefix_attention(const cass_cache_geom* cache, const cass_shared_attn* attn, const void* q, const void* k_prefix,
                                            const void* v_prefix, const void* k_cache, const void* v_cache, const int32_t* lens, void* out, float* lse,
                                            const float* weight_in, float* weight_out, void* scratch, size_t scratch_bytes, int32_t* d_status,
                                            void* stream_) {
    SaPlan plan;
    int rc = shared_plan(cache, attn, weight_out != nullptr, &plan);
    if (rc) return rc;
    SharedAttn& a = plan.a;
    if (!q || !out || !scratch || !d_status || (a.prefix && (!k_prefix || !v_prefix)) || (a.capacity && (!k_cache || !v_cache || !lens)))
        return CASS_ERR_INVALID_ARG;
    if ((weight_in && !weight_out) || (weight_out && !a.capacity)) return CASS_ERR_INVALID_ARG;
    const uintptr_t at16 = (uintptr_t)q | (uintptr_t)out | (uintptr_t)scratch | (a.prefix ? (uintptr_t)k_prefix | (uintptr_t)v_prefix : 0) |
                           (a.capacity ? (uintptr_t)k_cache | (uintptr_t)v_cache : 0);
    const uintptr_t at4 = (uintptr_t)lens | (uintptr_t)lse | (uintptr_t)weight_in | (uintptr_t)weight_out | (uintptr_t)d_status;
    if (at16 % 16 || at4 % 4) return CASS_ERR_INVALID_ARG;
    if (scratch_bytes < plan.bytes) return CASS_ERR_CAPACITY;
    uint8_t* mem = (uint8_t*)scratch;
    a.q = (const uint16_t*)q; a.kp = (const uint16_t*)k_prefix; a.vp = (const uint16_t*)v_prefix;
    a.kc = (const uint16_t*)k_cache; a.vc = (const uint16_t*)v_cache; a.lens = a.capacity ? lens : nullptr;
    a.part_o = (float*)(mem + plan.at_o); a.part_m = (float*)(mem + plan.at_m); a.part_l = (float*)(mem + plan.at_l);
    a.pre_o = (float*)(mem + plan.at_pre_o); a.pre_m = (float*)(mem + plan.at_pre_m); a.pre_l = (float*)(mem + plan.at_pre_l);
    a.scores = weight_out ? (float*)(mem + plan.at_scores) : nullptr;
    if (cache->dtype == CASS_BF16) return run_shared<CASS_BF16>(plan, (uint16_t*)out, lse, weight_in, weight_out, d_status, (cudaStream_t)stream_);
    return run_shared<CASS_F16>(plan, (uint16_t*)out, lse, weight_in, weight_out, d_status, (cudaStream_t)stream_);
}
