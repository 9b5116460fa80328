// The streaming kernel of the shared-prefix attention: a prefix behind up to 64 (sequence, row, query head) pairs, and every sequence's own
// cache.  Tiles of 64 positions come by TMA into a ring (one warp fetches, the others compute), both products run by mma.sync (16 pairs by
// 8 positions or dims), the softmax in registers with a running maximum.  What is bound by memory runs here: with few pairs a
// position's bytes cost more time on the bus than in the products.  The positions of all segments form one list of tiles that the CTAs share
// evenly, whatever the lengths are, and the lengths are read on the device.
// Fetched by every thread with 16-byte asynchronous copies instead, their addresses were half of 760 instructions a warp and tile, and
// the two warps a scheduler has needed 3900 clocks for a tile that memory brings in 2700: one cache of 32000 positions 31 us, 4.2 TB/s.
#pragma once

#include "tc.cuh"
#include "shared_attn.cuh"

namespace cass {

__device__ __forceinline__ void cp16(void* dst, const void* src, bool there) {      // zeros where there is nothing
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm4_t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* smem_dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
                     smem_u32(smem_dst)),
                 "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}

constexpr int kSaBoxPos = 32;                            // positions of a TMA box: a segment's last tile brings no more than it has to

template <int D, int MT>
struct SaShape {
    static constexpr int width = D % 64 == 0 ? 64 : 32;  // dims of a box: 128 or 64 bytes, swizzled over as many
    static constexpr int warps = MT == 1 ? 4 : 8;        // that compute; one more fetches
    static constexpr int threads = (warps + 1) * 32;
    static constexpr int groups = warps / MT;            // of positions: a warp takes 64 / groups of a tile's
    static constexpr int tok = kSaTok / groups;
    static constexpr int pairs = 16 * MT;
    static constexpr int kv_bytes = kSaTok * D * 2;      // K or V of a tile
    static constexpr int q_bytes = pairs * D * 2;        // Q travels with the first tile of a segment
    static constexpr int stage_bytes = 2 * kv_bytes + q_bytes;
    static constexpr int per_sm = MT == 1 && D <= 128 ? 2 : 1;
    static constexpr int room = per_sm == 2 ? 112 * 1024 : 225 * 1024;
    static constexpr int fit = room / stage_bytes, stages = fit < 8 ? fit : 8;
    static constexpr int smem = stages * stage_bytes + 1024;         // 1024: alignment of the swizzled boxes
    static_assert(stages >= 3, "one tile in use, two under way");
    static_assert(groups / 2 * MT * 64 * D <= 2 * kv_bytes, "the joining of a segment's warps fits a stage");
};

// Byte of 16-byte vector c of a row among a tile's (rows of `width` dims, box after box), as the swizzled copies leave them; eight rows'
// vectors of one column lie in different banks.
template <int D, int ROWS>
__device__ __forceinline__ uint32_t sa_at(int row, int c) {
    constexpr int kVecs = D % 64 == 0 ? 8 : 4;           // of a row in a box
    const int at = kVecs == 8 ? (c & 7) ^ (row & 7) : (c & 3) ^ ((row >> 1) & 3);
    return (uint32_t)((c / kVecs) * ROWS * kVecs * 16 + row * kVecs * 16 + (at << 4));
}

// One segment of the list as a worker sees it.
struct SaSegment {
    int index, head, first, seq, n;                      // number; KV head; first pair; sequence (-1: prefix); positions
    int64_t begin, end;                                  // tiles of the list
};

template <int DT, int D, int MT>
__global__ void __launch_bounds__(SaShape<D, MT>::threads, SaShape<D, MT>::per_sm)
    k_shared_stream(const __grid_constant__ CUtensorMap map_kp, const __grid_constant__ CUtensorMap map_vp, const __grid_constant__ CUtensorMap map_kc,
                    const __grid_constant__ CUtensorMap map_vc, SharedAttn a, int32_t* __restrict__ d_status) {
    using S = SaShape<D, MT>;
    using T = SaType<DT>;
    constexpr int kCount = S::warps * 32;                // threads that compute, and that count the tiles
    extern __shared__ uint8_t smem_dyn[];
    __shared__ int64_t s_scan[S::warps];
    __shared__ float s_ml[S::groups][S::pairs][2];
    __shared__ int s_seq, s_before;
    __shared__ uint64_t full[S::stages], empty[S::stages];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (tid == 0) {
        for (int i = 0; i < S::stages; ++i) { mbar_init(&full[i], 33); mbar_init(&empty[i], S::warps); }
        fence_mbar_init();
        s_seq = a.n_seq;
        s_before = 0;
    }
    pdl_wait();
    pdl_early<2>();

    // ---- the list: tiles of the prefix, then of the sequences ----
    const int p_tiles = a.p_groups ? ceil_div(a.prefix, kSaTok) : 0, seq_segs = a.c_groups * a.n_kv, p_segs = a.p_groups * a.n_kv;
    const int64_t p_total = (int64_t)p_tiles * p_segs;
    constexpr int kPer = kSaMaxSeq / kCount;              // sequences a thread counts, in order
    int mine = 0;
    if (warp < S::warps) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int b = tid * kPer + i;
            if (b < a.n_seq) mine += ceil_div(max(shared_len(a, b), 0), kSaTok);
        }
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31 && warp < S::warps) s_scan[warp] = upto;
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
    const int64_t t0 = shared_first_tile(total, workers, blockIdx.x);
    const int n_tiles = (int)(shared_first_tile(total, workers, blockIdx.x + 1) - t0);
    // the sequence that the first tile falls into (if it is none of the prefix's), found by the thread that counted it
    if (t0 >= p_total && warp < S::warps) {
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
    auto pairs_of = [&](const SaSegment& g) { return (g.seq < 0 ? a.n_seq : 1) * a.rows * a.group; };
    // Tile i of this worker is in stage i % stages.  A wait that runs out flags the status; the warp then goes on without waiting, so that
    // the barriers between the warps still meet.
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok && !mbar_wait_bounded(bar, parity)) {
            ok = false;
            atomicCAS(d_status, 0, CASS_ERR_TIMEOUT);
        }
        ok = __all_sync(0xffffffffu, ok);
    };

    if (warp == S::warps) {
        // ---- the warp that fetches ----
        int left = 0, stage = 0;
        uint32_t parity = 1;                             // of the stage's release before: the first round finds it free
        for (int i = 0; i < n_tiles; ++i) {
            const int64_t t = t0 + i;
            if (t >= cur.end) next(cur);
            wait(&empty[stage], parity);
            if (!ok) break;
            uint8_t* to = smem + stage * S::stage_bytes;
            if (i == 0 || t == cur.begin) {
                const int P = pairs_of(cur);
                for (int j = lane; j < S::pairs * (D / 8); j += 32) {
                    const int p = j / (D / 8), c = j % (D / 8), all = cur.first + p;
                    const bool there = all < P;
                    const int r = all / a.group, hq = cur.head * a.group + all - r * a.group;
                    const int64_t row = cur.seq < 0 ? (int64_t)(r / a.rows) * a.q_seq + (int64_t)(r % a.rows) * a.q_row
                                                    : (int64_t)cur.seq * a.q_seq + (int64_t)r * a.q_row;
                    cp16(to + 2 * S::kv_bytes + sa_at<D, S::pairs>(p, c), there ? a.q + row + (int64_t)hq * a.q_head + c * 8 : a.q, there);
                }
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[stage])) : "memory");
            if (lane == 0) {
                const int pos = (int)(t - cur.begin) * kSaTok, boxes = ceil_div(min(cur.n - pos, kSaTok), kSaBoxPos);
                const CUtensorMap *k = cur.seq < 0 ? &map_kp : &map_kc, *v = cur.seq < 0 ? &map_vp : &map_vc;
                mbar_expect_tx(&full[stage], boxes * (2 * kSaBoxPos * D * 2));
                for (int x = 0; x < D / S::width; ++x)
                    for (int y = 0; y < boxes; ++y) {
                        uint8_t* at = to + x * kSaTok * S::width * 2 + y * kSaBoxPos * S::width * 2;
                        tma_load_4d(at, k, x * S::width, pos + y * kSaBoxPos, cur.head, max(cur.seq, 0), &full[stage]);
                        tma_load_4d(at + S::kv_bytes, v, x * S::width, pos + y * kSaBoxPos, cur.head, max(cur.seq, 0), &full[stage]);
                    }
            }
            left = i + 1;
            if (++stage == S::stages) { stage = 0; parity ^= 1; }
        }
        if (!ok)                                         // what is in flight lands before the CTA ends (bounded)
            for (int i = max(left - S::stages, 0); i < left; ++i) mbar_wait_bounded(&full[i % S::stages], (uint32_t)(i / S::stages) & 1u);
        return;
    }

    // ---- the warps that compute ----
    const int mt = warp % MT, grp = warp / MT, row = lane >> 2, col = 2 * (lane & 3);
    const int q_r = mt * 16 + (lane & 15), q_c = lane >> 4;
    float o[D / 8][4], m[2], l[2];
    uint32_t qf[D / 16][4];                              // Q, from a segment's first tile on
    int lim[2], stage = 0;                               // positions that this thread's two rows see
    uint32_t parity = 0;
    auto sync_all = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kCount) : "memory"); };
    for (int i = 0; i < n_tiles; ++i) {
        const int64_t t = t0 + i;
        if (t >= cur.end) next(cur);
        wait(&full[stage], parity);
        uint8_t* at = smem + stage * S::stage_bytes;
        const uint32_t sK = smem_u32(at), sV = sK + S::kv_bytes, sQ = sV + S::kv_bytes;
        if (i == 0 || t == cur.begin) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) ldm4(qf[k], sQ + sa_at<D, S::pairs>(q_r, 2 * k + q_c));
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[k][j] = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                m[k] = -INFINITY;
                l[k] = 0.f;
                const int p = cur.first + mt * 16 + row + 8 * k;
                lim[k] = p >= pairs_of(cur) ? 0 : cur.seq < 0 ? a.prefix : cur.n - (a.rows - 1 - p / a.group);
            }
        }
        const int pos0 = (int)(t - cur.begin) * kSaTok + grp * S::tok;         // this warp's first position
        bool wrote = false;
        if (pos0 + S::tok > cur.n) {                     // behind the last position V is what the ring or the cache happens to hold
            for (int j = lane; j < S::tok * (D / 8); j += 32) {
                const int p = j / (D / 8);
                if (pos0 + p >= cur.n)
                    *reinterpret_cast<uint4*>(at + S::kv_bytes + sa_at<D, kSaTok>(grp * S::tok + p, j % (D / 8))) = make_uint4(0u, 0u, 0u, 0u);
            }
            wrote = true;
            __syncwarp();
        }
        float s[S::tok / 8][4];
#pragma unroll
        for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int j = 0; j < S::tok / 16; ++j) {
                uint32_t b[4];                           // positions 0-7 and 8-15, eight dims each twice
                ldm4(b, sK + sa_at<D, kSaTok>(grp * S::tok + j * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
                T::mma(s[2 * j], qf[k], b[0], b[1]);
                T::mma(s[2 * j + 1], qf[k], b[2], b[3]);
            }
        if (pos0 + S::tok > min(lim[0], lim[1])) {
#pragma unroll
            for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (pos0 + j * 8 + col + (e & 1) >= lim[e >> 1]) s[j][e] = -INFINITY;
        }
        if (a.scores && cur.seq >= 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int p = cur.first + mt * 16 + row + 8 * k;
                if (p >= a.rows * a.group) continue;
                float* to = a.scores + (((int64_t)cur.seq * a.n_kv + cur.head) * a.rows * a.group + p) * a.score_stride;
#pragma unroll
                for (int j = 0; j < S::tok / 8; ++j) {
                    const int pos = pos0 + j * 8 + col;  // even, as the stride is
                    if (pos < cur.n) *reinterpret_cast<float2*>(to + pos) = make_float2(s[j][2 * k] * a.scale_log2, s[j][2 * k + 1] * a.scale_log2);
                }
            }
        }
        float base[2], fix[2];
        bool grew = false;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float x = s[0][2 * k];
#pragma unroll
            for (int j = 0; j < S::tok / 8; ++j) x = fmaxf(x, fmaxf(s[j][2 * k], s[j][2 * k + 1]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            x = fmaxf(m[k], x * a.scale_log2);           // (the scale is positive)
            base[k] = x == -INFINITY ? 0.f : x;
            fix[k] = exp2_fast(m[k] - base[k]);
            grew |= x != m[k];
            m[k] = x;
        }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[k][j] *= fix[j >> 1];
            l[0] *= fix[0];
            l[1] *= fix[1];
        }
#pragma unroll
        for (int j = 0; j < S::tok / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[j][e] = exp2_fast(fmaf(s[j][e], a.scale_log2, -base[e >> 1]));
                l[e >> 1] += s[j][e];
            }
        // Positions that some of the sequence's rows do not see: what is no number in their V must not meet a 0 of P in the product.
        // It is taken out there and added, for the rows that see it, one by one.
        const bool guard = cur.seq >= 0 && a.rows > 1 && pos0 + S::tok > cur.n - (a.rows - 1) && pos0 < cur.n;
#pragma unroll
        for (int j = 0; j < S::tok / 16; ++j) {
            const uint32_t p[4] = {T::pack(s[2 * j][0], s[2 * j][1]), T::pack(s[2 * j][2], s[2 * j][3]), T::pack(s[2 * j + 1][0], s[2 * j + 1][1]),
                                   T::pack(s[2 * j + 1][2], s[2 * j + 1][3])};
            const int v_r = grp * S::tok + j * 16;
            auto outputs = [&](auto guarded) {
#pragma unroll
                for (int n = 0; n < D / 16; ++n) {
                    uint32_t b[4];                       // dims 0-7 (16 positions), dims 8-15
                    ldm4_t(b, sV + sa_at<D, kSaTok>(v_r + (lane & 15), 2 * n + (lane >> 4)));
                    if (decltype(guarded)::value) {
                        bool odd = false;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if ((b[e] & T::kExponent) == T::kExponent) { b[e] &= 0xFFFF0000u; odd = true; }
                            if ((b[e] >> 16 & T::kExponent) == T::kExponent) { b[e] &= 0x0000FFFFu; odd = true; }
                        }
                        if (__any_sync(0xffffffffu, odd)) {
                            for (int k = 0; k < 16; ++k) {           // position by position; p of (row, k) is in lane 4 row + (k % 8) / 2
                                const int pos = pos0 + j * 16 + k, src = (lane & ~3) | ((k & 7) >> 1);
                                float x[2];
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const float x0 = __shfl_sync(0xffffffffu, k < 8 ? s[2 * j][2 * e] : s[2 * j + 1][2 * e], src);
                                    const float x1 = __shfl_sync(0xffffffffu, k < 8 ? s[2 * j][2 * e + 1] : s[2 * j + 1][2 * e + 1], src);
                                    x[e] = (k & 1) ? x1 : x0;
                                }
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const uint32_t w = *reinterpret_cast<const uint32_t*>(at + S::kv_bytes + sa_at<D, kSaTok>(v_r + k, 2 * n + h) + col * 2);
#pragma unroll
                                    for (int c = 0; c < 2; ++c) {
                                        const uint32_t bits = c ? w >> 16 : w & 0xFFFFu;
                                        if ((bits & T::kExponent) != T::kExponent) continue;
#pragma unroll
                                        for (int e = 0; e < 2; ++e)
                                            if (pos < lim[e]) o[2 * n + h][2 * e + c] = fmaf(x[e], T::get(bits), o[2 * n + h][2 * e + c]);
                                    }
                                }
                            }
                        }
                    }
                    T::mma(o[2 * n], p, b[0], b[1]);
                    T::mma(o[2 * n + 1], p, b[2], b[3]);
                }
            };
            if (guard) outputs(std::true_type{});
            else outputs(std::false_type{});
        }
        // ---- the segment's end, or the worker's: the warps' positions are joined, through the stage that was read last ----
        if (i + 1 == n_tiles || t + 1 == cur.end) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
                l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
                if ((lane & 3) == 0) {
                    s_ml[grp][mt * 16 + row + 8 * k][0] = m[k];
                    s_ml[grp][mt * 16 + row + 8 * k][1] = l[k];
                }
            }
            sync_all();
            float all[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int p = mt * 16 + row + 8 * k;
#pragma unroll
                for (int g = 0; g < S::groups; ++g) all[k] = fmaxf(all[k], s_ml[g][p][0]);
                const float b = all[k] == -INFINITY ? 0.f : all[k];
#pragma unroll
                for (int g = 0; g < S::groups; ++g) sum[k] += exp2_fast(s_ml[g][p][0] - b) * s_ml[g][p][1];
                fix[k] = exp2_fast(m[k] - b);
            }
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[k][j] *= fix[j >> 1];
#pragma unroll
            for (int half = S::groups / 2; half > 0; half /= 2) {
                float4* box = reinterpret_cast<float4*>(at) + lane;
                if (grp >= half && grp < 2 * half) {
#pragma unroll
                    for (int k = 0; k < D / 8; ++k)
                        box[(((grp - half) * MT + mt) * (D / 8) + k) * 32] = make_float4(o[k][0], o[k][1], o[k][2], o[k][3]);
                }
                sync_all();
                if (grp < half) {
#pragma unroll
                    for (int k = 0; k < D / 8; ++k) {
                        const float4 x = box[((grp * MT + mt) * (D / 8) + k) * 32];
                        o[k][0] += x.x; o[k][1] += x.y; o[k][2] += x.z; o[k][3] += x.w;
                    }
                }
                if (half > 1) sync_all();
            }
            wrote = true;
            if (grp == 0) {
                const int64_t slot = (int64_t)blockIdx.x + cur.index;
                const int P = min(pairs_of(cur) - cur.first, S::pairs);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int p = mt * 16 + row + 8 * k;
                    if (p >= P) continue;
                    float* to = a.part_o + (slot * a.pairs + p) * D + col;
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(to + j * 8) = make_float2(o[j][2 * k], o[j][2 * k + 1]);
                    if ((lane & 3) == 0) {
                        a.part_m[slot * a.pairs + p] = all[k];
                        a.part_l[slot * a.pairs + p] = sum[k];
                    }
                }
            }
        }
        if (wrote) fence_proxy_async();                  // the next copy into the stage comes behind these writes
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&empty[stage])) : "memory");
        if (++stage == S::stages) { stage = 0; parity ^= 1; }
    }
}

// K or V as [sequence][head][position][dim], whatever the order in memory, in boxes of 32 positions.
inline int shared_cache_map(CUtensorMap* map, const uint16_t* at, int d, int positions, int heads, int seqs, int64_t pos, int64_t head, int64_t seq) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return CASS_ERR_CUDA;
    const int width = d % 64 == 0 ? 64 : 32;
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)positions, (cuuint64_t)heads, (cuuint64_t)seqs};
    const cuuint64_t strides[3] = {(cuuint64_t)(positions > 1 ? pos : d) * 2, (cuuint64_t)(heads > 1 ? head : d) * 2, (cuuint64_t)(seqs > 1 ? seq : d) * 2};
    const cuuint32_t box[4] = {(cuuint32_t)width, kSaBoxPos, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<uint16_t*>(at), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          width == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CASS_OK : CASS_ERR_INVALID_ARG;
}

template <int DT, int D, int MT>
int run_shared_stream(const SharedAttn& a, const CUtensorMap* maps, int32_t* d_status, cudaStream_t s) {
    using S = SaShape<D, MT>;
    CASS_ALLOW_SMEM(k_shared_stream<DT, D, MT>);
    CASS_PDL_LAUNCH((k_shared_stream<DT, D, MT>), dim3(a.ctas), dim3(S::threads), (size_t)S::smem, s, maps[0], maps[1], maps[2], maps[3], a, d_status);
    return CASS_OK;
}

template <int DT, int D>
int run_shared_stream_d(const SharedAttn& a, int mt, const CUtensorMap* maps, int32_t* d_status, cudaStream_t s) {
    if (mt == 1) return run_shared_stream<DT, D, 1>(a, maps, d_status, s);
    if constexpr (D <= 128) {
        if (mt == 2) return run_shared_stream<DT, D, 2>(a, maps, d_status, s);
        if (mt == 4) return run_shared_stream<DT, D, 4>(a, maps, d_status, s);
    }
    return CASS_ERR_UNSUPPORTED;
}

template <int DT>
int launch_shared_stream(const SharedAttn& a, int mt, int32_t* d_status, cudaStream_t s) {
    CUtensorMap maps[4] = {};
    int rc = CASS_OK;
    if (a.p_groups) {
        rc = shared_cache_map(&maps[0], a.kp, a.d, a.prefix, a.n_kv, 1, a.p_pos, a.p_head, 0);
        if (!rc) rc = shared_cache_map(&maps[1], a.vp, a.d, a.prefix, a.n_kv, 1, a.p_pos, a.p_head, 0);
    }
    if (!rc && a.capacity) {
        rc = shared_cache_map(&maps[2], a.kc, a.d, a.capacity, a.n_kv, a.n_seq, a.c_pos, a.c_head, a.c_seq);
        if (!rc) rc = shared_cache_map(&maps[3], a.vc, a.d, a.capacity, a.n_kv, a.n_seq, a.c_pos, a.c_head, a.c_seq);
    }
    if (rc) return rc;
    switch (a.d) {
        case 32: return run_shared_stream_d<DT, 32>(a, mt, maps, d_status, s);
        case 64: return run_shared_stream_d<DT, 64>(a, mt, maps, d_status, s);
        case 96: return run_shared_stream_d<DT, 96>(a, mt, maps, d_status, s);
        case 128: return run_shared_stream_d<DT, 128>(a, mt, maps, d_status, s);
        case 192: return run_shared_stream_d<DT, 192>(a, mt, maps, d_status, s);
        case 256: return run_shared_stream_d<DT, 256>(a, mt, maps, d_status, s);
    }
    return CASS_ERR_UNSUPPORTED;
}

}  // namespace cass
