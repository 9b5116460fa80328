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

// Two teams of four warps compute, on alternate tiles of a segment: one's softmax runs beside the other's products.  (All eight on one tile
// were in step with its latencies, 1.4 us a tile; two CTAs of one team each had their share of the list end at different times, 22 to
// 29 us after the start.)
template <int D, int MT>
struct SaShape {
    static constexpr int width = D % 64 == 0 ? 64 : 32;  // dims of a box: 128 or 64 bytes, swizzled over as many
    static constexpr int teams = D <= 128 ? 2 : 1;       // beyond, a thread's output and queries take all of its registers
    static constexpr int warps = 4 * teams;              // that compute; one more fetches
    static constexpr int threads = (warps + 1) * 32;
    static constexpr int groups = 4 / MT;                // of positions: a warp takes 64 / groups of a tile's, and 16 pairs
    static constexpr int tok = kSaTok / groups;
    static constexpr int pairs = 16 * MT;
    static constexpr int kv_bytes = kSaTok * D * 2;      // K or V of a tile
    static constexpr int stage_bytes = 2 * kv_bytes;
    static constexpr int q_bytes = pairs * D * 2;        // Q of a segment, two under way
    static constexpr int fit = (225 * 1024 - 2 * q_bytes) / stage_bytes, stages = fit < 8 ? fit : 8;
    static constexpr int smem = stages * stage_bytes + 2 * q_bytes + 1024;       // 1024: alignment of the swizzled boxes
    static_assert(stages >= teams + 1, "a tile under way beside those in use");
    static_assert(teams * groups * MT * 64 * D <= 2 * stage_bytes, "the joining of a segment's warps fits a stage");
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
    int begin, end;                                      // tiles of the list
};

template <int DT, int D, int MT>
__global__ void __launch_bounds__(SaShape<D, MT>::threads, 1)
    k_shared_stream(const __grid_constant__ CUtensorMap map_kp, const __grid_constant__ CUtensorMap map_vp, const __grid_constant__ CUtensorMap map_kc,
                    const __grid_constant__ CUtensorMap map_vc, SharedAttn a, int32_t* __restrict__ d_status) {
    using S = SaShape<D, MT>;
    using T = SaType<DT>;
    constexpr int kCount = S::warps * 32;                // threads that compute
    extern __shared__ uint8_t smem_dyn[];
    constexpr int kSets = S::teams * S::groups;          // of positions, over which a segment's pairs are joined
    __shared__ float s_ml[kSets][S::pairs][2];
    __shared__ uint64_t full[S::stages], empty[S::stages], q_full[2], q_empty[2];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (tid == 0) {
        for (int i = 0; i < S::stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 4); }
        for (int i = 0; i < 2; ++i) { mbar_init(&q_full[i], 32); mbar_init(&q_empty[i], S::warps); }
        fence_mbar_init();
        for (const CUtensorMap* map : {&map_kp, &map_vp, &map_kc, &map_vc}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    uint8_t* sQ0 = smem + S::stages * S::stage_bytes;
    // Behind the tensor-core kernel, which leaves this one's inputs alone and was not released before they were complete, it is waited for at the end.
    if (!a.behind_tc) pdl_wait();
    pdl_launch_dependents();                             // the merge counts the list while this kernel runs
    __syncthreads();

    // ---- the list: tiles of the prefix, then of the sequences; every warp counts it for itself, a lane some sequences in order ----
    const int per = ceil_div(a.n_seq, 32);
    int mine = 0;
    for (int i = 0; i < per; ++i) {
        const int b = lane * per + i;
        if (b < a.n_seq) mine += ceil_div(max(shared_len(a, b), 0), kSaTok);
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    const SaList list = shared_list(a, __shfl_sync(0xffffffffu, upto, 31));
    const int seq_segs = list.seq_segs, p_segs = list.p_segs;
    const int t0 = shared_first_tile(list, blockIdx.x), n_tiles = shared_first_tile(list, blockIdx.x + 1) - t0;
    if ((int)blockIdx.x >= list.workers || n_tiles <= 0) {
        if (a.behind_tc) pdl_wait();
        return;
    }
    int seq0 = 0, before0 = 0;                           // the sequence that the first tile falls into (if it is none of the prefix's), tiles before it
    if (t0 >= list.p_total) {
        const int at = (t0 - list.p_total) / seq_segs;   // in tiles of sequences: a sequence's segments are equally long
        const int who = __ffs(__ballot_sync(0xffffffffu, at >= upto - mine && at < upto)) - 1;
        before0 = __shfl_sync(0xffffffffu, upto - mine, who);
        seq0 = who * per;
        for (int i = 0; i < per; ++i) {
            const int n = ceil_div(max(shared_len(a, seq0), 0), kSaTok);
            if (at < before0 + n) break;
            before0 += n;
            ++seq0;
        }
    }

    auto first_of_seq = [&](SaSegment& g, int b, int begin) {     // segment 0 of the first sequence >= b that has tiles
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
        const int len = g.end - g.begin;
        g.begin = g.end;
        g.end += len;
    };
    SaSegment cur;
    if (t0 < list.p_total) {
        const int i = t0 / list.p_tiles;
        cur = {i, i % a.n_kv, i / a.n_kv * S::pairs, -1, a.prefix, i * list.p_tiles, (i + 1) * list.p_tiles};
    } else {
        first_of_seq(cur, seq0, list.p_total + before0 * seq_segs);
        const int len = cur.end - cur.begin;
        const int i = (t0 - cur.begin) / len;            // its segment
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
        int left = 0, stage = 0, segs = 0;
        uint32_t parity = 1;                             // of the stage's release before: the first round finds it free
        for (int i = 0; i < n_tiles; ++i) {
            const int t = t0 + i;
            if (t >= cur.end) next(cur);
            wait(&empty[stage], parity);
            if (!ok) break;
            if (lane == 0) {
                uint8_t* to = smem + stage * S::stage_bytes;
                const int pos = (t - cur.begin) * kSaTok, boxes = ceil_div(min(cur.n - pos, kSaTok), kSaBoxPos);
                const CUtensorMap *k = cur.seq < 0 ? &map_kp : &map_kc, *v = cur.seq < 0 ? &map_vp : &map_vc;
                mbar_expect_tx(&full[stage], boxes * (2 * kSaBoxPos * D * 2));
                for (int x = 0; x < D / S::width; ++x)
                    for (int y = 0; y < boxes; ++y) {
                        uint8_t* at = to + x * kSaTok * S::width * 2 + y * kSaBoxPos * S::width * 2;
                        tma_load_4d(at, k, x * S::width, pos + y * kSaBoxPos, cur.head, max(cur.seq, 0), &full[stage]);
                        tma_load_4d(at + S::kv_bytes, v, x * S::width, pos + y * kSaBoxPos, cur.head, max(cur.seq, 0), &full[stage]);
                    }
            }
            __syncwarp();
            left = i + 1;
            if (++stage == S::stages) { stage = 0; parity ^= 1; }
            if (i == 0 || t == cur.begin) {              // a segment's queries
                const int slot = segs & 1, P = pairs_of(cur);
                wait(&q_empty[slot], ((uint32_t)(segs >> 1) & 1u) ^ 1u);
                if (!ok) break;
                uint8_t* to = sQ0 + slot * S::q_bytes;
                for (int j = lane; j < S::pairs * (D / 8); j += 32) {
                    const int p = j / (D / 8), c = j % (D / 8), all = cur.first + p;
                    const bool there = all < P;
                    const int r = all / a.group, hq = cur.head * a.group + all - r * a.group;
                    const int64_t row = cur.seq < 0 ? (int64_t)(r / a.rows) * a.q_seq + (int64_t)(r % a.rows) * a.q_row
                                                    : (int64_t)cur.seq * a.q_seq + (int64_t)r * a.q_row;
                    cp16(to + sa_at<D, S::pairs>(p, c), there ? a.q + row + (int64_t)hq * a.q_head + c * 8 : a.q, there);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&q_full[slot])) : "memory");
                ++segs;
            }
        }
        if (!ok)                                         // what is in flight lands before the CTA ends (bounded)
            for (int i = max(left - S::stages, 0); i < left; ++i) mbar_wait_bounded(&full[i % S::stages], (uint32_t)(i / S::stages) & 1u);
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (a.behind_tc) pdl_wait();
        return;
    }

    // ---- the warps that compute ----
    const int team = warp / 4, mt = warp % MT, grp = warp % 4 / MT, set = team * S::groups + grp, row = lane >> 2, col = 2 * (lane & 3);
    const int q_r = mt * 16 + (lane & 15), q_c = lane >> 4;
    float o[D / 8][4], m[2], l[2], fix[2];
    uint32_t qf[D / 16][4];                              // Q, from a segment's first tile on
    int lim[2];                                          // positions that this thread's two rows see
    auto sync_all = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kCount) : "memory"); };
    auto arrive = [&](uint64_t* bar) {
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
    };
    int stage = 0, segs = 0;                             // of tile i
    uint32_t parity = 0;
    for (int i = 0; i < n_tiles; ++i) {
        const int t = t0 + i;
        if (t >= cur.end) next(cur);
        if (i == 0 || t == cur.begin) {
            const uint32_t sQ = smem_u32(sQ0 + (segs & 1) * S::q_bytes);
            wait(&q_full[segs & 1], (uint32_t)(segs >> 1) & 1u);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) ldm4(qf[k], sQ + sa_at<D, S::pairs>(q_r, 2 * k + q_c));
            arrive(&q_empty[segs & 1]);
            ++segs;
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
        uint8_t* at = smem + stage * S::stage_bytes;
        uint64_t* release = &empty[stage];
        const bool mine = S::teams == 1 || (i & 1) == team, ends = i + 1 == n_tiles || t + 1 == cur.end;
        bool wrote = false;
        const uint32_t tile_parity = parity;
        if (++stage == S::stages) { stage = 0; parity ^= 1; }
        if (mine) {
            wait(&full[release - empty], tile_parity);
            const uint32_t sK = smem_u32(at), sV = sK + S::kv_bytes;
            const int pos0 = (t - cur.begin) * kSaTok + grp * S::tok;         // this warp's first position
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
            float base[2];
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
        }
        // ---- the segment's end, or the worker's: the warps' positions are joined, through the stage that was read last ----
        if (ends) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
                l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
                if ((lane & 3) == 0) {
                    s_ml[set][mt * 16 + row + 8 * k][0] = m[k];
                    s_ml[set][mt * 16 + row + 8 * k][1] = l[k];
                }
            }
            sync_all();
            float all[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int p = mt * 16 + row + 8 * k;
#pragma unroll
                for (int g = 0; g < kSets; ++g) all[k] = fmaxf(all[k], s_ml[g][p][0]);
                const float b = all[k] == -INFINITY ? 0.f : all[k];
#pragma unroll
                for (int g = 0; g < kSets; ++g) sum[k] += exp2_fast(s_ml[g][p][0] - b) * s_ml[g][p][1];
                fix[k] = exp2_fast(m[k] - b);
            }
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[k][j] *= fix[j >> 1];
#pragma unroll
            for (int half = kSets / 2; half > 0; half /= 2) {
                float4* box = reinterpret_cast<float4*>(at) + lane;
                if (set >= half && set < 2 * half) {
#pragma unroll
                    for (int k = 0; k < D / 8; ++k)
                        box[(((set - half) * MT + mt) * (D / 8) + k) * 32] = make_float4(o[k][0], o[k][1], o[k][2], o[k][3]);
                }
                sync_all();
                if (set < half) {
#pragma unroll
                    for (int k = 0; k < D / 8; ++k) {
                        const float4 x = box[((set * MT + mt) * (D / 8) + k) * 32];
                        o[k][0] += x.x; o[k][1] += x.y; o[k][2] += x.z; o[k][3] += x.w;
                    }
                }
                if (half > 1) sync_all();
            }
            wrote = true;
            if (set == 0) {
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
        // The next copy into the stage comes behind what was written there: by this tile's team, and in the join by all.
        if (wrote) fence_proxy_async();
        if (ends) sync_all();
        if (mine) arrive(release);
    }
    if (a.behind_tc) pdl_wait();
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
