// The streaming kernel of the shared-prefix attention: a prefix behind few (sequence, row, query head) pairs, or of a head size that the
// tensor-core kernel does not take, and every sequence's own cache.  Tiles of 64 positions come by TMA into a ring (one warp fetches, the others compute), both products run by mma.sync (16 pairs by
// 8 positions or dims), the softmax in registers with a running maximum.  What is bound by memory runs here: with few pairs a
// position's bytes cost more time on the bus than in the products.  The positions of all segments form one list of tiles that the CTAs share,
// whatever the lengths are, and the lengths are read on the device.
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

// The next CTA of the grid that has not started is taken over, if there is one: 16 bytes at `to` say so, and complete on `bar`.
__device__ __forceinline__ void take_over(void* to, uint64_t* bar) {
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(to)), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ int taken_over(const void* at) {                            // its number in the grid; -1: there was none left
    uint32_t yes, x;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\tld.shared.b128 r, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\tselp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
        : "=r"(yes), "=r"(x)
        : "r"(smem_u32(at))
        : "memory");
    return yes ? (int)x : -1;
}

constexpr int kSaBoxPos = 32;                            // positions of a TMA box: a segment's last tile brings no more than it has to

// Four warps compute; two CTAs an SM, so that one's join and latencies run beside the other's products.  (Eight warps of one CTA, all in a
// run: 2.2 us for its end and the next one's begin.)
template <int D, int MT>
struct SaShape {
    static constexpr int width = D % 64 == 0 ? 64 : 32;  // dims of a box: 128 or 64 bytes, swizzled over as many
    static constexpr int warps = 4;                      // that compute; one more fetches
    static constexpr int threads = (warps + 1) * 32;
    static constexpr int sets = warps / MT;              // of positions: a warp takes 64 / sets of a tile's, and 16 pairs
    static constexpr int tok = kSaTok / sets;
    static constexpr int pairs = 16 * MT;
    static constexpr int kv_bytes = kSaTok * D * 2;      // K or V of a tile
    static constexpr int stage_bytes = 2 * kv_bytes;
    static constexpr int q_bytes = pairs * D * 2;        // Q of a run
    static constexpr int per_sm = shared_stream_per_sm(D, MT);
    static constexpr int room = per_sm == 2 ? 112 * 1024 : 225 * 1024;
    static constexpr int runs = MT == 1 ? 2 : 1;         // whose queries are there or under way
    static constexpr int fit = (room - 1024 - runs * q_bytes) / stage_bytes, stages = fit < 8 ? fit : 8;
    static constexpr int smem = stages * stage_bytes + runs * q_bytes + 1024;    // 1024: alignment of the swizzled boxes
    static_assert(stages >= 3, "one tile in use, two under way");
    static_assert(sets == 1 || 2 * warps * 32 * D <= stage_bytes, "the warps' outputs fit a stage");
};

// Byte of 16-byte vector c of a row among a tile's (rows of `width` dims, box after box), as the swizzled copies leave them; eight rows'
// vectors of one column lie in different banks.
template <int D, int ROWS>
__device__ __forceinline__ uint32_t sa_at(int row, int c) {
    constexpr int kVecs = D % 64 == 0 ? 8 : 4;           // of a row in a box
    const int at = kVecs == 8 ? (c & 7) ^ (row & 7) : (c & 3) ^ ((row >> 1) & 3);
    return (uint32_t)((c / kVecs) * ROWS * kVecs * 16 + row * kVecs * 16 + (at << 4));
}

// One segment of the list.
struct SaSegment {
    int index, head, first, seq, n;                      // number; KV head; first pair; sequence (-1: prefix); positions
    int begin, end;                                      // tiles of the list
};
// Tiles of one segment in one piece of the list, as the fetching warp describes them to the others; tiles < 0: there are no more.
struct alignas(16) SaRun {
    int slot, head, first, seq, n, pos, tiles, pad;      // slot of the part; KV head; first pair; sequence; positions; first position
};

template <int DT, int D, int MT>
__global__ void __launch_bounds__(SaShape<D, MT>::threads, SaShape<D, MT>::per_sm)
    k_shared_stream(const __grid_constant__ CUtensorMap map_kp, const __grid_constant__ CUtensorMap map_vp, const __grid_constant__ CUtensorMap map_kc,
                    const __grid_constant__ CUtensorMap map_vc, SharedAttn a, int32_t* __restrict__ d_status) {
    using S = SaShape<D, MT>;
    using T = SaType<DT>;
    constexpr int kCount = S::warps * 32;                // threads that compute
    extern __shared__ uint8_t smem_dyn[];
    __shared__ float2 s_ml[S::sets][S::pairs];
    __shared__ uint64_t full[S::stages], empty[S::stages], r_full[S::runs], r_empty[S::runs], answered, meet[S::sets];
    __shared__ __align__(16) uint4 s_answer;             // which piece comes next
    __shared__ SaRun s_run[S::runs];
    uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (tid == 0) {
        for (int i = 0; i < S::stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], S::warps); }
        for (int i = 0; i < S::runs; ++i) { mbar_init(&r_full[i], 33); mbar_init(&r_empty[i], S::warps); }
        mbar_init(&answered, 1);
        for (int i = 0; i < S::sets; ++i) mbar_init(&meet[i], MT);
        fence_mbar_init();
        for (const CUtensorMap* map : {&map_kp, &map_vp, &map_kc, &map_vc}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    uint8_t* sQ0 = smem + S::stages * S::stage_bytes;
    // Behind the tensor-core kernel, which leaves this one's inputs alone and was not released before they were complete, it is waited for at the end.
    if (!a.behind_tc) pdl_wait();
    pdl_launch_dependents();                             // the merge, whose CTAs take the SMs as they get free
    __syncthreads();

    // Tiles go through the stages in turn.  A wait that runs out flags the status; the warp then goes on without waiting, so that
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
        // the list: a lane counts some sequences' tiles, in order
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
        SaSegment cur;
        auto first_of_seq = [&](int b, int begin) {      // segment 0 of the first sequence >= b that has tiles
            int n = 0;
            for (; b < a.n_seq; ++b) {
                n = shared_len(a, b);
                if (n > 0) break;
            }
            cur = {p_segs + b * seq_segs, 0, 0, b, n, begin, begin + ceil_div(n, kSaTok)};
        };
        auto next = [&]() {
            if (++cur.head == a.n_kv) { cur.head = 0; cur.first += S::pairs; }
            ++cur.index;
            if (cur.seq < 0 ? cur.index == p_segs : cur.index == p_segs + (cur.seq + 1) * seq_segs) {
                first_of_seq(cur.seq + 1, cur.end);
                return;
            }
            const int len = cur.end - cur.begin;
            cur.begin = cur.end;
            cur.end += len;
        };
        auto at_segment = [&](int i) {                   // i segments further in a row of equally long ones
            const int len = cur.end - cur.begin, groups = i / a.n_kv;
            cur.index += i; cur.head = i - groups * a.n_kv; cur.first = groups * S::pairs;
            cur.begin += i * len; cur.end += i * len;
        };
        auto find = [&](int t) {                         // the segment that tile t is in
            if (t < list.p_total) {
                cur = {0, 0, 0, -1, a.prefix, 0, list.p_tiles};
                at_segment(t / list.p_tiles);
                return;
            }
            const int at = (t - list.p_total) / seq_segs;          // in tiles of sequences: a sequence's segments are equally long
            const int who = __ffs(__ballot_sync(0xffffffffu, at >= upto - mine && at < upto)) - 1;
            int before = __shfl_sync(0xffffffffu, upto - mine, who), b = who * per;
            for (int i = 0; i < per; ++i, ++b) {
                const int n = ceil_div(max(shared_len(a, b), 0), kSaTok);
                if (at < before + n) break;
                before += n;
            }
            first_of_seq(b, list.p_total + before * seq_segs);
            at_segment((t - cur.begin) / (cur.end - cur.begin));
        };
        constexpr int kQRows = (S::pairs + 31) / 32;
        int left = 0, stage = 0, runs = 0;
        uint32_t parity = 1;                             // of the stage's release before: the first round finds it free
        auto fetch = [&](int t) {                        // one tile
            wait(&empty[stage], parity);
            if (!ok) return;
            if (lane == 0) {
                uint8_t* to = smem + stage * S::stage_bytes;
                const int pos = (t - cur.begin) * kSaTok, boxes = ceil_div(min(cur.n - pos, kSaTok), kSaBoxPos), seq = max(cur.seq, 0);
                const CUtensorMap *k = cur.seq < 0 ? &map_kp : &map_kc, *v = cur.seq < 0 ? &map_vp : &map_vc;
                mbar_expect_tx(&full[stage], boxes * (2 * kSaBoxPos * D * 2));
                for (int x = 0; x < D / S::width; ++x)
                    for (int y = 0; y < boxes; ++y) {
                        uint8_t* at = to + x * kSaTok * S::width * 2 + y * kSaBoxPos * S::width * 2;
                        tma_load_4d(at, k, x * S::width, pos + y * kSaBoxPos, cur.head, seq, &full[stage]);
                        tma_load_4d(at + S::kv_bytes, v, x * S::width, pos + y * kSaBoxPos, cur.head, seq, &full[stage]);
                    }
            }
            __syncwarp();
            ++left;
            if (++stage == S::stages) { stage = 0; parity ^= 1; }
        };
        auto tell = [&](int piece, int t, int tiles) {    // a run and its queries
            const int slot = runs % S::runs;
            wait(&r_empty[slot], ((uint32_t)(runs / S::runs) & 1u) ^ 1u);
            if (!ok) return;
            ++runs;
            if (tiles > 0) {
                const int P = (cur.seq < 0 ? a.n_seq : 1) * a.rows * a.group;
                uint8_t* to = sQ0 + slot * S::q_bytes;
                int64_t row[kQRows];                     // where the queries of a lane's pairs lie
#pragma unroll
                for (int i = 0; i < kQRows; ++i) {
                    const int all = cur.first + lane + 32 * i, r = all / a.group, seq = cur.seq < 0 ? r / a.rows : cur.seq;
                    row[i] = all < P ? (int64_t)seq * a.q_seq + (int64_t)(cur.seq < 0 ? r - seq * a.rows : r) * a.q_row +
                                           (int64_t)(cur.head * a.group + all - r * a.group) * a.q_head
                                     : -1;
                }
#pragma unroll
                for (int i = 0; i < kQRows; ++i)
                    for (int j = lane; j < (S::pairs < 32 ? S::pairs : 32) * (D / 8); j += 32) {
                        const int p = j / (D / 8), c = j % (D / 8);          // (D / 8 a divisor of 32 or not, all lanes take part)
                        const int64_t at = __shfl_sync(0xffffffffu, row[i], p);
                        cp16(to + sa_at<D, S::pairs>(32 * i + p, c), at >= 0 ? a.q + at + c * 8 : a.q, at >= 0);
                    }
            }
            if (lane == 0) {
                if (tiles > 0 && t == cur.begin) a.slots[cur.index].x = piece + cur.index;
                if (tiles > 0 && t + tiles == cur.end) a.slots[cur.index].y = piece + cur.index;
                s_run[slot] = {piece + cur.index, cur.head, cur.first, cur.seq, cur.n, (t - cur.begin) * kSaTok, tiles, 0};
                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&r_full[slot])) : "memory");
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&r_full[slot])) : "memory");
        };
        // CTAs of the grid are pieces: the first of every span, then the second of every span, ...
        int cta = blockIdx.x, ctas = 0;
        for (; cta >= 0 && ok; ++ctas) {
            const int level = cta / a.ctas, w = cta - level * a.ctas, piece = w * list.levels + level;
            const int first = shared_span(list, w), tiles = shared_span(list, w + 1) - first;
            const int t0 = first + shared_cut(list, tiles, level), t1 = level < list.levels ? first + shared_cut(list, tiles, level + 1) : t0;
            bool asked = false;
            auto ask = [&]() {                           // for the next piece, while this one is fetched
                if (!asked && lane == 0) {
                    mbar_expect_tx(&answered, 16);
                    take_over(&s_answer, &answered);
                }
                asked = true;
            };
            if (t0 < t1) find(t0);
            for (int t = t0; t < t1 && ok;) {
                if (t >= cur.end) next();
                const int end = min(t1, cur.end);
                fetch(t);
                if (ok) tell(piece, t, end - t);
                ask();
                for (++t; t < end && ok; ++t) fetch(t);
            }
            ask();
            wait(&answered, (uint32_t)ctas & 1u);
            cta = ok ? taken_over(&s_answer) : -1;
            fence_proxy_async();                         // the next answer comes behind this reading
            __syncwarp();
        }
        if (ok) tell(0, 0, -1);
        if (!ok) {                                       // what is in flight lands before the CTA ends (bounded): copies, and the last question's answer
            for (int i = max(left - S::stages, 0); i < left; ++i) mbar_wait_bounded(&full[i % S::stages], (uint32_t)(i / S::stages) & 1u);
            mbar_wait_bounded(&answered, (uint32_t)(ctas - 1) & 1u);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (a.behind_tc) pdl_wait();
        return;
    }

    // ---- the warps that compute ----
    const int mt = warp % MT, set = warp / MT, row = lane >> 2, col = 2 * (lane & 3);
    const int q_r = mt * 16 + (lane & 15), q_c = lane >> 4;
    float o[D / 8][4], m[2], l[2];
    uint32_t qf[D / 16][4];                              // Q, from a segment's first tile on
    int lim[2];                                          // positions that this thread's two rows see
    auto sync_all = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kCount) : "memory"); };
    auto arrive = [&](uint64_t* bar) {
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
    };
    int stage = 0;                                       // of the next tile
    uint32_t parity = 0;
    for (int runs = 0;; ++runs) {
        const int slot = runs % S::runs;
        wait(&r_full[slot], (uint32_t)(runs / S::runs) & 1u);
        int go;                                          // all of the warps, or none: there are barriers ahead
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                     : "=r"(go)
                     : "r"((int)ok), "n"(kCount)
                     : "memory");
        if (!go) break;
        const SaRun run = s_run[slot];
        if (run.tiles < 0) break;
        const uint32_t sQ = smem_u32(sQ0 + slot * S::q_bytes);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) ldm4(qf[k], sQ + sa_at<D, S::pairs>(q_r, 2 * k + q_c));
        arrive(&r_empty[slot]);
        const int P = min((run.seq < 0 ? a.n_seq : 1) * a.rows * a.group - run.first, S::pairs);
#pragma unroll
        for (int k = 0; k < D / 8; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[k][j] = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            m[k] = -INFINITY;
            l[k] = 0.f;
            const int p = mt * 16 + row + 8 * k;
            lim[k] = p >= P ? 0 : run.seq < 0 ? a.prefix : run.n - (a.rows - 1 - (run.first + p) / a.group);
        }
        uint8_t* at = smem;
        uint64_t* release = empty;                       // the last tile's stage is kept for the join
        for (int i = 0; i < run.tiles; ++i) {
            if (i > 0) arrive(release);
            at = smem + stage * S::stage_bytes;
            release = &empty[stage];
            wait(&full[stage], parity);
            if (++stage == S::stages) { stage = 0; parity ^= 1; }
            const uint32_t sK = smem_u32(at), sV = sK + S::kv_bytes;
            const int pos0 = run.pos + i * kSaTok + set * S::tok;         // this warp's first position
            if (pos0 + S::tok > run.n) {                     // behind the last position V is what the ring or the cache happens to hold
                for (int j = lane; j < S::tok * (D / 8); j += 32) {
                    const int p = j / (D / 8);
                    if (pos0 + p >= run.n)
                        *reinterpret_cast<uint4*>(at + S::kv_bytes + sa_at<D, kSaTok>(set * S::tok + p, j % (D / 8))) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_proxy_async();                     // the next copy into the stage comes behind these writes
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
                    ldm4(b, sK + sa_at<D, kSaTok>(set * S::tok + j * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
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
            if (a.scores && run.seq >= 0) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int p = run.first + mt * 16 + row + 8 * k;
                    if (p >= a.rows * a.group) continue;
                    float* to = a.scores + (((int64_t)run.seq * a.n_kv + run.head) * a.rows * a.group + p) * a.score_stride;
#pragma unroll
                    for (int j = 0; j < S::tok / 8; ++j) {
                        const int pos = pos0 + j * 8 + col;  // even, as the stride is
                        if (pos < run.n) *reinterpret_cast<float2*>(to + pos) = make_float2(s[j][2 * k] * a.scale_log2, s[j][2 * k + 1] * a.scale_log2);
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
                base[k] -= T::kLift;
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
            // Positions that some of the sequence's rows do not see: what is no number in their V must not meet a 0 of P in the product.  It
            // is added here, for the rows that see it, and taken out.  (In the product's loop the guard took the loads ahead of the products
            // apart, and made the code too long for the instruction cache: 16 x 5 rows behind 16000 positions 77 us for 63.)
            if (run.seq >= 0 && a.rows > 1 && pos0 + S::tok > run.n - (a.rows - 1) && pos0 < run.n) {
                const int t_lo = max(run.n - (a.rows - 1) - pos0, 0), t_hi = min(run.n - pos0, S::tok);      // of this warp's positions
                uint8_t* v = at + S::kv_bytes;
                bool odd = false;
                for (int j = t_lo * (D / 8) + lane; j < t_hi * (D / 8); j += 32) {
                    const uint4 w = *reinterpret_cast<const uint4*>(v + sa_at<D, kSaTok>(set * S::tok + j / (D / 8), j % (D / 8)));
                    const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) odd |= (e[c] & T::kExponent) == T::kExponent || (e[c] >> 16 & T::kExponent) == T::kExponent;
                }
                // (The warps of these positions find the same.  They meet at a barrier with a bounded wait: after a wait that ran out they
                // may have read different things.  Two meetings each time, phases 0 and 1; what became of them is looked at behind both: in each
                // of them it cost 16 x 5 rows behind 16000 positions 1.9 us, never running.)
                bool met = true;
                auto meeting = [&](uint32_t phase) {
                    __syncwarp();
                    if (MT > 1) {
                        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&meet[set])) : "memory");
                        if (!mbar_wait_bounded(&meet[set], phase)) met = false;
                        __syncwarp();
                    }
                };
                if (__any_sync(0xffffffffu, odd)) {
#pragma unroll 1
                    for (int t = t_lo; t < t_hi; ++t) {
                        float x[2];                      // p of this thread's rows: in lane 4 row + (t % 8) / 2
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            x[e] = 0.f;
#pragma unroll
                            for (int j = 0; j < S::tok / 8; ++j)
                                if (t / 8 == j) x[e] = __shfl_sync(0xffffffffu, (t & 1) ? s[j][2 * e + 1] : s[j][2 * e], (lane & ~3) | ((t & 7) >> 1));
                        }
#pragma unroll
                        for (int k = 0; k < D / 8; ++k) {
                            const uint32_t w = *reinterpret_cast<const uint32_t*>(v + sa_at<D, kSaTok>(set * S::tok + t, k) + col * 2);
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                const uint32_t bits = c ? w >> 16 : w & 0xFFFFu;
                                if ((bits & T::kExponent) != T::kExponent) continue;
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    if (pos0 + t < lim[e]) o[k][2 * e + c] = fmaf(x[e], T::get(bits), o[k][2 * e + c]);
                            }
                        }
                    }
                    meeting(0);
                    for (int j = t_lo * (D / 2) + lane; j < t_hi * (D / 2); j += 32) {
                        const int t = j / (D / 2), c = j % (D / 2);
                        uint32_t* w = reinterpret_cast<uint32_t*>(v + sa_at<D, kSaTok>(set * S::tok + t, c / 4) + (c % 4) * 4);
                        uint32_t bits = *w;
                        if ((bits & T::kExponent) == T::kExponent) bits &= 0xFFFF0000u;
                        if ((bits >> 16 & T::kExponent) == T::kExponent) bits &= 0x0000FFFFu;
                        *w = bits;
                    }
                    meeting(1);
                    fence_proxy_async();                 // the next copy into the stage comes behind these writes
                    if (MT > 1 && !__all_sync(0xffffffffu, met)) {
                        ok = false;
                        if (lane == 0) atomicCAS(d_status, 0, CASS_ERR_TIMEOUT);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < S::tok / 16; ++j) {
                const uint32_t p[4] = {T::pack(s[2 * j][0], s[2 * j][1]), T::pack(s[2 * j][2], s[2 * j][3]), T::pack(s[2 * j + 1][0], s[2 * j + 1][1]),
                                       T::pack(s[2 * j + 1][2], s[2 * j + 1][3])};
#pragma unroll
                for (int n = 0; n < D / 16; ++n) {
                    uint32_t b[4];                       // dims 0-7 (16 positions), dims 8-15
                    ldm4_t(b, sV + sa_at<D, kSaTok>(set * S::tok + j * 16 + (lane & 15), 2 * n + (lane >> 4)));
                    T::mma(o[2 * n], p, b[0], b[1]);
                    T::mma(o[2 * n + 1], p, b[2], b[3]);
                }
            }
        }
        // ---- the run's end: the warps' positions are joined, through the stage that was read last ----
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
            l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
            if ((lane & 3) == 0) s_ml[set][mt * 16 + row + 8 * k] = make_float2(m[k], l[k]);
        }
        sync_all();
        float all[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
        float* part = a.part_o + ((int64_t)run.slot * a.pairs + mt * 16 + row) * D + col;
        // a warp leaves its own outputs, rows 0 to 7 apart from rows 8 to 15, and adds up all sets' of some dims
        float2* box = reinterpret_cast<float2*>(at) + lane;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int p = mt * 16 + row + 8 * h;
#pragma unroll
            for (int g = 0; g < S::sets; ++g) all[h] = fmaxf(all[h], s_ml[g][p].x);
            const float b = all[h] == -INFINITY ? 0.f : all[h], fix = exp2_fast(m[h] - b);
#pragma unroll
            for (int g = 0; g < S::sets; ++g) sum[h] += exp2_fast(s_ml[g][p].x - b) * s_ml[g][p].y;
            if (S::sets > 1 && 8 * h < P) {
#pragma unroll
                for (int k = 0; k < D / 8; ++k) box[((h * S::warps + warp) * (D / 8) + k) * 32] = make_float2(o[k][2 * h] * fix, o[k][2 * h + 1] * fix);
            }
        }
        if (S::sets > 1) sync_all();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int p = mt * 16 + row + 8 * h;
            if (8 * h >= P) break;
#pragma unroll
            for (int k0 = 0; k0 < D / 8; k0 += S::sets) {
                const int k = k0 + set;
                if (k >= D / 8) break;
                float2 x = make_float2(o[k0][2 * h], o[k0][2 * h + 1]);
                if (S::sets > 1) {
                    x = make_float2(0.f, 0.f);
#pragma unroll
                    for (int g = 0; g < S::sets; ++g) {
                        const float2 y = box[((h * S::warps + g * MT + mt) * (D / 8) + k) * 32];         // of the warp of set g and these pairs
                        x.x += y.x;
                        x.y += y.y;
                    }
                }
                if (p < P) *reinterpret_cast<float2*>(part + (int64_t)8 * h * D + k * 8) = x;
            }
            if (set == 0 && p < P && (lane & 3) == 0) a.part_ml[(int64_t)run.slot * a.pairs + p] = make_float2(all[h] - T::kLift, sum[h]);
        }
        fence_proxy_async();
        arrive(release);
    }
    if (a.behind_tc) pdl_wait();
}

// K or V as [sequence][head][position][dim], whatever the order in memory, in boxes of 32 positions.
inline int shared_cache_map(CUtensorMap* map, const uint16_t* at, int d, int positions, int heads, int seqs, int64_t pos, int64_t head, int64_t seq) {
    const int width = d % 64 == 0 ? 64 : 32;
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)positions, (cuuint64_t)heads, (cuuint64_t)seqs};
    const cuuint64_t strides[3] = {(cuuint64_t)(positions > 1 ? pos : d) * 2, (cuuint64_t)(heads > 1 ? head : d) * 2, (cuuint64_t)(seqs > 1 ? seq : d) * 2};
    const cuuint32_t box[4] = {(cuuint32_t)width, kSaBoxPos, 1, 1};
    return tc_map(map, 4, at, dims, strides, box, width == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

template <int DT, int D, int MT>
int run_shared_stream(const SharedAttn& a, const CUtensorMap* maps, int levels, int32_t* d_status, cudaStream_t s) {
    using S = SaShape<D, MT>;
    CASS_ALLOW_SMEM(k_shared_stream<DT, D, MT>);
    CASS_PDL_LAUNCH((k_shared_stream<DT, D, MT>), dim3(levels * a.ctas), dim3(S::threads), (size_t)S::smem, s, maps[0], maps[1], maps[2], maps[3], a, d_status);
    return CASS_OK;
}

template <int DT, int D>
int run_shared_stream_d(const SharedAttn& a, int mt, const CUtensorMap* maps, int levels, int32_t* d_status, cudaStream_t s) {
    if (mt == 1) return run_shared_stream<DT, D, 1>(a, maps, levels, d_status, s);
    if constexpr (D <= 128) {
        if (mt == 2) return run_shared_stream<DT, D, 2>(a, maps, levels, d_status, s);
        if (mt == 4) return run_shared_stream<DT, D, 4>(a, maps, levels, d_status, s);
    }
    return CASS_ERR_UNSUPPORTED;
}

template <int DT>
int launch_shared_stream(const SharedAttn& a, int mt, int levels, int32_t* d_status, cudaStream_t s) {
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
        case 32: return run_shared_stream_d<DT, 32>(a, mt, maps, levels, d_status, s);
        case 64: return run_shared_stream_d<DT, 64>(a, mt, maps, levels, d_status, s);
        case 96: return run_shared_stream_d<DT, 96>(a, mt, maps, levels, d_status, s);
        case 128: return run_shared_stream_d<DT, 128>(a, mt, maps, levels, d_status, s);
        case 192: return run_shared_stream_d<DT, 192>(a, mt, maps, levels, d_status, s);
        case 256: return run_shared_stream_d<DT, 256>(a, mt, maps, levels, d_status, s);
    }
    return CASS_ERR_UNSUPPORTED;
}

}  // namespace cass
