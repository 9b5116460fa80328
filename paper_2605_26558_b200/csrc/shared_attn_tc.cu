// The shared prefix's part of the attention where many queries see it: tiles of 128 (sequence, row, query head) pairs by 128 positions on
// the tensor cores (tcgen05), for head sizes 64 and 128.
// A CTA holds the queries of one or two tiles of a KV head and takes a range of the prefix through both products:
//   scores [128 pairs x 128 positions] = Q K^T, in tensor memory; softmax numerators P over them, 16 bits; output [128 pairs x d] += P V.
// A pair is a lane of tensor memory and a thread, so the softmax crosses no threads.  The output stays in tensor memory; it is rescaled only
// when a pair's maximum has grown by more than 2^8 (fp16: 2^4) since the base that its numerators are relative to, which after the first
// tiles hardly happens.  Two warpgroups alternate on the tensor cores: with two tiles of
// pairs each has one, and both use the same K and V; with one they take the positions' tiles in turn.  While one's numerators are formed
// the other's products run.
// Bound: with one tile of pairs K and V bytes, 1.31 us for the 64 KB of 128 positions on every SM, 7.4 TB/s.  With two, the chain of
// a tile (scores, softmax, product): the two warpgroups' chains overlap, but tensor pipe (54 % of the clocks, fp16 52) and exponentials (16 a clock: 1024
// clocks a tile, as both products take) are each busy half of the time; 2.1 us for the four products, 1.18 PFLOP/s, 73 % of a library
// product's rate.  The positions' tiles by halves of 64 took 2.45 us, four softmax warpgroups of 64 columns 2.25.
#include "tc.cuh"
#include "shared_attn.cuh"

namespace cass {

constexpr int kStThreads = 384;                          // warp 0: TMA; warp 1: MMA issue and tensor memory; warps 4-7 and 8-11: softmax, output
constexpr int kStRegsLaunch = 168, kStRegsIssue = 56, kStRegsSoftmax = 224;          // a softmax thread holds its 128 scores of a tile
static_assert(128 * kStRegsIssue + 256 * kStRegsSoftmax <= kStThreads * kStRegsLaunch, "the shares come from what the block was launched with");
constexpr uint32_t kStS = 0, kStO = 256;                 // tensor memory: two score (and P) buffers, two outputs, 128 columns each
constexpr int kStFewTiles = 4;                           // (tiles of pairs, of positions) an SM up to which SMs are left to the streaming kernel

template <int D>
struct StShape {
    static constexpr int q_tile = kStTile * D * 2;       // Q of 128 pairs; K or V of 128 positions: boxes of 128 x 64, 128-byte swizzle
    static constexpr int slots = D == 128 ? 5 : 8;
    static constexpr int smem = (2 + slots) * q_tile + 256 + 1024;
    static_assert((2 * slots + 6) * 8 + 4 <= 256, "the barriers behind the ring");
    static_assert(slots * q_tile >= 8 * 32 * D * 4, "the outputs pass through the ring");
    static_assert(smem <= (int)kSmemPerBlock, "shared memory of a CTA");
};

__device__ __forceinline__ void st_mma_tmem_a(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 columns of the thread's lane, not waited for.
__device__ __forceinline__ void st_ld32(uint32_t taddr, float* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
          "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
          "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
          "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr));
}
__device__ __forceinline__ void st_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_st32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]),
        "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
// kind::f16, D fp32, A and B of type DT; b_mn_major: B is stored with its columns contiguous
template <int DT>
constexpr uint32_t st_idesc(int m, int n, bool b_mn_major) {
    return (1u << 4) | ((DT == CASS_BF16 ? 1u : 0u) << 7) | ((DT == CASS_BF16 ? 1u : 0u) << 10) | ((b_mn_major ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void st_arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }

// grid: one CTA for every (split, head, two tiles of pairs), then for every (split, head) of the tile left over.  A role that gives up a wait
// flags the status and goes to the end; the others' waits run out in turn.
template <int DT, int D>
__global__ void __launch_bounds__(kStThreads, 1) k_shared_prefix_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                    SharedAttn a, int32_t* __restrict__ d_status) {
    using S = StShape<D>;
    using T = SaType<DT>;
    constexpr float kLift = T::kLift > 0.f ? T::kLift - T::kGrowth : 0.f;        // numerators may outgrow the base
    constexpr int kBoxes = D / 64, kTile = S::q_tile, kBox = kStTile * 64 * 2;
    extern __shared__ uint8_t smem_dyn[];
    uint8_t* base = reinterpret_cast<uint8_t*>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    uint8_t *sQ = base, *sT = base + 2 * kTile;
    uint64_t* full = reinterpret_cast<uint64_t*>(sT + S::slots * kTile);
    uint64_t *empty = full + S::slots, *s_full = empty + S::slots, *p_done = s_full + 2, *o_full = p_done + 2, *drained = o_full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
    int64_t* s_q = reinterpret_cast<int64_t*>(sT + (S::slots - 1) * kTile);      // where a pair's query lies, -1: there is none; before the slot's first tile
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    // ---- which pairs, which positions ----
    const int ctas2 = a.pre_s2 * a.n_kv * a.pre_n2;
    const bool two = (int)blockIdx.x < ctas2;            // two tiles of pairs
    int i = two ? blockIdx.x : blockIdx.x - ctas2;
    const int cta = two ? i % a.pre_n2 : a.pre_n2;
    if (two) i /= a.pre_n2;
    const int head = i % a.n_kv, split = i / a.n_kv, splits = two ? a.pre_s2 : a.pre_s1;
    const int tiles = ceil_div(a.prefix, kStTile), j0 = (int)((int64_t)tiles * split / splits), n = (int)((int64_t)tiles * (split + 1) / splits) - j0;
    const int first = cta * 2 * kStTile, P = a.n_seq * a.rows * a.group;
    if (tid == 0) {
        for (int b = 0; b < S::slots; ++b) { mbar_init(&full[b], 1); mbar_init(&empty[b], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&s_full[b], 1); mbar_init(&p_done[b], 4); }
        mbar_init(o_full, 1);
        mbar_init(drained, 1);
        fence_mbar_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    // K and V tiles in the order of the products that read them; the first ones travel while Q is gathered
    int it = 0;
    bool ok = true;
    const int ahead = two ? 1 : 2;                       // score products before the first output product
    auto load = [&](int x) {                             // the x-th tile of that order
        const int lead = min(ahead, n), y = x - lead;    // K 0 .. lead - 1, then V 0, K lead, V 1, ...; V alone at the end
        const int pairs = n - lead;                      // (V, K) pairs
        const bool is_v = y >= 0 && (y >= 2 * pairs || y % 2 == 0);
        const int j = y < 0 ? x : y >= 2 * pairs ? y - pairs : is_v ? y / 2 : y / 2 + lead;
        const int s = x % S::slots;
        mbar_expect_tx(&full[s], kTile);
#pragma unroll
        for (int b = 0; b < kBoxes; ++b)
            tma_load_3d(sT + s * kTile + b * kBox, is_v ? &map_v : &map_k, b * 64, head, (j0 + j) * kStTile, &full[s]);
    };
    if (tid == 0)
        for (; it < min(2 * n, S::slots - 1); ++it) load(it);
    if (warp >= 4) {
        // Q: pair p of the tiles = ((sequence x rows + row) x group + head in the group), zeros beyond the last
        const int x = tid - 128, c8 = x % (D / 8), rows = (two ? 2 : 1) * kStTile;
        if (x < rows) {
            const int all = first + x, r = all / a.group, g = all - r * a.group, seq = r / a.rows;
            s_q[x] = all < P ? (int64_t)seq * a.q_seq + (int64_t)(r - seq * a.rows) * a.q_row + (int64_t)(head * a.group + g) * a.q_head : -1;
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        constexpr int kStep = 256 / (D / 8), kUnroll = kStTile / kStep;      // rows at a time, a tile under way
        for (int p0 = x / (D / 8); p0 < rows; p0 += kStep * kUnroll) {
            uint4 v[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int64_t at = s_q[p0 + u * kStep];
                v[u] = at >= 0 ? *reinterpret_cast<const uint4*>(a.q + at + c8 * 8) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int p = p0 + u * kStep;
                *reinterpret_cast<uint4*>(sQ + (p / kStTile) * kTile + (c8 >> 3) * kBox + (p % kStTile) * 128 + (((c8 ^ p) & 7) << 4)) = v[u];
            }
        }
        fence_proxy_async();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_launch_dependents();                             // the streaming kernel, which waits for this one at its end
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kStRegsIssue));
        if (warp == 0) {
            if (tid == 0) {
                for (; it < 2 * n; ++it) {
                    ok = mbar_wait_bounded(&empty[it % S::slots], ((uint32_t)(it / S::slots) & 1u) ^ 1u);
                    if (!ok) break;
                    load(it);
                }
                if (!ok) atomicCAS(d_status, 0, CASS_ERR_TIMEOUT);
            }
        } else if (warp == 1) {
            if (tc_elect()) {
                it = 0;
                auto tile_in = [&]() -> const uint8_t* {     // the next tile, once it has arrived
                    const int s = it % S::slots;
                    ok = ok && mbar_wait_bounded(&full[s], (uint32_t)(it / S::slots) & 1u);
                    tc_fence_after();
                    return sT + s * kTile;
                };
                auto tile_out = [&]() { tc_commit(&empty[it % S::slots]); ++it; };
                auto scores = [&](int w, const uint8_t* k) {
                    constexpr uint32_t idesc = st_idesc<DT>(kStTile, kStTile, false);
                    const uint8_t* q = sQ + (two ? w : 0) * kTile;
#pragma unroll
                    for (int b = 0; b < kBoxes; ++b) {
                        const uint64_t ad = tc_smem_desc(q + b * kBox), bd = tc_smem_desc(k + b * kBox);
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            tc_mma(tmem + kStS + w * 128, ad + (uint64_t)(kk * 2), bd + (uint64_t)(kk * 2), idesc, (uint32_t)((b | kk) != 0));
                    }
                    tc_commit(&s_full[w]);
                };
                auto output = [&](int w, int use, const uint8_t* v) {            // the warpgroup's use-th tile
                    ok = ok && mbar_wait_bounded(&p_done[w], (uint32_t)use & 1u);
                    tc_fence_after();
                    if (!ok) return;
                    constexpr uint32_t idesc = st_idesc<DT>(kStTile, D, true);
#pragma unroll
                    for (int kk = 0; kk < kStTile / 16; ++kk)
                        st_mma_tmem_a(tmem + kStO + w * 128, tmem + kStS + w * 128 + kk * 8, tc_smem_desc(v + kk * 2048, kBox), idesc,
                                      (uint32_t)((use | kk) != 0));
                };
                // Scores go over the numerators that the output product before them, issued earlier, has read: products run in order.
                if (two) {
                    for (int j = 0; j <= n && ok; ++j) {
                        const uint8_t* v = nullptr;
                        if (j > 0) {
                            v = tile_in();                   // V of tile j - 1
                            if (ok) output(0, j - 1, v);
                        }
                        const int v_slot = it % S::slots;
                        if (j > 0) ++it;
                        const uint8_t* k = nullptr;
                        if (j < n && ok) {
                            k = tile_in();
                            if (ok) scores(0, k);
                        }
                        if (j > 0 && ok) {
                            output(1, j - 1, v);
                            if (ok) tc_commit(&empty[v_slot]);
                        }
                        if (j < n && ok) {
                            scores(1, k);
                            tile_out();
                        }
                    }
                } else {
                    for (int j = 0; j < min(2, n) && ok; ++j) {
                        const uint8_t* k = tile_in();
                        if (ok) { scores(j, k); tile_out(); }
                    }
                    for (int j = 0; j < n && ok; ++j) {
                        const uint8_t* v = tile_in();
                        if (ok) output(j & 1, j >> 1, v);
                        if (!ok) break;
                        tile_out();
                        if (j + 2 < n) {
                            const uint8_t* k = tile_in();
                            if (ok) { scores(j & 1, k); tile_out(); }
                        }
                    }
                }
                if (ok) tc_commit(o_full);
                else {
                    atomicCAS(d_status, 0, CASS_ERR_TIMEOUT);
                    for (int s = it; s < it + S::slots; ++s)                     // what is in flight lands before the CTA ends (bounded)
                        mbar_wait_bounded(&full[s % S::slots], (uint32_t)(s / S::slots) & 1u);
                }
                tc_commit(drained);                      // also who gives up, and whoever gives up beside it: tensor memory is freed behind the last product
                mbar_wait_bounded(drained, 0);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kStRegsSoftmax));
        const int wg = (warp - 4) >> 2, q = warp & 3, row = q * 32 + lane;   // the thread's pair of its tile
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16), sc = lanes + kStS + wg * 128, oc = lanes + kStO + wg * 128;
        const int uses = two ? n : (n - wg + 1) / 2;
        float m = -INFINITY, l = 0.f;                    // the base of the numerators; their sum
        for (int u = 0; u < uses; ++u) {
            const int j = j0 + (two ? u : 2 * u + wg);
            ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(&s_full[wg], (uint32_t)u & 1u));
            if (!ok) break;
            tc_fence_after();
            float s[128];
#pragma unroll
            for (int c = 0; c < 128; c += 32) st_ld32(sc + c, s + c);
            st_wait_ld();
            const int left = a.prefix - j * kStTile;     // positions of the tile
            if (left < kStTile) {
#pragma unroll
                for (int c = 0; c < 128; ++c) s[c] = c < left ? s[c] : -INFINITY;
            }
            float x[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
            for (int c = 4; c < 128; ++c) x[c & 3] = fmaxf(x[c & 3], s[c]);
            const float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) * a.scale_log2;      // (the scale is positive)
            const bool grew = top > m + T::kGrowth;       // also from -inf
            if (__any_sync(0xffffffffu, grew)) {
                const float fix = grew ? exp2_fast(m - top) : 1.f;
                if (grew) m = top;
                if (u > 0) {
                    l *= fix;
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        uint32_t b[32];
                        st_ld32(oc + c, o);
                        st_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) b[e] = __float_as_uint(o[e] * fix);
                        st_st32(oc + c, b);
                    }
                }
            }
            const float from = (m == -INFINITY ? 0.f : m) - kLift;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 128; c += 64) {
                uint32_t b[32];
#pragma unroll
                for (int e = 0; e < 64; e += 2) {
                    const float p0 = exp2_fast(fmaf(s[c + e], a.scale_log2, -from)), p1 = exp2_fast(fmaf(s[c + e + 1], a.scale_log2, -from));
                    sum[e & 2] += p0;
                    sum[(e & 2) + 1] += p1;
                    b[e / 2] = T::pack(p0, p1);
                }
                st_st32(sc + c / 2, b);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            st_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) st_arrive(&p_done[wg]);
        }
        ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(o_full, 0));
        if (ok) {
            tc_fence_after();
            const int all = first + (two ? wg * kStTile : 0) + row;
            const int64_t at = two ? (((int64_t)split * a.n_kv + head) * a.pre_n2 + cta) * 2 * kStTile + wg * kStTile + row
                                   : a.pre_at1 + ((int64_t)(2 * split + wg) * a.n_kv + head) * kStTile + row;
            if (all < P) a.pre_ml[at] = make_float2(m - kLift, l);
            // through the ring (every product that read it is done), so that a warp's stores are whole rows
            float4* box = reinterpret_cast<float4*>(sT) + (warp - 4) * 32 * (D / 4);
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                float o[32];
                st_ld32(oc + c, o);
                st_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; e += 4)
                    box[lane * (D / 4) + (((c + e) / 4) ^ (lane & 7))] = uses ? make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            __syncwarp();
            float* to = a.pre_o + (at - lane) * D;
            const int there = min(32, P - (all - lane));
#pragma unroll 8
            for (int x = lane; x < there * (D / 4); x += 32) {
                const int r = x / (D / 4), c = x % (D / 4);
                reinterpret_cast<float4*>(to)[x] = box[r * (D / 4) + (c ^ (r & 7))];
            }
        } else if (lane == 0) atomicCAS(d_status, 0, CASS_ERR_TIMEOUT);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

bool shared_tc_usable(const SharedAttn& a) {
    const int64_t most = (int64_t)1 << 38;               // a tensor map's strides: below 2^40 bytes
    return (a.d == 64 || a.d == 128) && a.p_pos < most && a.p_head < most;
}

int64_t shared_tc_plan(SharedAttn& a) {
    const int P = a.n_seq * a.rows * a.group, pair_tiles = ceil_div(P, kStTile), tiles = ceil_div(a.prefix, kStTile);
    const bool odd = pair_tiles & 1;
    a.pre_n2 = pair_tiles / 2;
    // CTAs over the positions: the least time of the slower kind with at most one CTA an SM (if there are not more heads and pairs
    // than that anyway).  A tile of positions takes two tiles of pairs 2.1 us (the products, 1.2 PFLOP/s), one tile 1.3 (K and V at the
    // memory's rate); an output to be left behind 3.
    // (Measured for head size 128.  For 64 products, bytes and outputs are half of it, the exponentials are not; the choice is taken alike.)
    // SMs are left to the streaming kernel, which starts beside this one: the products do not need the memory's rate that the caches do.
    // Their share is what that kernel's tiles take, 0.6 us each (1.5 with more than 16 pairs), if the caches are 3/4 full, half at most; and
    // half where there is little to do, as each SM more saves less than the parts that it leaves cost.  64 sequences (40 heads) behind
    // 32768 positions with caches of 1000: 100 -> 89 us on 96 SMs, 8 sequences (32 heads) behind 4000 with 600: 23.9 -> 22.1 on 72.
    a.pre_s2 = a.pre_n2 ? 1 : 0;
    a.pre_s1 = odd ? 1 : 0;
    const double here = (double)tiles * a.n_kv * (a.pre_n2 * 2.1 + (odd ? 1.3 : 0.0));
    const double there = 0.75 * (a.capacity / kSaTok + 1) * a.n_seq * a.n_kv * a.c_groups * (a.rows * a.group > 16 ? 1.5 : 0.6);
    const bool little = (int64_t)tiles * a.n_kv * pair_tiles <= kStFewTiles * kSms;
    const double share = !a.capacity ? 0.0 : little ? 0.5 : there / (here + there) < 0.5 ? there / (here + there) : 0.5;
    const int sms = kSms - (int)(share * kSms);
    double best = 1e30;
    for (int s2 = a.pre_n2 ? 1 : 0; s2 <= (a.pre_n2 ? (tiles < kSms ? tiles : kSms) : 0); ++s2) {
        const int room = sms / a.n_kv - s2 * a.pre_n2;
        if (odd ? room < 1 : room < 0) break;
        const int s1 = !odd ? 0 : room < tiles ? room : tiles;
        const double t2 = s2 ? ceil_div(tiles, s2) * 2.1 + 3.0 : 0.0, t1 = s1 ? ceil_div(tiles, s1) * 1.3 + 3.0 : 0.0, t = t1 > t2 ? t1 : t2;
        if (t < best) { best = t; a.pre_s2 = s2; a.pre_s1 = s1; }
    }
    a.pre_at1 = (int64_t)a.pre_s2 * a.n_kv * a.pre_n2 * 2 * kStTile;
    return a.pre_at1 + (int64_t)2 * a.pre_s1 * a.n_kv * kStTile;
}

// The prefix's K or V as [position][head][dim], whatever the order in memory, in boxes of 128 positions x 64 dims; zeros behind the last position.
static int prefix_map(CUtensorMap* m, const SharedAttn& a, const uint16_t* at) {
    const cuuint64_t gdim[3] = {(cuuint64_t)a.d, (cuuint64_t)a.n_kv, (cuuint64_t)a.prefix};
    const cuuint64_t gstride[2] = {(cuuint64_t)(a.n_kv > 1 ? a.p_head : a.d) * 2, (cuuint64_t)(a.prefix > 1 ? a.p_pos : a.d) * 2};
    const cuuint32_t box[3] = {64, 1, kStTile};
    return tc_map(m, 3, at, gdim, gstride, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int DT, int D>
static int run_tc(const SharedAttn& a, const CUtensorMap& mk, const CUtensorMap& mv, int32_t* d_status, cudaStream_t s) {
    CASS_ALLOW_SMEM(k_shared_prefix_tc<DT, D>);
    const int ctas = a.n_kv * (a.pre_s2 * a.pre_n2 + a.pre_s1);
    CASS_PDL_LAUNCH((k_shared_prefix_tc<DT, D>), dim3(ctas), dim3(kStThreads), (size_t)StShape<D>::smem, s, mk, mv, a, d_status);
    return CASS_OK;
}

int launch_shared_prefix_tc(const SharedAttn& a, int dtype, int32_t* d_status, cudaStream_t s) {
    CUtensorMap mk, mv;
    int rc = prefix_map(&mk, a, a.kp);
    if (!rc) rc = prefix_map(&mv, a, a.vp);
    if (rc) return rc;
    if (dtype == CASS_BF16) return a.d == 64 ? run_tc<CASS_BF16, 64>(a, mk, mv, d_status, s) : run_tc<CASS_BF16, 128>(a, mk, mv, d_status, s);
    return a.d == 64 ? run_tc<CASS_F16, 64>(a, mk, mv, d_status, s) : run_tc<CASS_F16, 128>(a, mk, mv, d_status, s);
}

}  // namespace cass
