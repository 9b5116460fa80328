// Attention of a batch behind a shared prefix.  All sequences' queries of a KV head form the rows of one product with the prefix,
// which is read once for 16 to 256 of them; every sequence's own cache is read by its own queries.  Both leave partial results (output, maximum, sum) that
// k_shared_merge joins; the weights that the caches' positions got follow from the scores, once the sums are known.
//
// The prefix behind few queries and the caches are shared_stream.cuh's, the prefix behind many is shared_attn_tc.cu's.
#include "shared_attn.cuh"

namespace cass {

// ---- joining the parts ----

// Parts of one pair: at `o` and `ml`, `step` pairs apart.
struct SaParts {
    const float* o;
    const float2* ml;
    int64_t step;
    int n;
};

// grid: (query heads, rows, sequences), WARPS warps a head: one where there are many pairs, more where there are few with many parts.
// Bound: latency (two round trips behind the wait: where the parts lie, and the parts, eight of them together with a running maximum over
// the rounds; four where a warp joins a head's, which has few parts then: 23680 pairs of 37 sequences 32 us by eight, 20 by four).  What runs once pays for each of its instructions, some 6 clocks: places by divisions in every block took 2 us more.
constexpr int merge_threads(int warps) { return warps > 1 ? 32 * warps : 128; }

template <int DT, int WARPS>
__global__ void __launch_bounds__(merge_threads(WARPS)) k_shared_merge(SharedAttn a, int seg_shift, uint32_t group_magic, uint16_t* __restrict__ out,
                                                                       float* __restrict__ lse, int32_t* __restrict__ d_status) {
    using T = SaType<DT>;
    constexpr int kWarps = merge_threads(WARPS) / 32, kParts = WARPS == 1 ? 4 : 8;
    __shared__ __align__(16) float s_o[WARPS == 1 ? 1 : kWarps][256];
    __shared__ float2 s_ml[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int hq = blockIdx.x * (kWarps / WARPS) + warp / WARPS, r = blockIdx.y, b = blockIdx.z;
    const int head = a.group == 1 ? hq : (int)__umulhi((uint32_t)hq, group_magic), P = a.rows * a.group, p = r * a.group + hq - head * a.group;
    const int raw = a.lens ? a.lens[b] : 0, n = min(raw, a.capacity), seen = n - (a.rows - 1 - r);
    pdl_wait();
    if (a.lse) pdl_launch_dependents();                  // the weights, behind
    if (hq >= a.n_q || n < 0) return;                    // (n < 0: the sequence is not there)
    if (p == 0 && head == 0 && warp % WARPS == 0 && lane == 0 && raw > a.capacity) atomicCAS(d_status, 0, CASS_ERR_CAPACITY);
    // ---- where the parts lie: the prefix's, then the cache's ----
    SaParts first, second;
    const int all = b * P + p, seg = p >> seg_shift, in_seg = p & ((1 << seg_shift) - 1);        // the pair among those of all sequences; its segment
    int2 pre = make_int2(0, -1), own = make_int2(0, -1);
    if (a.p_groups) pre = shared_slots(a.slots[(all >> seg_shift) * a.n_kv + head], a.n_slots);
    if (n > 0) own = shared_slots(a.slots[a.p_groups * a.n_kv + (b * a.c_groups + seg) * a.n_kv + head], a.n_slots);
    if (a.prefix && !a.p_groups) {
        const bool two = all / (2 * kStTile) < a.pre_n2;
        const int64_t at = two ? ((int64_t)head * a.pre_n2 + all / (2 * kStTile)) * 2 * kStTile + all % (2 * kStTile)
                               : a.pre_at1 + (int64_t)head * kStTile + all % (2 * kStTile);
        first = {a.pre_o + at * a.d, a.pre_ml + at, (int64_t)a.n_kv * (two ? a.pre_n2 * 2 : 1) * kStTile, two ? a.pre_s2 : 2 * a.pre_s1};
    } else {
        const int64_t at = (int64_t)pre.x * a.pairs + (all & ((1 << seg_shift) - 1));
        first = {a.part_o + at * a.d, a.part_ml + at, a.pairs, pre.y - pre.x + 1};
    }
    {
        const int64_t at = (int64_t)own.x * a.pairs + in_seg;
        second = {a.part_o + at * a.d, a.part_ml + at, a.pairs, own.y - own.x + 1};
    }
    const bool sees = a.prefix > 0 || seen > 0;
    uint16_t* to = out + (int64_t)b * a.out_seq + (int64_t)r * a.out_row + (int64_t)hq * a.out_head;
    auto put = [&](int c, float4 x, float L) {
        const float inv = 1.f / L;
        if (sees) *reinterpret_cast<uint2*>(to + c) = make_uint2(T::pack(x.x * inv, x.y * inv), T::pack(x.z * inv, x.w * inv));
        else *reinterpret_cast<uint2*>(to + c) = make_uint2(0u, 0u);
    };
    float M = -INFINITY, L = 0.f;
    for (int c = lane * 4; c < ((a.d + 127) & ~127); c += 128) {     // all lanes, also those beyond d
        const bool in = c < a.d;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        M = -INFINITY;
        L = 0.f;
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
            const SaParts part = k ? second : first;
            const int count = part.n;
            const int64_t step = part.step * WARPS, step_o = step * a.d;
            const float2* ml = part.ml + (warp % WARPS) * part.step;
            const float* o = part.o + (warp % WARPS) * part.step * a.d + (in ? c : 0);
#pragma unroll 1
            for (int i = warp % WARPS; i < count; i += kParts * WARPS) {
                // loads without a branch between them: the last part again where there are no more
                float2 x[kParts];
                float4 y[kParts];
                float top = M;
#pragma unroll
                for (int j = 0; j < kParts; ++j) {
                    x[j] = *ml;
                    y[j] = *reinterpret_cast<const float4*>(o);
                    const bool more = i + (j + 1) * WARPS < count;
                    ml += more ? step : 0;
                    o += more ? step_o : 0;
                }
#pragma unroll
                for (int j = 0; j < kParts; ++j) {
                    if (j && i + j * WARPS >= count) { x[j] = make_float2(-INFINITY, 0.f); y[j] = make_float4(0.f, 0.f, 0.f, 0.f); }
                    top = fmaxf(top, x[j].x);
                }
                const float base = top == -INFINITY ? 0.f : top, fix = exp2_fast(M - base);
                M = top;
                L *= fix;
                sum.x *= fix; sum.y *= fix; sum.z *= fix; sum.w *= fix;
#pragma unroll
                for (int j = 0; j < kParts; ++j) {
                    const float f = exp2_fast(x[j].x - base);
                    L = fmaf(f, x[j].y, L);
                    sum.x = fmaf(f, y[j].x, sum.x); sum.y = fmaf(f, y[j].y, sum.y); sum.z = fmaf(f, y[j].z, sum.z); sum.w = fmaf(f, y[j].w, sum.w);
                }
            }
        }
        if (WARPS == 1) { if (in) put(c, sum, L); }
        else if (in) *reinterpret_cast<float4*>(&s_o[warp][c]) = sum;
    }
    if (WARPS > 1) {
        if (lane == 0) s_ml[warp] = make_float2(M, L);
        __syncthreads();
        if (warp != 0) return;
        const float2 x = lane < WARPS ? s_ml[lane] : make_float2(-INFINITY, 0.f);
        M = warp_max(x.x);
        const float f = exp2_fast(x.x - (M == -INFINITY ? 0.f : M));
        L = warp_sum(f * x.y);
        for (int c = lane * 4; c < ((a.d + 127) & ~127); c += 128) {
            float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                const float g = __shfl_sync(0xffffffffu, f, i);
                const float4 y = *reinterpret_cast<const float4*>(&s_o[i][c < a.d ? c : 0]);
                z.x = fmaf(g, y.x, z.x); z.y = fmaf(g, y.y, z.y); z.z = fmaf(g, y.z, z.z); z.w = fmaf(g, y.w, z.w);
            }
            if (c < a.d) put(c, z, L);
        }
    }
    if (lane == 0) {
        const float z = M + log2f(L);
        if (lse) lse[((int64_t)b * a.rows + r) * a.n_q + hq] = sees ? z * 0.693147180559945309f : -INFINITY;
        if (a.lse) a.lse[((int64_t)b * a.n_kv + head) * P + p] = z;
    }
}

// The weights that the positions of the caches got: the scores' share of the sums.  grid: (blocks of positions, KV heads, sequences).
// The scores were there before the merge released this kernel; they travel while it finishes.  A thread takes four positions and all pairs, or
// (SPLIT, more pairs than travel at a time) a warp takes every fourth pair: 80 pairs of 37 sequences of 146 positions 14.8 us without, 8.3 so;
// 20 pairs of 16 sequences of 1000 7.5 and 6.0.
constexpr int kSwThreads = 128, kSwPairs = 8, kSwMaxPairs = 256;
constexpr int sw_positions(bool split) { return split ? 128 : kSwThreads * 4; }

template <bool SPLIT>
__global__ void __launch_bounds__(kSwThreads) k_shared_weights(SharedAttn a, const float* in, float* out) {
    __shared__ float s_lse[kSwMaxPairs];
    __shared__ int s_end[kSwMaxPairs];
    __shared__ __align__(16) float s_sum[SPLIT ? kSwThreads / 32 : 1][SPLIT ? 128 : 4];
    constexpr int kStep = SPLIT ? kSwThreads / 32 : 1;
    const int tid = threadIdx.x, head = blockIdx.y, b = blockIdx.z, P = a.rows * a.group;
    const int first = SPLIT ? tid >> 5 : 0, base = blockIdx.x * sw_positions(SPLIT), pos = base + (SPLIT ? tid & 31 : tid) * 4;
    const int n = shared_len(a, b);
    const int64_t row = (int64_t)b * a.n_kv + head;
    const float* from = a.scores + row * P * a.score_stride + min(pos, max(n - 1, 0) & ~3);
    float4 x[kSwPairs];
    auto load = [&](int q0) {
#pragma unroll
        for (int i = 0; i < kSwPairs; ++i) x[i] = *reinterpret_cast<const float4*>(from + (int64_t)min(q0 + i * kStep, P - 1) * a.score_stride);
    };
    if (n > 0) load(first);
    pdl_wait();
    if (n < 0) return;                                   // the sequence is not there
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (n > 0) {
        for (int q = tid; q < P; q += kSwThreads) {
            s_lse[q] = a.lse[row * P + q];
            s_end[q] = n - (a.rows - 1 - q / a.group);   // what the pair sees
        }
        __syncthreads();
        for (int q0 = first; q0 < P; q0 += kSwPairs * kStep) {
            if (q0 != first) load(q0);
#pragma unroll
            for (int i = 0; i < kSwPairs; ++i) {
                if (q0 + i * kStep >= P) break;
                const int left = s_end[q0 + i * kStep] - pos;
                const float z = s_lse[q0 + i * kStep], v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += e < left ? exp2_fast(v[e] - z) : 0.f;
            }
        }
    }
    in = in ? in + row * a.capacity : nullptr;
    out += row * a.capacity;
    if constexpr (SPLIT) {
        *reinterpret_cast<float4*>(&s_sum[first][pos - base]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
        __syncthreads();
        const int at = base + tid;
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < kStep; ++i) all += s_sum[i][tid];
        if (at < a.capacity && (at < n || in != out)) out[at] = (in ? in[at] : 0.f) + all;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (pos + i < a.capacity && (pos + i < n || in != out)) out[pos + i] = (in ? in[pos + i] : 0.f) + sum[i];
    }
}

// ---- host ----

struct SaPlan {
    SharedAttn a;
    int mt, levels;
    bool tc;
    size_t at_o, at_ml, at_slots, at_scores, at_lse, at_pre_o, at_pre_ml, bytes;
};

// Pairs from which on a warp joins one alone.  us of a call, by one warp and by eight: 256 pairs 23.7, 21.9; 384 25.8, 24.2; 512 27.6, 28.1; 768 31.9,
// 33.4; 1536 40.4, 49.7.
constexpr int kSmManyPairs = 3 * kSms;
constexpr int kSmFewPairs = kSms / 2;                    // joined by 16 warps where a list is long: one cache of 32000 positions 37.8 -> 36.5 us; 256 pairs 20.3 -> 22.9
// A prefix is streamed behind up to 32 pairs a KV head while (pairs, 16 at least) x positions x KV heads is below this: a launch less.
// us, streamed and on the tensor cores, 8 KV heads of 128: 4 pairs, 4000 positions 12.5, 14.1; 32000 positions 35.0, 30.6; 16 pairs 13.5, 15.2
// and 40.0, 37.1; 24 pairs 15.9, 15.6 and 51.6, 37.8; 32 pairs, 1000 positions 16.1, 16.6; 2 heads of 64, 32 pairs, 2000 positions 9.4, 11.3.
constexpr int kSaStreamPairs = 32;
constexpr int64_t kSaStreamWork = 768 * 1024;

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
    plan->tc = a.prefix && shared_tc_usable(a) && (all > kSaStreamPairs || (int64_t)(all > 16 ? all : 16) * a.prefix * a.n_kv > kSaStreamWork);
    const int most = a.prefix && !plan->tc ? (all > P ? all : P) : P;
    // Pairs a CTA takes at a time: 64 where a cache has so many that hardly any place is empty, else 32 in two CTAs an SM.  us, 64 and 32: a cache of
    // 4000 behind 36 pairs 30.6, 33.5; 20 caches of 117 behind 64 21.9, 23.3; 6 of 2405 behind 80 104, 92; a prefix of 8000 behind 64 pairs of 96 dims 36.7, 33.4.
    plan->mt = a.d > 128 || most <= 16 ? 1 : P > 32 && 2 * ceil_div(P, 64) == ceil_div(P, 32) ? 4 : 2;
    const int seg = 16 * plan->mt;
    a.pairs = most < seg ? most : seg;
    a.p_groups = a.prefix && !plan->tc ? ceil_div(all, seg) : 0;
    a.c_groups = ceil_div(P, seg);
    a.score_stride = (int64_t)align_up(a.capacity, 4);
    // (with a cache's rows apart the sum fits any memory; a prefix without tensor cores may be walked by many groups)
    const int64_t tiles = (int64_t)a.p_groups * a.n_kv * ceil_div(a.prefix, kSaTok) + (int64_t)a.n_seq * a.n_kv * a.c_groups * (a.capacity / kSaTok + 1);
    if (tiles > kSaMaxTiles) return CASS_ERR_UNSUPPORTED;
    a.ctas = kSms * shared_stream_per_sm(a.d, plan->mt);
    if (tiles < a.ctas) a.ctas = tiles > 1 ? (int)tiles : 1;
    plan->levels = shared_levels((int)(tiles / a.ctas));
    size_t off = 0;
    auto take = [&](size_t b) { const size_t o2 = off; off = align_up(off + b, 256); return o2; };
    const size_t segments = (size_t)a.n_kv * ((size_t)a.p_groups + (size_t)a.n_seq * a.c_groups), slots = (size_t)kSaLevels * a.ctas + segments;
    a.n_slots = (int)slots;
    plan->at_o = take(slots * a.pairs * a.d * 4);
    plan->at_ml = take(slots * a.pairs * 8);
    plan->at_slots = take(segments * 8);
    a.behind_tc = plan->tc;
    const size_t pre = plan->tc ? (size_t)shared_tc_plan(a) : 0;
    plan->at_pre_o = take(pre * a.d * 4);
    plan->at_pre_ml = take(pre * 8);
    plan->at_scores = take(with_weights ? (size_t)a.n_seq * a.n_q * a.rows * a.score_stride * 4 : 0);
    plan->at_lse = take(with_weights ? (size_t)a.n_seq * a.n_q * a.rows * 4 : 0);
    plan->bytes = off < 256 ? 256 : off;
    return CASS_OK;
}

template <int DT>
static int run_shared(const SaPlan& plan, uint16_t* out, float* lse, const float* weight_in, float* weight_out, int32_t* d_status, cudaStream_t s) {
    const SharedAttn& a = plan.a;
    int rc = plan.tc ? launch_shared_prefix_tc(a, DT, d_status, s) : CASS_OK;
    if (rc) return rc;
    rc = DT == CASS_BF16 ? launch_shared_stream_bf16(a, plan.mt, plan.levels, d_status, s) : launch_shared_stream_f16(a, plan.mt, plan.levels, d_status, s);
    if (rc) return rc;
    const uint32_t magic = a.group == 1 ? 0u : 0xFFFFFFFFu / (uint32_t)a.group + 1u;         // head x group < 2^32
    const int seg_shift = plan.mt == 1 ? 4 : plan.mt == 2 ? 5 : 6;
    const int64_t pairs = (int64_t)a.n_seq * a.rows * a.n_q;
#define CASS_SHARED_MERGE(W_)                                                                                                               \
    CASS_PDL_LAUNCH((k_shared_merge<DT, W_>), dim3(W_ > 1 ? a.n_q : ceil_div(a.n_q, merge_threads(1) / 32), a.rows, a.n_seq),                 \
                    dim3(merge_threads(W_)), 0, s, a, seg_shift, magic, out, lse, d_status)
    if (pairs >= kSmManyPairs) CASS_SHARED_MERGE(1);
    else if (pairs <= kSmFewPairs && plan.levels > 1) CASS_SHARED_MERGE(16);
    else CASS_SHARED_MERGE(8);
#undef CASS_SHARED_MERGE
    if (weight_out) {
        const bool split = a.rows * a.group > kSwPairs;
        const dim3 grid(ceil_div(a.capacity, sw_positions(split)), a.n_kv, a.n_seq);
        if (split) CASS_PDL_LAUNCH(k_shared_weights<true>, grid, dim3(kSwThreads), 0, s, a, weight_in, weight_out);
        else CASS_PDL_LAUNCH(k_shared_weights<false>, grid, dim3(kSwThreads), 0, s, a, weight_in, weight_out);
    }
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
    a.part_o = (float*)(mem + plan.at_o); a.part_ml = (float2*)(mem + plan.at_ml); a.slots = (int2*)(mem + plan.at_slots);
    a.pre_o = (float*)(mem + plan.at_pre_o); a.pre_ml = (float2*)(mem + plan.at_pre_ml);
    a.scores = weight_out ? (float*)(mem + plan.at_scores) : nullptr;
    a.lse = weight_out ? (float*)(mem + plan.at_lse) : nullptr;
    if (cache->dtype == CASS_BF16) return run_shared<CASS_BF16>(plan, (uint16_t*)out, lse, weight_in, weight_out, d_status, (cudaStream_t)stream_);
    return run_shared<CASS_F16>(plan, (uint16_t*)out, lse, weight_in, weight_out, d_status, (cudaStream_t)stream_);
}
