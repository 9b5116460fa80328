// Attention of a batch behind a shared prefix.  All sequences' queries of a KV head form the rows of one product with the prefix,
// which is read once; every sequence's own cache is read by its own queries.  Both leave partial results (output, maximum, sum) that
// k_shared_merge joins; the weights that the caches' positions got follow from the scores, once the sums are known.
//
// The prefix behind few queries and the caches are shared_stream.cuh's, the prefix behind many is shared_attn_tc.cu's.
#include "shared_attn.cuh"

namespace cass {

// ---- joining the parts ----
constexpr int kSmThreads = 256, kSmWarps = kSmThreads / 32;
constexpr int kSmMaxParts = (2 * kSaLevels + 2) * kSms;          // of a pair: at most all units', and two of every CTA of the tensor-core kernel
constexpr int kSmPos = 4 * kSmThreads;                   // positions of a weights block

// Where the parts of (sequence b, head, pair p of the sequence) lie: those of the prefix, then those of its cache, in order.
struct SaParts {
    int64_t pre0, own0, pre_step;                        // first places, distance of two of the prefix (of the cache: a.pairs), in pairs
    int n_pre, n_own;
    bool pre_tc;
    __device__ __forceinline__ int count() const { return n_pre + n_own; }
};

__device__ SaParts shared_parts(const SharedAttn& a, const SaList& list, int seg_pairs, int b, int head, int p, int tiles_before, int n) {
    SaParts r{};
    const int all = b * a.rows * a.group + p;            // the pair among those of all sequences
    if (list.p_tiles) {
        const int s = all / seg_pairs * a.n_kv + head;
        const int w0 = shared_unit_of(list, s * list.p_tiles), w1 = shared_unit_of(list, (s + 1) * list.p_tiles - 1);
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
        const int k = p / seg_pairs * a.n_kv + head, first = list.p_total + tiles_before * list.seq_segs + k * tiles;
        const int w0 = shared_unit_of(list, first), w1 = shared_unit_of(list, first + tiles - 1);
        r.own0 = (int64_t)(w0 + list.p_segs + b * list.seq_segs + k) * a.pairs + p % seg_pairs;
        r.n_own = w1 - w0 + 1;
    }
    return r;
}

// grid: blocks of the (sequence, row, query head)s, WARPS warps each, then (with weights) one for every 1024 positions of every (sequence, KV
// head).  A warp a pair where there are many pairs, eight where there are few with many parts.
template <int DT, int WARPS>
__global__ void __launch_bounds__(kSmThreads) k_shared_merge(SharedAttn a, int seg_pairs, int pair_blocks, int pos_blocks, uint16_t* __restrict__ out,
                                                             float* __restrict__ lse, const float* weight_in, float* weight_out,
                                                             int32_t* __restrict__ d_status) {
    using T = SaType<DT>;
    __shared__ float s_w[WARPS == 1 ? kSmWarps : 1][kSmMaxParts];
    __shared__ __align__(16) float s_o[WARPS == 1 ? 1 : kSmWarps][256];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
        if (b >= a.n_seq) { pdl_wait(); return; }
        head = hq / a.group; p = r * a.group + hq % a.group;
    }
    // The lengths were complete before the streaming kernel released this one: where the parts lie is known by the time they are there.
    const int n = shared_len(a, b);
    int before = 0, tiles = 0;
    for (int i = lane; i < a.n_seq; i += 32) {
        const int t = ceil_div(max(shared_len(a, i), 0), kSaTok);
        tiles += t;
        before += i < b ? t : 0;
    }
    before = __reduce_add_sync(0xffffffffu, before);
    tiles = __reduce_add_sync(0xffffffffu, tiles);
    const SaList list = shared_list(a, tiles);
    const SaParts s = shared_parts(a, list, seg_pairs, b, head, p, before, n);
    pdl_wait();
    if (n < 0) return;                                   // the sequence is not there

    // Maximum of all parts and their sum relative to it, by a warp; w: the parts' factors, 2^(m - M).  What 256 parts need is loaded in one go.
    auto sums = [&](const SaParts& s, float* w, float& M, float& L) {
        const int count = s.count();
        const float *pm = s.pre_tc ? a.pre_m : a.part_m, *pl = s.pre_tc ? a.pre_l : a.part_l;
        float m[8], l[8];
        M = -INFINITY;
        L = 0.f;
        for (int i0 = lane; i0 - lane < count; i0 += 256) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + 32 * j;
                m[j] = -INFINITY;
                l[j] = 0.f;
                if (i < count) {
                    const bool pre = i < s.n_pre;
                    const int64_t at = pre ? s.pre0 + i * s.pre_step : s.own0 + (int64_t)(i - s.n_pre) * a.pairs;
                    m[j] = (pre ? pm : a.part_m)[at];
                    l[j] = (pre ? pl : a.part_l)[at];
                }
            }
            float top = M;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, m[j]);
            top = warp_max(top);
            const float base = top == -INFINITY ? 0.f : top, fix = exp2_fast(M - base);
            if (w && M != top)                           // beyond 256 parts: the factors so far follow
                for (int i = lane; i < i0 - lane; i += 32) w[i] *= fix;
            L *= fix;
            M = top;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = exp2_fast(m[j] - base);
                L += f * l[j];
                if (w && i0 + 32 * j < count) w[i0 + 32 * j] = f;
            }
        }
        L = warp_sum(L);
        __syncwarp();
    };
    if (weights) {
        const int pos = chunk * kSmPos + tid * 4, per_group = list.p_tiles ? seg_pairs : 2 * kStTile;
        const float* in = weight_in ? weight_in + ((int64_t)b * a.n_kv + head) * a.capacity : nullptr;
        float* to = weight_out + ((int64_t)b * a.n_kv + head) * a.capacity;
        float* s_lse = &s_w[0][0];
        float sum[4] = {0.f, 0.f, 0.f, 0.f}, was[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) was[i] = in && pos + i < a.capacity ? in[pos + i] : 0.f;
        if (chunk * kSmPos < n) {
            for (int q = warp; q < P; q += kSmWarps) {
                SaParts t = s;                           // of pair 0: those of its neighbours lie beside them, up to the next group's
                if (q / seg_pairs == 0 && (b * P + q) / per_group == b * P / per_group) { t.pre0 += q; t.own0 += q; }
                else t = shared_parts(a, list, seg_pairs, b, head, q, before, n);
                float M, L;
                sums(t, nullptr, M, L);
                if (lane == 0) s_lse[q] = M + log2f(L);
            }
            __syncthreads();
            const float* from = a.scores + ((int64_t)b * a.n_kv + head) * P * a.score_stride + pos;
            for (int q0 = 0; q0 < P; q0 += 8) {
                float4 x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (q0 + i < P && pos < n) x[i] = *reinterpret_cast<const float4*>(from + (q0 + i) * a.score_stride);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (q0 + i >= P) continue;
                    const int end = n - (a.rows - 1 - (q0 + i) / a.group);           // what the pair sees
                    const float z = s_lse[q0 + i], v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (pos + e < end) sum[e] += exp2_fast(v[e] - z);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (pos + i < a.capacity && (pos + i < n || in != to)) to[pos + i] = was[i] + sum[i];
        return;
    }
    if (p == 0 && head == 0 && warp % WARPS == 0 && lane == 0 && a.lens && a.lens[b] > a.capacity) atomicCAS(d_status, 0, CASS_ERR_CAPACITY);
    const int parts = s.count();
    float M, L, *w = s_w[WARPS == 1 ? warp : 0];
    if (WARPS == 1 || warp == 0) sums(s, w, M, L);
    if (WARPS > 1) {
        __shared__ float s_total[2];
        if (tid == 0) { s_total[0] = M; s_total[1] = L; }
        __syncthreads();
        M = s_total[0];
        L = s_total[1];
    }
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
        for (int i0 = warp % WARPS; i0 < parts; i0 += 8 * WARPS) {               // eight parts under way
            float4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + j * WARPS;
                if (i >= parts) continue;
                const bool pre = i < s.n_pre;
                const int64_t at = pre ? s.pre0 + i * s.pre_step : s.own0 + (int64_t)(i - s.n_pre) * a.pairs;
                x[j] = *reinterpret_cast<const float4*>((pre ? po : a.part_o) + at * a.d + c);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (i0 + j * WARPS >= parts) continue;
                const float f = w[i0 + j * WARPS];
                sum.x = fmaf(f, x[j].x, sum.x); sum.y = fmaf(f, x[j].y, sum.y); sum.z = fmaf(f, x[j].z, sum.z); sum.w = fmaf(f, x[j].w, sum.w);
            }
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
    int mt, units;                                       // units: no list that there can be has more
    bool tc;
    size_t at_o, at_m, at_l, at_scores, at_pre_o, at_pre_m, at_pre_l, bytes;
};

constexpr int kSmManyPairs = 4 * kSms;                   // joined by a warp each
constexpr int kSaStreamPairs = 16;                       // pairs behind a prefix up to which it is streamed

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
    a.score_stride = (int64_t)align_up(a.capacity, 4);
    // (with a cache's rows apart the sum fits any memory; a prefix without tensor cores may be walked by many groups)
    const int64_t tiles = (int64_t)a.p_groups * a.n_kv * ceil_div(a.prefix, kSaTok) + (int64_t)a.n_seq * a.n_kv * a.c_groups * (a.capacity / kSaTok + 1);
    if (tiles > kSaMaxTiles) return CASS_ERR_UNSUPPORTED;
    a.ctas = kSms * shared_stream_per_sm(a.d, plan->mt);
    plan->units = (int)(tiles < kSaLevels * a.ctas ? tiles : kSaLevels * a.ctas);
    size_t off = 0;
    auto take = [&](size_t b) { const size_t o2 = off; off = align_up(off + b, 256); return o2; };
    const size_t slots = (size_t)kSaLevels * a.ctas + (size_t)a.n_kv * ((size_t)a.p_groups + (size_t)a.n_seq * a.c_groups);
    plan->at_o = take(slots * a.pairs * a.d * 4);
    plan->at_m = take(slots * a.pairs * 4);
    plan->at_l = take(slots * a.pairs * 4);
    a.behind_tc = plan->tc;
    const size_t pre = plan->tc ? (size_t)shared_tc_plan(a) : 0;
    plan->at_pre_o = take(pre * a.d * 4);
    plan->at_pre_m = take(pre * 4);
    plan->at_pre_l = take(pre * 4);
    plan->at_scores = take(with_weights ? (size_t)a.n_seq * a.n_q * a.rows * a.score_stride * 4 : 0);
    plan->bytes = off < 256 ? 256 : off;
    return CASS_OK;
}

template <int DT>
static int run_shared(const SaPlan& plan, uint16_t* out, float* lse, const float* weight_in, float* weight_out, int32_t* d_status, cudaStream_t s) {
    const SharedAttn& a = plan.a;
    int rc = plan.tc ? launch_shared_prefix_tc(a, DT, d_status, s) : CASS_OK;
    if (rc) return rc;
    rc = DT == CASS_BF16 ? launch_shared_stream_bf16(a, plan.mt, plan.units, d_status, s) : launch_shared_stream_f16(a, plan.mt, plan.units, d_status, s);
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
