// Eviction from a cache: of every (sequence, KV head) the first, the last and the heaviest positions stay and move to the front.
// k_evict_select: the threshold by a radix selection of the weights' bits as ordered integers, eight bits a pass, then the
// positions in order.  A cluster of CTAs takes a (sequence, head), each a contiguous part of the middle, read once and kept in shared
// memory; histograms, then counts, cross the cluster through distributed shared memory.
// k_evict_move: rows by 16-byte vectors.  Bound: memory (a kept row is read and written once), and for small caches the latency of the
// selection's passes.
#include <cooperative_groups.h>

#include "kernels.cuh"

namespace cg = cooperative_groups;

namespace cass {

constexpr int kEvThreads = 512;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvKeys = 40 * 1024;                       // most keys of a CTA that stay in shared memory
constexpr int kEvMaxCluster = 8;

struct EvictArgs {
    int n_kv, capacity, budget, n_first, n_last;
};

// Larger weight, larger integer; -0 as +0, NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __float_as_uint(w);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;
    if (u == 0x80000000u) return 0x80000000u;
    return (u >> 31) ? ~u : u | 0x80000000u;
}

struct EvictShared {
    uint32_t hist[256 * 32];                             // a column a lane: the lanes of a warp never meet at an address
    uint32_t bins[2][256];                               // this CTA's sums, read by the others; two, so that one barrier a pass is enough
    uint32_t counts[2];                                  // positions above the threshold, at it
    uint32_t total[256];
    uint32_t warp_above[kEvWarps], warp_equal[kEvWarps];
    uint32_t digit, left;
};

// grid: (CTAs of a cluster, KV heads, sequences)
template <bool STAGED>
__global__ void __launch_bounds__(kEvThreads) k_evict_select(EvictArgs a, const float* __restrict__ weight, const int32_t* __restrict__ lens,
                                                             int32_t* __restrict__ kept_all) {
    extern __shared__ uint32_t s_keys[];
    __shared__ EvictShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_early<0>();
    const size_t at = (size_t)blockIdx.z * a.n_kv + blockIdx.y;
    const int n = lens[blockIdx.z];
    int32_t* kept = kept_all + at * a.budget;
    if (n < 0 || n > a.capacity || n <= a.budget) {      // the same for the whole cluster
        const int stay = n < 0 || n > a.capacity ? 0 : n;
        for (int i = rank * kEvThreads + tid; i < a.budget; i += cs * kEvThreads) kept[i] = i < stay ? i : -1;
        return;
    }
    for (int i = rank * kEvThreads + tid; i < a.n_first + a.n_last; i += cs * kEvThreads) {
        if (i < a.n_first) kept[i] = i;
        else kept[a.budget - a.n_last + (i - a.n_first)] = n - a.n_last + (i - a.n_first);
    }
    const int mid = n - a.n_first - a.n_last, take = a.budget - a.n_first - a.n_last;      // take < mid
    if (take == 0) return;
    const int per = ceil_div(mid, cs), lo = min(rank * per, mid), m = min(per, mid - lo);  // this CTA's part of the middle
    const float* w = weight + at * a.capacity + a.n_first + lo;
    if (STAGED)
        for (int i = tid; i < m; i += kEvThreads) s_keys[i] = weight_key(w[i]);
    auto key = [&](int i) { return STAGED ? s_keys[i] : weight_key(w[i]); };
    uint32_t prefix = 0, left = (uint32_t)take;          // the threshold's bits so far; how many of the keys that share them stay
#pragma unroll 1
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        for (int i = tid; i < 256 * 32; i += kEvThreads) sh.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < m; i += kEvThreads) {
            const uint32_t k = key(i);
            if (pass == 0 || (k >> (shift + 8)) == prefix) atomicAdd(&sh.hist[((k >> shift) & 255u) * 32 + lane], 1u);
        }
        __syncthreads();
        for (int b = warp; b < 256; b += kEvWarps) {
            const uint32_t v = __reduce_add_sync(0xffffffffu, sh.hist[b * 32 + lane]);
            if (lane == 0) sh.bins[pass & 1][b] = v;
        }
        cluster.sync();
        if (tid < 256) {
            uint32_t v = 0;
            for (int c = 0; c < cs; ++c) v += cluster.map_shared_rank(&sh.bins[pass & 1][0], c)[tid];
            sh.total[tid] = v;
        }
        __syncthreads();
        if (warp == 0) {
            // bins from the largest down, eight a lane; the one in which the count reaches `left`
            uint32_t v[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) { v[i] = sh.total[255 - (lane * 8 + i)]; sum += v[i]; }
            uint32_t before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += x;
            }
            before -= sum;
            if (before < left && left <= before + sum) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (before < left && left <= before + v[i]) { sh.digit = 255 - (lane * 8 + i); sh.left = left - before; }
                    before += v[i];
                }
            }
        }
        __syncthreads();
        prefix = (prefix << 8) | sh.digit;
        left = sh.left;
    }
    // `prefix` is the threshold: all above it stay, and the first `left` at it.  A warp takes a contiguous piece of the part.
    const int piece = ceil_div(ceil_div(m, kEvWarps), 32) * 32, w0 = min(warp * piece, m), w1 = min(w0 + piece, m);
    uint32_t above = 0, equal = 0;
    for (int i = w0; i < w1; i += 32) {
        const bool in = i + lane < w1;
        const uint32_t k = in ? key(i + lane) : 0u;
        above += __popc(__ballot_sync(0xffffffffu, in && k > prefix));
        equal += __popc(__ballot_sync(0xffffffffu, in && k == prefix));
    }
    if (lane == 0) { sh.warp_above[warp] = above; sh.warp_equal[warp] = equal; }
    __syncthreads();
    if (tid == 0) {
        uint32_t x = 0, y = 0;
        for (int i = 0; i < kEvWarps; ++i) { x += sh.warp_above[i]; y += sh.warp_equal[i]; }
        sh.counts[0] = x;
        sh.counts[1] = y;
    }
    cluster.sync();
    uint32_t a0 = 0, e0 = 0;                             // above and at the threshold before this warp's piece
    for (int c = 0; c < rank; ++c) {
        const uint32_t* o = cluster.map_shared_rank(&sh.counts[0], c);
        a0 += o[0];
        e0 += o[1];
    }
    for (int i = 0; i < warp; ++i) { a0 += sh.warp_above[i]; e0 += sh.warp_equal[i]; }
    const uint32_t lt = lanemask_lt();
    int32_t* out = kept + a.n_first;
    for (int i = w0; i < w1; i += 32) {
        const bool in = i + lane < w1;
        const uint32_t k = in ? key(i + lane) : 0u;
        const uint32_t ga = __ballot_sync(0xffffffffu, in && k > prefix), ge = __ballot_sync(0xffffffffu, in && k == prefix);
        const uint32_t eq = e0 + __popc(ge & lt);        // ties before this position
        const bool stay = in && (k > prefix || (k == prefix && eq < left));
        if (stay) out[a0 + __popc(ga & lt) + min(eq, left)] = a.n_first + lo + i + lane;
        a0 += __popc(ga);
        e0 += __popc(ge);
    }
    cluster.sync();                                      // nobody leaves while its counts may be read
}

// ---- moving what stays ----
constexpr int kEvMoveThreads = 256;
constexpr int kEvMoveUnroll = 8;

struct EvictMove {
    const uint8_t *k, *v;
    uint8_t *k_out, *v_out;
    int64_t seq, pos, head, seq_out, pos_out, head_out;              // bytes
    const float* weight;
    float* weight_out;
    int n_kv, capacity, capacity_out, budget;
    int cols, parts, rows;                                           // vectors of a row a CTA takes; CTAs a row; rows a CTA
};

// grid: (parts x row ranges x {K, V} + weights and lengths, KV heads, sequences).  In place a CTA takes all rows of its columns in order:
// row j comes from a place >= j, so what a round writes was read in it or before, and no later round reads it.
__global__ void __launch_bounds__(kEvMoveThreads) k_evict_move(EvictMove a, const int32_t* lens, const int32_t* __restrict__ kept_all,
                                                               int32_t* new_lens) {
    pdl_wait();
    pdl_early<0>();
    const int tid = threadIdx.x, head = blockIdx.y, seq = blockIdx.z;
    const int n = *reinterpret_cast<const volatile int32_t*>(lens + seq);          // or min(n, budget), if new_lens = lens is written by now
    const size_t at = (size_t)seq * a.n_kv + head;
    const int32_t* __restrict__ kept = kept_all + at * a.budget;
    const bool there = n >= 0 && n <= a.capacity;
    const int count = there ? min(n, a.budget) : 0;
    if (blockIdx.x == gridDim.x - 1) {
        if (head == 0 && tid == 0) new_lens[seq] = there ? count : n;
        if (!there || !a.weight_out) return;
        const float* from = a.weight + at * a.capacity;
        float* to = a.weight_out + at * a.capacity_out;
        for (int j0 = tid; j0 < ceil_div(count, kEvMoveThreads) * kEvMoveThreads; j0 += kEvMoveThreads * kEvMoveUnroll) {
            float x[kEvMoveUnroll];
#pragma unroll
            for (int i = 0; i < kEvMoveUnroll; ++i) {
                const int j = j0 + i * kEvMoveThreads;
                if (j < count) x[i] = from[kept[j]];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kEvMoveUnroll; ++i) {
                const int j = j0 + i * kEvMoveThreads;
                if (j < count) to[j] = x[i];
            }
        }
        __syncthreads();
        for (int j = count + tid; j < a.capacity_out; j += kEvMoveThreads) to[j] = 0.f;
        return;
    }
    const int part = blockIdx.x % a.parts, rest = blockIdx.x / a.parts;
    const bool is_v = rest & 1;
    const int first = (rest >> 1) * a.rows, last = min(first + a.rows, count);
    const int c = tid % a.cols, y = tid / a.cols, ny = kEvMoveThreads / a.cols;
    const int64_t col = ((int64_t)part * a.cols + c) * 16;
    const uint8_t* from = (is_v ? a.v : a.k) + (int64_t)seq * a.seq + (int64_t)head * a.head + col;
    uint8_t* to = (is_v ? a.v_out : a.k_out) + (int64_t)seq * a.seq_out + (int64_t)head * a.head_out + col;
    for (int j0 = first; j0 < last; j0 += ny * kEvMoveUnroll) {      // the same rounds for all threads: there is a barrier in them
        uint4 x[kEvMoveUnroll];
        int src[kEvMoveUnroll];
#pragma unroll
        for (int i = 0; i < kEvMoveUnroll; ++i) {
            const int j = j0 + i * ny + y;
            src[i] = y < ny && j < last ? kept[j] : -1;
            if (from == to && src[i] == j) src[i] = -1;              // it is there
        }
#pragma unroll
        for (int i = 0; i < kEvMoveUnroll; ++i)
            if (src[i] >= 0) x[i] = *reinterpret_cast<const uint4*>(from + src[i] * a.pos);
        if (from == to) __syncthreads();
#pragma unroll
        for (int i = 0; i < kEvMoveUnroll; ++i)
            if (src[i] >= 0) *reinterpret_cast<uint4*>(to + (int64_t)(j0 + i * ny + y) * a.pos_out) = x[i];
    }
}

// No two rows of a cache overlap, whatever the order of its dimensions; also its alignment.
bool cache_geom_ok(const cass_cache_geom& g, bool any) {
    if (g.dtype != CASS_BF16 && g.dtype != CASS_F16) return false;
    if (g.n_seq < 1 || g.n_kv_heads < 1 || g.head_dim < 1 || g.capacity < (any ? 0 : 1)) return false;
    if (g.seq_stride < 0 || g.pos_stride < 0 || g.head_stride < 0 || (g.seq_stride | g.pos_stride | g.head_stride) % 8) return false;
    if (g.capacity == 0) return true;
    // dimensions by growing stride: each clears what the smaller ones span
    struct { int64_t stride, n; } d[3] = {{g.seq_stride, g.n_seq}, {g.pos_stride, g.capacity}, {g.head_stride, g.n_kv_heads}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (d[j].n <= 1 ? false : (d[j + 1].n <= 1 || d[j].stride > d[j + 1].stride)) { auto t = d[j]; d[j] = d[j + 1]; d[j + 1] = t; }
    int64_t span = g.head_dim;
    for (const auto& x : d) {
        if (x.n <= 1) continue;
        if (x.stride < span || x.stride > ((int64_t)1 << 46) / x.n) return false;
        span += x.stride * (x.n - 1);
    }
    return true;
}

static int evict_cluster(const EvictArgs& a, int n_seq) {
    int cs = 1;                                          // parts of at least 2048 positions, one CTA an SM
    while (cs < kEvMaxCluster && a.capacity / (cs * 2) >= 2048 && (int64_t)n_seq * a.n_kv * cs * 2 <= kSms) cs *= 2;
    while (cs < kEvMaxCluster && ceil_div(a.capacity, cs) > kEvKeys) cs *= 2;
    return cs;
}

template <bool STAGED>
static int launch_select(const EvictArgs& a, int n_seq, int cs, size_t smem, const float* weight, const int32_t* lens, int32_t* kept, cudaStream_t s) {
    CASS_ALLOW_SMEM(k_evict_select<STAGED>);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cs, a.n_kv, n_seq); cfg.blockDim = dim3(kEvThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = pdl_enabled();
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cs; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, k_evict_select<STAGED>, a, weight, lens, kept) != cudaSuccess) return CASS_ERR_CUDA;
    return CASS_OK;
}

}  // namespace cass

using namespace cass;

extern "C" int cass_kv_evict(const cass_cache_geom* cache, void* k_cache, void* v_cache, const float* weight, const int32_t* lens, int budget,
                             int n_first, int n_last, const cass_cache_geom* cache_out, void* k_out, void* v_out, float* weight_out, int32_t* kept,
                             int32_t* new_lens, void* stream_) {
    if (!cache || !k_cache || !v_cache || !weight || !lens || !kept || !new_lens || !cache_geom_ok(*cache, false)) return CASS_ERR_INVALID_ARG;
    const bool in_place = !cache_out;
    if (in_place ? (k_out || v_out) : (!k_out || !v_out || !cache_geom_ok(*cache_out, false))) return CASS_ERR_INVALID_ARG;
    const cass_cache_geom &g = *cache, &o = in_place ? *cache : *cache_out;
    if (o.dtype != g.dtype || o.n_seq != g.n_seq || o.n_kv_heads != g.n_kv_heads || o.head_dim != g.head_dim) return CASS_ERR_INVALID_ARG;
    if (budget < 1 || budget > o.capacity || n_first < 0 || n_last < 0 || n_first > budget || n_last > budget - n_first) return CASS_ERR_INVALID_ARG;
    if (in_place) { k_out = k_cache; v_out = v_cache; }
    else if (k_out == k_cache || v_out == v_cache || k_out == v_cache || v_out == k_cache) return CASS_ERR_INVALID_ARG;
    if (((uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)k_out | (uintptr_t)v_out) & 15) return CASS_ERR_INVALID_ARG;
    if (((uintptr_t)weight | (uintptr_t)weight_out | (uintptr_t)lens | (uintptr_t)kept | (uintptr_t)new_lens) & 3) return CASS_ERR_INVALID_ARG;
    if (weight_out == weight && o.capacity != g.capacity && g.n_seq * (int64_t)g.n_kv_heads > 1) return CASS_ERR_INVALID_ARG;
    if (g.head_dim % 8 || g.head_dim > 512 || g.n_seq > 65535 || g.n_kv_heads > 65535) return CASS_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream_;
    const EvictArgs a{g.n_kv_heads, g.capacity, budget, n_first, n_last};
    const int cs = evict_cluster(a, g.n_seq), per = ceil_div(g.capacity, cs);
    const int rc = per <= kEvKeys ? launch_select<true>(a, g.n_seq, cs, (size_t)per * 4, weight, lens, kept, s)
                                  : launch_select<false>(a, g.n_seq, cs, 0, weight, lens, kept, s);
    if (rc) return rc;
    EvictMove m{};
    m.k = (const uint8_t*)k_cache; m.v = (const uint8_t*)v_cache; m.k_out = (uint8_t*)k_out; m.v_out = (uint8_t*)v_out;
    m.seq = g.seq_stride * 2; m.pos = g.pos_stride * 2; m.head = g.head_stride * 2;
    m.seq_out = o.seq_stride * 2; m.pos_out = o.pos_stride * 2; m.head_out = o.head_stride * 2;
    m.weight = weight; m.weight_out = weight_out;
    m.n_kv = g.n_kv_heads; m.capacity = g.capacity; m.capacity_out = o.capacity; m.budget = budget;
    const int vecs = g.head_dim / 8;
    m.cols = vecs;
    m.rows = budget;
    if (in_place) {
        // all rows of a column range by one CTA: narrow ranges, down to a sector of 32 bytes, until every SM has one
        while (m.cols % 2 == 0 && m.cols > 2 && (int64_t)g.n_seq * g.n_kv_heads * 2 * (vecs / m.cols) < kSms) m.cols /= 2;
    } else {
        m.rows = kEvMoveThreads / m.cols * kEvMoveUnroll;
    }
    m.parts = vecs / m.cols;
    const int64_t blocks = (int64_t)m.parts * 2 * ceil_div(budget, m.rows) + 1;
    if (blocks > 0x7FFFFFFF) return CASS_ERR_UNSUPPORTED;
    CASS_PDL_LAUNCH(k_evict_move, dim3((unsigned)blocks, g.n_kv_heads, g.n_seq), dim3(kEvMoveThreads), 0, s, m, lens, kept, new_lens);
    return CASS_OK;
}
