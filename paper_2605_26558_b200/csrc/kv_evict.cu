// Eviction from a cache: of every (sequence, KV head) the first, the last and the heaviest positions stay and move to the front.
// k_evict_select: the threshold by a radix selection of the weights' bits as ordered integers, then the positions in order.  The range
// that the weights take is cut into 2048 bins, the bin that the threshold falls into likewise, and so on: with bins of fixed bits a few were
// hit by everybody, and additions to one address of shared memory queue (3.6 clocks each; 32 heads of 32768 positions 71 us).  Weights
// without a bit set, which are many where a position got nothing, are counted by the warp while 0 lies outside the others' range; a NaN or a
// negative weight among them brings them into one bin (32 heads of 32768 positions, 90 % of them 0: 35.5 us a call, with a NaN in every head
// 40.2).  A CTA takes a (sequence, head), its keys read once and kept in registers; long caches take a cluster, and histograms and counts
// cross it through distributed shared memory.
// k_evict_move: rows by 16-byte vectors.
// Bound: the selection's latency (its passes, each a few barriers) and, for the rows, memory (a kept row is read and written once).
// 2 heads of 1152 positions 5.1 us of selection, 64 of 4095 7.2, 32 of 32768 15; the rows of the last (4096 kept of each, 67 MB in and out) 20 us.
#include <cooperative_groups.h>

#include "kernels.cuh"

namespace cg = cooperative_groups;

namespace cass {

constexpr int kEvThreads = 1024;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvMaxCluster = 8;
constexpr int kEvMaxOut = 0x7FFFFFFF - 0xFFFF;           // positions that stay, or of a cache whose weights are written: loops step past them in 32 bits
constexpr uint32_t kEvZero = 0x80000000u;                // key of a weight of 0

struct EvictArgs {
    int n_kv, capacity, budget, n_first, n_last;
};

// Larger weight, larger integer; -0 as +0, NaN 1, below every number; 0 is no key.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return w == w ? k : 1u;
}

struct EvictShared {
    uint32_t bins[2][2048];                              // this CTA's histogram, read by the others; two, so that one barrier a pass is enough
    uint32_t counts[2];                                  // positions above the threshold, at it
    uint32_t warp_sum[kEvWarps];
    uint32_t warp_above[kEvWarps], warp_equal[kEvWarps];
    uint32_t warp_low[kEvWarps], warp_high[kEvWarps];
    uint32_t range[3];                                   // of this CTA: the least and the largest key but zero's, zeros
    uint32_t digit, left, all;
};

// grid: (CTAs of a cluster, KV heads, sequences).  A warp takes a contiguous piece of its CTA's part, KEYS keys a lane; KEYS = 0: pieces of
// any length, their weights read again in every pass.
template <int KEYS>
__global__ void __launch_bounds__(kEvThreads) k_evict_select(EvictArgs a, const float* __restrict__ weight, const int32_t* __restrict__ lens,
                                                             int32_t* __restrict__ kept_all) {
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
    const int mid = n - a.n_first - a.n_last, take = a.budget - a.n_first - a.n_last;      // take < mid
    const int per = (mid - 1) / cs + 1, lo = min(rank * per, mid), m = min(per, mid - lo);  // this CTA's part of the middle
    const int piece = KEYS ? KEYS * 32 : ceil_div(ceil_div(m, kEvWarps), 32) * 32, w0 = min(warp * piece, m), w1 = min(w0 + piece, m);
    const float* w = weight + at * a.capacity + a.n_first + lo;
    uint32_t keys[KEYS ? KEYS : 1];
    if (KEYS && take) {
#pragma unroll
        for (int j = 0; j < KEYS; ++j) {
            const int i = w0 + j * 32 + lane;
            keys[j] = i < w1 ? weight_key(w[i]) : 0u;    // 0: no key
        }
    }
    // every key of the warp's piece in order, 32 at a time: f(key or 0, position)
    auto each = [&](auto f) {
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (w0 + j * 32 < w1) f(keys[j], w0 + j * 32 + lane);
        } else {
            for (int i = w0; i < w1; i += 32) f(i + lane < w1 ? weight_key(w[i + lane]) : 0u, i + lane);
        }
    };
    for (int i = rank * kEvThreads + tid; i < a.n_first + a.n_last; i += cs * kEvThreads) {
        if (i < a.n_first) kept[i] = i;
        else kept[a.budget - a.n_last + (i - a.n_first)] = n - a.n_last + (i - a.n_first);
    }
    if (take == 0) return;
    // ---- the range of the keys other than zero's ----
    uint32_t low = 0xFFFFFFFFu, high = 0u, zeros = 0u;
    each([&](uint32_t k, int) {
        if (k == kEvZero) ++zeros;
        else { low = min(low, k - 1u); high = max(high, k); }          // (no key: the largest value, the least)
    });
    zeros = __reduce_add_sync(0xffffffffu, zeros);
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    if (lane == 0) { sh.warp_low[warp] = low; sh.warp_high[warp] = high; sh.warp_sum[warp] = zeros; }
    __syncthreads();
    low = __reduce_min_sync(0xffffffffu, sh.warp_low[lane]);
    high = __reduce_max_sync(0xffffffffu, sh.warp_high[lane]);
    zeros = __reduce_add_sync(0xffffffffu, sh.warp_sum[lane]);
    if (cs > 1) {
        if (tid == 0) { sh.range[0] = low; sh.range[1] = high; sh.range[2] = zeros; }
        cluster.sync();
        const uint32_t* o = cluster.map_shared_rank(&sh.range[0], min(lane, cs - 1));
        low = __reduce_min_sync(0xffffffffu, o[0]);
        high = __reduce_max_sync(0xffffffffu, o[1]);
        zeros = __reduce_add_sync(0xffffffffu, lane < cs ? o[2] : 0u);
    }
    ++low;                                               // 0 and no key: there are only zeros
    const bool others = high != 0u, zero_in = others && kEvZero >= low && kEvZero <= high;
    // ---- the threshold: the least key that stays, and how many of the keys at it ----
    uint32_t threshold = kEvZero, left = (uint32_t)take, base = low, span = high - low;
    int shift = others ? max(32 - __clz(span) - 11, 0) : 0;
    bool search = others;
    if (others && !zero_in && kEvZero > high) {          // zeros above all others
        if (left <= zeros) search = false;
        else left -= zeros;
    }
#pragma unroll 1
    for (int pass = 0; search; ++pass) {
        uint32_t* bins = sh.bins[pass & 1];
        reinterpret_cast<uint2*>(bins)[tid] = make_uint2(0u, 0u);
        __syncthreads();
        each([&](uint32_t k, int) {
            if (k - base <= span) atomicAdd(&bins[(k - base) >> shift], 1u);
        });
        if (cs > 1) cluster.sync();
        else __syncthreads();
        // two bins a thread, from the largest down
        uint32_t v0 = 0, v1 = 0;
        for (int c = 0; c < cs; ++c) {
            const uint32_t* from = cs > 1 ? cluster.map_shared_rank(bins, c) : bins;
            const uint2 x = reinterpret_cast<const uint2*>(from)[1023 - tid];
            v0 += x.y;
            v1 += x.x;
        }
        uint32_t upto = v0 + v1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) sh.warp_sum[warp] = upto;
        __syncthreads();
        const uint32_t sums = sh.warp_sum[lane], before = upto - v0 - v1 + __reduce_add_sync(0xffffffffu, lane < warp ? sums : 0u);
        if (pass == 0 && !zero_in && kEvZero < low) {    // zeros below all others
            const uint32_t all = __reduce_add_sync(0xffffffffu, sums);
            if (left > all) { left -= all; break; }
        }
        if (before < left && left <= before + v0 + v1) { // one thread: the count reaches `left` in one of its bins
            const bool first = left <= before + v0;
            sh.digit = 2047 - 2 * tid - (first ? 0 : 1);
            sh.left = left - before - (first ? 0u : v0);
            sh.all = sh.left == (first ? v0 : v1);
        }
        __syncthreads();
        base += sh.digit << shift;
        left = sh.left;
        threshold = base;
        if (sh.all || shift == 0) break;                 // the whole bin stays, from its lowest key on; or it has one key only
        span = min((1u << shift) - 1u, high - base);     // (zeros may lie right behind the largest key, in its bin)
        shift = max(shift - 11, 0);
    }
    // all above the threshold stay, and the first `left` at it
    uint32_t above = 0, equal = 0;
    each([&](uint32_t k, int) {
        above += k > threshold;
        equal += k == threshold;
    });
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) { sh.warp_above[warp] = above; sh.warp_equal[warp] = equal; }
    __syncthreads();
    // what lies before this warp: in its CTA, and in the CTAs before it
    uint32_t a0 = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_above[lane] : 0u), e0 = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_equal[lane] : 0u);
    if (cs > 1) {
        if (tid == kEvThreads - 1) { sh.counts[0] = a0 + above; sh.counts[1] = e0 + equal; }
        cluster.sync();
        const uint32_t* o = cluster.map_shared_rank(&sh.counts[0], min(lane, cs - 1));
        a0 += __reduce_add_sync(0xffffffffu, lane < rank ? o[0] : 0u);
        e0 += __reduce_add_sync(0xffffffffu, lane < rank ? o[1] : 0u);
    }
    const uint32_t lt = lanemask_lt();
    int32_t* out = kept + a.n_first;
    each([&](uint32_t k, int i) {
        const uint32_t ga = __ballot_sync(0xffffffffu, k > threshold), ge = __ballot_sync(0xffffffffu, k == threshold);
        if (!(ga | ge)) return;
        const uint32_t eq = e0 + __popc(ge & lt);        // ties before this position
        if (k > threshold || (k == threshold && eq < left)) out[a0 + __popc(ga & lt) + min(eq, left)] = a.n_first + lo + i;
        a0 += __popc(ga);
        e0 += __popc(ge);
    });
    if (cs > 1) cluster.sync();                          // nobody leaves while its counts may be read
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

// CTAs of a cluster.  Two or more where each still has 4096 positions or more (below that the cluster's barriers cost more than the
// keys that a CTA has less: 64 heads of 4095 positions by pairs of CTAs 32.1 us, by one each 30.7) and every CTA has an SM; more where the
// keys would not fit the registers (32 heads of 32768 by four CTAs of 8 keys a thread 37.0 us, by one of 32 74).
static int evict_cluster(const EvictArgs& a, int n_seq) {
    int cs = 1;
    const int64_t capacity = a.capacity;                 // up to 2^31 - 1
    while (cs < kEvMaxCluster && capacity / (cs * 2) >= 4 * kEvThreads && (int64_t)n_seq * a.n_kv * cs * 2 <= kSms) cs *= 2;
    while (cs < kEvMaxCluster && capacity > (int64_t)cs * kEvThreads * 16) cs *= 2;
    return cs;
}

template <int KEYS>
static int launch_select(const EvictArgs& a, int n_seq, int cs, const float* weight, const int32_t* lens, int32_t* kept, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cs, a.n_kv, n_seq); cfg.blockDim = dim3(kEvThreads); cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = pdl_enabled();
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cs; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, k_evict_select<KEYS>, a, weight, lens, kept) != cudaSuccess) return CASS_ERR_CUDA;
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
    if (k_out == v_out) return CASS_ERR_INVALID_ARG;     // two CTAs would move the same rows
    if (((uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)k_out | (uintptr_t)v_out) & 15) return CASS_ERR_INVALID_ARG;
    if (((uintptr_t)weight | (uintptr_t)weight_out | (uintptr_t)lens | (uintptr_t)kept | (uintptr_t)new_lens) & 3) return CASS_ERR_INVALID_ARG;
    if (weight_out == weight && o.capacity != g.capacity && g.n_seq * (int64_t)g.n_kv_heads > 1) return CASS_ERR_INVALID_ARG;
    if (g.head_dim % 8 || g.head_dim > 512 || g.n_seq > 65535 || g.n_kv_heads > 65535) return CASS_ERR_UNSUPPORTED;
    if (budget > kEvMaxOut || (weight_out && o.capacity > kEvMaxOut)) return CASS_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream_;
    const EvictArgs a{g.n_kv_heads, g.capacity, budget, n_first, n_last};
    const int cs = evict_cluster(a, g.n_seq), per = (g.capacity - 1) / cs + 1;
    const int rc = per <= kEvThreads       ? launch_select<1>(a, g.n_seq, cs, weight, lens, kept, s)
                   : per <= 2 * kEvThreads  ? launch_select<2>(a, g.n_seq, cs, weight, lens, kept, s)
                   : per <= 4 * kEvThreads  ? launch_select<4>(a, g.n_seq, cs, weight, lens, kept, s)
                   : per <= 8 * kEvThreads  ? launch_select<8>(a, g.n_seq, cs, weight, lens, kept, s)
                   : per <= 16 * kEvThreads ? launch_select<16>(a, g.n_seq, cs, weight, lens, kept, s)
                                            : launch_select<0>(a, g.n_seq, cs, weight, lens, kept, s);
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
        // all rows of a column range by one CTA: narrow ranges, down to a sector of 32 bytes, until every SM has one.  8 heads of 128 dims,
        // 2048 of 4096 positions kept: 25.6 us by whole rows, 10.4 so; four sequences of them 25.9 and 20.6; 8192 of 32768 kept: 89 and 41
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
