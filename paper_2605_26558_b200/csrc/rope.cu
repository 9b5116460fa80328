// Rotary positions of queries and keys in the caller's layout: y = g (cos t, -sin t; sin t, cos t) (a, b) for every pair of a head,
// t = position * frequency of the pair.
// Bound: memory (each value read and written once).  A CTA takes the rows whose sines and cosines its threads form in one go, one
// (row, pair) a thread: the angle in 64 bits, reduced there to a quarter turn, then sincospif of at most 1/4, so that no table bounds the
// positions.  The product with the frequency (itself rounded, of a power good to a unit or two), and that with 1 / pi, are off by a few 2^-53 of the
// angle: less than the sine's own 2^-24 up to some 2^27 radians, up to 2^-20 at 2^31.  All heads of the row share them
// through shared memory; a thread's values travel while they are formed.  8191 rows of 40 half-rotated heads of 128 into other tensors 28.6 us, 5.9 TB/s, 90 % of a copy's
// rate; the gradient of 32768 fp32 rows of 48 heads 234 us, 6.9 TB/s, a little above a copy's.
#include <cmath>
#include <cuda_fp16.h>

#include "kernels.cuh"

namespace cass {

// ---- frequencies ----

bool rope_params_ok(const cass_rope_params& p) {
    if (p.rot_dim < 2 || p.rot_dim % 2 || p.scaling < CASS_ROPE_PLAIN || p.scaling > CASS_ROPE_YARN) return false;
    if (!(p.theta > 1.0) || !std::isfinite(p.theta) || !(p.gain >= 0.0) || !std::isfinite(p.gain)) return false;
    if (p.scaling != CASS_ROPE_PLAIN && (!(p.factor > 0.0) || !std::isfinite(p.factor))) return false;
    if (p.scaling == CASS_ROPE_NTK && p.rot_dim <= 2) return false;
    if (p.scaling == CASS_ROPE_BANDS || p.scaling == CASS_ROPE_YARN)
        return p.low > 0.0 && p.high > p.low && std::isfinite(p.high) && p.trained_len > 0.0 && std::isfinite(p.trained_len);
    return true;
}

__device__ double rope_frequency(const cass_rope_params& p, int j) {
    constexpr double kTwoPi = 6.283185307179586476925;
    const double r = (double)p.rot_dim;
    const double theta = p.scaling == CASS_ROPE_NTK ? p.theta * pow(p.factor, r / (r - 2.0)) : p.theta;
    const double f = pow(theta, -2.0 * (double)j / r);
    if (p.scaling == CASS_ROPE_LINEAR) return f / p.factor;
    if (p.scaling == CASS_ROPE_BANDS) {
        const double turns = p.trained_len * f / kTwoPi, m = fmin(fmax((turns - p.low) / (p.high - p.low), 0.0), 1.0);
        return m * f + (1.0 - m) * f / p.factor;
    }
    if (p.scaling == CASS_ROPE_YARN) {
        const double half = r / (2.0 * log(p.theta));                   // pair that makes u turns: half * ln(trained_len / (2 pi u))
        const double a = fmax(floor(half * log(p.trained_len / (kTwoPi * p.high))), 0.0);
        const double b = fmin(ceil(half * log(p.trained_len / (kTwoPi * p.low))), r - 1.0);
        const double m = fmin(fmax(((double)j - a) / fmax(b - a, 0.001), 0.0), 1.0);
        return m * f / p.factor + (1.0 - m) * f;
    }
    return f;
}

__device__ double rope_gain(const cass_rope_params& p) {
    if (p.gain > 0.0) return p.gain;
    return p.scaling == CASS_ROPE_YARN && p.factor > 1.0 ? 0.1 * log(p.factor) + 1.0 : 1.0;
}

__global__ void k_rope_freqs(cass_rope_params p, double* __restrict__ freqs) {
    const int half = p.rot_dim / 2;
    for (int j = blockIdx.x * blockDim.x + threadIdx.x; j <= half; j += gridDim.x * blockDim.x) freqs[j] = j < half ? rope_frequency(p, j) : rope_gain(p);
}

// The session's tables: cosines and sines of every position and pair.
__global__ void k_rope_table(float* __restrict__ cos_t, float* __restrict__ sin_t, int max_seq, cass_rope_params p) {
    const int half = p.rot_dim / 2;
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (size_t)max_seq * half) return;
    const double ang = (double)(int)(i / half) * rope_frequency(p, (int)(i % half)), gain = rope_gain(p);
    cos_t[i] = (float)(cos(ang) * gain);
    sin_t[i] = (float)(sin(ang) * gain);
}

int launch_rope_table(float* cos_t, float* sin_t, int max_seq, const cass_rope_params& p, cudaStream_t s) {
    const size_t n = (size_t)max_seq * (p.rot_dim / 2);
    k_rope_table<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(cos_t, sin_t, max_seq, p);
    CASS_LAUNCH_CHECK();
    return CASS_OK;
}

// ---- rotation ----

constexpr int kRopeThreads = 256;
constexpr int kRopeUnroll = 4;             // (row, head, slot) items of a thread under way

// cos and sin of position * frequency.
__device__ __forceinline__ float2 rope_turn(int pos, double f) {
    double h = (double)pos * f * 0.318309886183790671538;               // half turns
    h -= 2.0 * rint(0.5 * h);                                           // -1 .. 1
    const double q = rint(2.0 * h);                                     // quarter turns
    float s, c;
    sincospif((float)(h - 0.5 * q), &s, &c);
    const int n = (int)q & 3;
    const float cc = (n & 1) ? s : c, ss = (n & 1) ? c : s;
    return make_float2(n == 1 || n == 2 ? -cc : cc, n >= 2 ? -ss : ss);
}

// Two neighbouring values: a 32-bit word of a 16-bit type, or two of fp32.
template <class T> struct RopeTwo;
template <> struct RopeTwo<__nv_bfloat16> {
    using Raw = uint32_t;
    static __device__ __forceinline__ float2 get(Raw w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ Raw put(float2 v) {
        Raw r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(v.y), "f"(v.x));
        return r;
    }
};
template <> struct RopeTwo<__half> {
    using Raw = uint32_t;
    static __device__ __forceinline__ float2 get(Raw w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ Raw put(float2 v) {
        Raw r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(v.y), "f"(v.x));
        return r;
    }
};
template <> struct RopeTwo<float> {
    using Raw = float2;
    static __device__ __forceinline__ float2 get(Raw w) { return w; }
    static __device__ __forceinline__ Raw put(float2 v) { return v; }
};
__device__ __forceinline__ float rope_get(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float rope_get(__half v) { return __half2float(v); }
__device__ __forceinline__ float rope_get(float v) { return v; }
__device__ __forceinline__ void rope_put(__nv_bfloat16& to, float v) { to = __float2bfloat16_rn(v); }
__device__ __forceinline__ void rope_put(__half& to, float v) { to = __float2half_rn(v); }
__device__ __forceinline__ void rope_put(float& to, float v) { to = v; }

template <class T, int V> struct RopeVec { struct alignas(sizeof(T) * V) Type { typename RopeTwo<T>::Raw w[V / 2]; }; };
template <class T> struct RopeVec<T, 1> { using Type = T; };

struct RopeArgs {
    cass_rope_geom g;
    int rows, per_cta;                     // rows; rows a CTA takes
    int slots, rot_slots;                  // 2 V values each: all of a head's, and those of its pairs (the rest is copied)
    int transpose;
    int lanes, step_rows, step_heads;      // slots side by side; the distance of a thread's items
};

// A slot is V pairs, 2 V values: two vectors half a rotation apart, or side by side where pairs are interleaved (IL) or copied.
// Sines and cosines lie as a warp's lanes read them: of two pairs together, slot after slot.
// Single values and a runtime choice of the layout inside one kernel took 256 instructions a slot of eight pairs and its place in local
// memory: 8191 rows of 40 half-rotated heads 73 us.
template <class T, int V, bool IL>
__global__ void __launch_bounds__(kRopeThreads, 4) k_rope(RopeArgs a, const double* __restrict__ freqs, const int32_t* __restrict__ positions,
                                                          const T* q, const T* k, T* q_out, T* k_out) {
    extern __shared__ __align__(16) float s_turn[];
    using Vec = typename RopeVec<T, V>::Type;
    const int tid = threadIdx.x, half = a.g.rot_dim / 2, heads = a.g.n_q_heads + a.g.n_k_heads;
    const int row0 = blockIdx.x * a.per_cta, rows = min(a.per_cta, a.rows - row0);
    const int y = tid / a.lanes, x0 = tid - y * a.lanes, ny = kRopeThreads / a.lanes;
    const int r0 = y / heads, h0 = y - r0 * heads;
    const bool works = y < ny;
    pdl_wait();
    pdl_early<0>();
    Vec vl[kRopeUnroll], vh[kRopeUnroll];
    auto place = [&](int x, int& lo, int& hi) {                         // where the slot's two vectors begin within a head
        const bool apart = !IL && x < a.rot_slots;
        lo = apart ? x * V : x * 2 * V;
        hi = apart ? half + x * V : lo + V;
    };
    auto step = [&](int& row, int& head) {
        row += a.step_rows;
        head += a.step_heads;
        if (head >= heads) { head -= heads; ++row; }
    };
    auto load = [&](int x, int row, int head) {                         // kRopeUnroll items from (row, head) on
        int lo, hi;
        place(x, lo, hi);
#pragma unroll
        for (int i = 0; i < kRopeUnroll; ++i) {
            if (row < rows) {
                const int kh = head - a.g.n_q_heads;
                const int64_t r = row0 + row;
                const T* from = kh < 0 ? q + r * a.g.q_row + head * a.g.q_head : k + r * a.g.k_row + kh * a.g.k_head;
                if (V > 1 || lo < a.g.head_dim) vl[i] = *reinterpret_cast<const Vec*>(from + lo);
                if (V > 1 || hi < a.g.head_dim) vh[i] = *reinterpret_cast<const Vec*>(from + hi);
            }
            step(row, head);
        }
    };
    if (works && x0 < a.slots) load(x0, r0, h0);                        // they travel while the sines are formed
    const float gain = (float)freqs[half];
    for (int i = tid; i < rows * half; i += kRopeThreads) {
        const int r = i / half, j = i - r * half;
        float2 t = rope_turn(positions ? positions[row0 + r] : row0 + r, freqs[j]);
        if (a.transpose) t.y = -t.y;
        const int at = V == 1 ? i : ((r * (V / 2) + j % V / 2) * a.rot_slots + j / V) * 2 + (j & 1);
        reinterpret_cast<float2*>(s_turn)[at] = make_float2(t.x * gain, t.y * gain);
    }
    __syncthreads();
    if (!works) return;
    for (int x = x0; x < a.slots; x += a.lanes) {
        const bool turns = x < a.rot_slots;
        int lo, hi, row = r0, head = h0;
        place(x, lo, hi);
        while (row < rows) {
            if (x != x0 || row != r0 || head != h0) load(x, row, head);
#pragma unroll
            for (int i = 0; i < kRopeUnroll; ++i) {
                if (row < rows) {
                    if (turns) {
                        if constexpr (V == 1) {
                            const float2 t = reinterpret_cast<const float2*>(s_turn)[row * half + x];
                            const float2 r = rope_pair(rope_get(vl[i]), rope_get(vh[i]), t.x, t.y);
                            rope_put(vl[i], r.x);
                            rope_put(vh[i], r.y);
                        } else {
                            const float4* turn = reinterpret_cast<const float4*>(s_turn) + row * (V / 2) * a.rot_slots + x;
#pragma unroll
                            for (int w = 0; w < V / 2; ++w) {
                                const float4 t = turn[w * a.rot_slots];                  // pairs 2 w and 2 w + 1
                                if constexpr (IL) {
                                    // words 2 w and 2 w + 1 of the slot's V: a pair each
                                    auto& first = 2 * w < V / 2 ? vl[i].w[2 * w % (V / 2)] : vh[i].w[2 * w % (V / 2)];
                                    auto& second = 2 * w + 1 < V / 2 ? vl[i].w[(2 * w + 1) % (V / 2)] : vh[i].w[(2 * w + 1) % (V / 2)];
                                    const float2 u = RopeTwo<T>::get(first), v = RopeTwo<T>::get(second);
                                    first = RopeTwo<T>::put(rope_pair(u.x, u.y, t.x, t.y));
                                    second = RopeTwo<T>::put(rope_pair(v.x, v.y, t.z, t.w));
                                } else {
                                    const float2 u = RopeTwo<T>::get(vl[i].w[w]), v = RopeTwo<T>::get(vh[i].w[w]);
                                    const float2 e = rope_pair(u.x, v.x, t.x, t.y), f = rope_pair(u.y, v.y, t.z, t.w);
                                    vl[i].w[w] = RopeTwo<T>::put(make_float2(e.x, f.x));
                                    vh[i].w[w] = RopeTwo<T>::put(make_float2(e.y, f.y));
                                }
                            }
                        }
                    }
                    const int kh = head - a.g.n_q_heads;
                    const int64_t r = row0 + row;
                    T* to = kh < 0 ? q_out + r * a.g.q_out_row + head * a.g.q_out_head : k_out + r * a.g.k_out_row + kh * a.g.k_out_head;
                    if (V > 1 || lo < a.g.head_dim) *reinterpret_cast<Vec*>(to + lo) = vl[i];
                    if (V > 1 || hi < a.g.head_dim) *reinterpret_cast<Vec*>(to + hi) = vh[i];
                }
                step(row, head);
            }
        }
    }
}

// Cells of `inner` values at row_stride * row + head_stride * head that do not overlap.
static bool cells_apart(int64_t rows, int64_t heads, int64_t row_stride, int64_t head_stride, int64_t inner) {
    if (row_stride < 0 || head_stride < 0) return false;
    if (rows <= 1) return heads <= 1 || head_stride >= inner;
    if (heads <= 1) return row_stride >= inner;
    if (head_stride >= inner && row_stride >= (heads - 1) * head_stride + inner) return true;
    return row_stride >= inner && head_stride >= (rows - 1) * row_stride + inner;
}

template <class T, int V>
static int run_rope(RopeArgs a, const double* freqs, const int32_t* positions, const void* q, const void* k, void* q_out, void* k_out, int copied,
                    cudaStream_t s) {
    const int half = a.g.rot_dim / 2, heads = a.g.n_q_heads + a.g.n_k_heads;
    a.rot_slots = half / V;
    a.slots = a.rot_slots + ceil_div(copied, 2 * V);
    a.lanes = a.slots < kRopeThreads ? a.slots : kRopeThreads;
    const int ny = kRopeThreads / a.lanes;
    a.step_rows = ny / heads;
    a.step_heads = ny % heads;
    a.per_cta = half >= kRopeThreads ? 1 : kRopeThreads / half;
    // By vectors, no more rows than a thread has items under way: a CTA's loads all travel while its sines are formed.  8191 rows of 40
    // half-rotated heads 28.6 us, with all rows whose sines its threads form in one go 31.4; 32768 fp32 rows of 48 heads 234 and 244; by two
    // values 8191 whole heads 51 and 44, by single ones 82 and 77.  Three items in five CTAs an SM took 29.5 and 235, eight in two 32.6 and 241.
    if (V * sizeof(T) == 16) {
        const int fit = kRopeUnroll * ny / heads;
        if (a.per_cta > fit) a.per_cta = fit > 1 ? fit : 1;
    }
    // few rows: all SMs before full CTAs (148 rows of 40 heads of 128: 4.7 us by full CTAs, 3.1 so)
    const auto groups = [&](int of) { return (int)(((int64_t)a.rows + of - 1) / of); };          // (rows may be 2^31 - 1)
    if (a.per_cta > groups(kSms)) a.per_cta = groups(kSms);
    const size_t smem = (size_t)a.per_cta * half * sizeof(float2);
    const dim3 grid(groups(a.per_cta));
    if (a.g.interleaved)
        CASS_PDL_LAUNCH((k_rope<T, V, true>), grid, dim3(kRopeThreads), smem, s, a, freqs, positions, (const T*)q, (const T*)k, (T*)q_out, (T*)k_out);
    else
        CASS_PDL_LAUNCH((k_rope<T, V, false>), grid, dim3(kRopeThreads), smem, s, a, freqs, positions, (const T*)q, (const T*)k, (T*)q_out, (T*)k_out);
    return CASS_OK;
}

// 16-byte vectors where sizes, strides and places allow them, else words of two 16-bit values, else single values: 8191 rows of 40 heads
// of 128 in place 24, 44 and 77 us.
template <class T>
static int choose_rope(const cass_rope_geom& g, const double* freqs, const int32_t* positions, int rows, const void* q, const void* k, void* q_out,
                       void* k_out, int transpose, cudaStream_t s) {
    RopeArgs a{};
    a.g = g;
    a.rows = rows;
    a.transpose = transpose;
    const bool in_place = (!q || q == q_out) && (!k || k == k_out);
    const int copied = in_place ? 0 : g.head_dim - g.rot_dim;            // values behind the pairs that have to move
    int64_t strides = 0;
    if (q) strides |= g.q_row | g.q_head | g.q_out_row | g.q_out_head;
    if (k) strides |= g.k_row | g.k_head | g.k_out_row | g.k_out_head;
    const uintptr_t at = (uintptr_t)q | (uintptr_t)k | (uintptr_t)q_out | (uintptr_t)k_out;
    auto fits = [&](int v) { return g.rot_dim / 2 % v == 0 && copied % (2 * v) == 0 && strides % v == 0 && at % (v * sizeof(T)) == 0; };
    constexpr int V = 16 / sizeof(T);
    if (fits(V)) return run_rope<T, V>(a, freqs, positions, q, k, q_out, k_out, copied, s);
    if constexpr (V == 8)
        if (fits(2)) return run_rope<T, 2>(a, freqs, positions, q, k, q_out, k_out, copied, s);
    return run_rope<T, 1>(a, freqs, positions, q, k, q_out, k_out, copied, s);
}

}  // namespace cass

using namespace cass;

extern "C" int cass_rope_freqs(const cass_rope_params* params, double* freqs, void* stream_) {
    if (!params || !freqs || ((uintptr_t)freqs & 7) || !rope_params_ok(*params)) return CASS_ERR_INVALID_ARG;
    k_rope_freqs<<<1, 128, 0, (cudaStream_t)stream_>>>(*params, freqs);
    CASS_LAUNCH_CHECK();
    return CASS_OK;
}

extern "C" int cass_rope(const cass_rope_geom* geom, const double* freqs, const int32_t* positions, int rows, const void* q, const void* k,
                         void* q_out, void* k_out, int transpose, void* stream_) {
    if (!geom || !freqs || ((uintptr_t)freqs & 7) || rows < 0) return CASS_ERR_INVALID_ARG;
    cass_rope_geom g = *geom;
    if (g.dtype != CASS_BF16 && g.dtype != CASS_F16 && g.dtype != CASS_F32) return CASS_ERR_INVALID_ARG;
    if (g.rot_dim < 2 || g.rot_dim % 2 || g.head_dim < g.rot_dim || g.n_q_heads < 0 || g.n_k_heads < 0) return CASS_ERR_INVALID_ARG;
    if (g.rot_dim > 4096) return CASS_ERR_UNSUPPORTED;                   // one row's sines and cosines in shared memory
    if (g.n_q_heads == 0 && g.n_k_heads == 0) return CASS_ERR_INVALID_ARG;
    if (rows > 0) {                                                      // (tensors without rows have no address)
        if ((g.n_q_heads > 0) != (q != nullptr) || (g.n_k_heads > 0) != (k != nullptr)) return CASS_ERR_INVALID_ARG;
        if ((q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr)) return CASS_ERR_INVALID_ARG;
    }
    const int64_t heads = (int64_t)g.n_q_heads + g.n_k_heads;
    if (heads > 65535 || heads * rows > 0x7FFFFFFFll) return CASS_ERR_UNSUPPORTED;
    const uintptr_t size = g.dtype == CASS_F32 ? 4 : 2;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)q_out | (uintptr_t)k_out) % size || ((uintptr_t)positions & 3)) return CASS_ERR_INVALID_ARG;
    if (q && (g.q_row < 0 || g.q_head < 0 || !cells_apart(rows, g.n_q_heads, g.q_out_row, g.q_out_head, g.head_dim))) return CASS_ERR_INVALID_ARG;
    if (k && (g.k_row < 0 || g.k_head < 0 || !cells_apart(rows, g.n_k_heads, g.k_out_row, g.k_out_head, g.head_dim))) return CASS_ERR_INVALID_ARG;
    // the same place in another layout would be read after it was written
    if (q && q == q_out && ((rows > 1 && g.q_row != g.q_out_row) || (g.n_q_heads > 1 && g.q_head != g.q_out_head))) return CASS_ERR_INVALID_ARG;
    if (k && k == k_out && ((rows > 1 && g.k_row != g.k_out_row) || (g.n_k_heads > 1 && g.k_head != g.k_out_head))) return CASS_ERR_INVALID_ARG;
    if (rows == 0) return CASS_OK;
    cudaStream_t s = (cudaStream_t)stream_;
    if (g.dtype == CASS_BF16) return choose_rope<__nv_bfloat16>(g, freqs, positions, rows, q, k, q_out, k_out, transpose, s);
    if (g.dtype == CASS_F16) return choose_rope<__half>(g, freqs, positions, rows, q, k, q_out, k_out, transpose, s);
    return choose_rope<float>(g, freqs, positions, rows, q, k, q_out, k_out, transpose, s);
}
