// The norm of many gradients together and their scaling to a largest norm:
//     norm = sqrt(sum g^2) ,   out = g min(1, max_norm / norm)          (gradients that are not finite: nothing is scaled)
// The factor is fp32.  A norm above fp32's largest value, or a factor below its smallest normal one, which would have few bits left, are kept in 64
// bits, and the gradients then multiplied so, one by one.
// Two launches.  The first walks all tensors in chunks, a number of CTAs that the sizes fix, and leaves one sum per CTA in 64 bits;
// in the second every CTA adds those sums up in the same order and scales its chunks, the last read first (of small gradients the
// L2 cache has all; of 483 MB it keeps nothing: the second reading takes all of them from memory again).  Squares of up to 16
// elements are added in 32 bits, everything above in 64; those whose sum leaves the middle of the range (below 1e-30, where squares
// are lost, or above 1e30, infinities and NaN among them) are taken again in 64 bits.
// Bound by memory: 483 MB of gradients 240 us, two readings and a writing at 6.0 TB/s (74 us the norm, at 6.5).  384 small vectors take
// 16 us on the device, 25 with the host's part of the call, which is the longer one.
// The table of tensors travels in the launch's parameters: no copy to the device, and a captured graph has it by value.
#include <cfloat>

#include "ssd_internal.h"

namespace ssd {

namespace {

constexpr int CL_THREADS = 256, CL_VECS = 4;                       // 16-byte vectors per thread and chunk

struct ClipTensor {
    const void *in;
    void *out;
    int64_t n;
    int32_t dtype;
    int32_t first;                 // number of its first chunk
};
template <int MAX> struct ClipTable {
    int32_t n, chunks;
    ClipTensor t[MAX];
};
// CTAs per SM that scale, all at once: 483 MB of gradients (clipped, with their norm) take 241 us, with 2, 4, 5 of them 276, 248, 250
constexpr int CL_SCALE = 3;
// Tables of 3, 15 and 30 KB of launch parameters, whose copying is host time: 384 vectors 28 us with the large one, 24 with the middle one
constexpr int CL_SMALL = 96, CL_MIDDLE = 480, CL_LARGE = 960;
static_assert(sizeof(ClipTable<CL_LARGE>) + 64 <= 32764, "launch parameters");

__host__ __device__ constexpr int64_t chunk_elems(int dtype) { return (int64_t)CL_THREADS * CL_VECS * (dtype == SSD_DTYPE_F32 ? 4 : 8); }

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// g times the factor; the factor 1 leaves every bit of it, of a NaN too
template <typename T> __device__ __forceinline__ T scaled(T g, float scale) { return scale == 1.f ? g : from_f<T>(to_f(g) * scale); }

// the same of the elements of 32 bits, by a factor that is not 1
template <typename T> __device__ __forceinline__ uint32_t scaled_word(uint32_t w, float scale) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(__uint_as_float(w) * scale);
    const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(w << 16) * scale, __uint_as_float(w & 0xffff0000u) * scale);
    return *reinterpret_cast<const uint32_t *>(&v);
}

template <typename T> struct alignas(16) Vec {
    T v[16 / sizeof(T)];
};

template <int MAX> __device__ __forceinline__ int find_tensor(const ClipTable<MAX> &tab, int chunk) {
    int lo = 0, hi = tab.n - 1;                                     // the last tensor whose first chunk is not behind `chunk`
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.t[mid].first <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Squares of the elements of 16 bytes, of n of them, in 64 bits.  Zeros, as unused rows have them, end here at once: the norm of 360 MB of them takes 76 us
// (132 without this second load, 65 that of other values; with the test in the ordinary path that became 81).
template <typename T> __device__ __noinline__ double squares_64(const T *f, int64_t n) {
    double d = 0.;
    if (n >= (int64_t)(16 / sizeof(T))) {
        const uint4 w = *reinterpret_cast<const uint4 *>(f);
        if (((w.x | w.y | w.z | w.w) & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu)) == 0u) return 0.;
    }
    for (int64_t i = 0; i < n && i < (int64_t)(16 / sizeof(T)); ++i) d += (double)to_f(f[i]) * (double)to_f(f[i]);
    return d;
}
__device__ __forceinline__ float2 pair_of(const Vec<float> &v, int i) { return make_float2(v.v[2 * i], v.v[2 * i + 1]); }
__device__ __forceinline__ float2 pair_of(const Vec<__nv_bfloat16> &v, int i) {
    const uint32_t w = reinterpret_cast<const uint32_t *>(&v)[i];
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
// squares of the elements of 16 bytes
template <typename T> __device__ __forceinline__ float squares(const Vec<T> &v) {
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < (int)(8 / sizeof(T)); ++i) {
        const float2 f = pair_of(v, i);
        s = __ffma2_rn(f, f, s);
    }
    return s.x + s.y;
}

// elements [begin, end) of a tensor whose address is a multiple of 16 bytes, else one by one
template <typename T> __device__ __forceinline__ double chunk_squares(const T *in, int64_t begin, int64_t end) {
    constexpr int V = 16 / sizeof(T);
    double s = 0.;
    if (((uintptr_t)in & 15) == 0) {
        Vec<T> v[CL_VECS];
#pragma unroll
        for (int k = 0; k < CL_VECS; ++k) {
            const int64_t at = begin + ((int64_t)k * CL_THREADS + threadIdx.x) * V;
            v[k] = Vec<T>{};
            if (at + V <= end) v[k] = *reinterpret_cast<const Vec<T> *>(in + at);
            else
                for (int i = 0; i < V; ++i)
                    if (at + i < end) v[k].v[i] = in[at + i];
        }
        // pairs of vectors: sums of 8 or 16 squares, of positive terms
#pragma unroll
        for (int k = 0; k < CL_VECS; k += 2) {
            const float f = squares(v[k]) + squares(v[k + 1]);
            if (f > 1e-30f && f < 1e30f) s += (double)f;
            else {
                const int64_t at = begin + ((int64_t)k * CL_THREADS + threadIdx.x) * V, next = at + CL_THREADS * V;
                s += squares_64(in + at, end - at) + squares_64(in + next, end - next);
            }
        }
    } else {
        for (int64_t at = begin + threadIdx.x; at < end; at += CL_THREADS) s += (double)to_f(in[at]) * (double)to_f(in[at]);
    }
    return s;
}

template <typename T> __device__ __forceinline__ void chunk_scale(const T *in, T *out, int64_t begin, int64_t end, float scale) {
    constexpr int V = 16 / sizeof(T);
    if ((((uintptr_t)in | (uintptr_t)out) & 15) == 0) {
        uint4 v[CL_VECS];
#pragma unroll
        for (int k = 0; k < CL_VECS; ++k) {
            const int64_t at = begin + ((int64_t)k * CL_THREADS + threadIdx.x) * V;
            if (at + V <= end) v[k] = *reinterpret_cast<const uint4 *>(in + at);
        }
#pragma unroll
        for (int k = 0; k < CL_VECS; ++k) {
            const int64_t at = begin + ((int64_t)k * CL_THREADS + threadIdx.x) * V;
            if (at + V <= end) {
                if (scale != 1.f) v[k] = make_uint4(scaled_word<T>(v[k].x, scale), scaled_word<T>(v[k].y, scale), scaled_word<T>(v[k].z, scale), scaled_word<T>(v[k].w, scale));
                *reinterpret_cast<uint4 *>(out + at) = v[k];
            } else {
#pragma unroll 1
                for (int64_t i = at; i < end; ++i) out[i] = scaled(in[i], scale);
            }
        }
    } else {
#pragma unroll 1
        for (int64_t at = begin + threadIdx.x; at < end; at += CL_THREADS) out[at] = scaled(in[at], scale);
    }
}

__device__ __forceinline__ double block_sum(double s, double *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.;
#pragma unroll
    for (int i = 0; i < CL_THREADS / 32; ++i) s += red[i];
    return s;
}

template <int MAX> __global__ void __launch_bounds__(CL_THREADS) k_clip_norm(const __grid_constant__ ClipTable<MAX> tab, double *part) {
    __shared__ double red[CL_THREADS / 32];
    pdl_launch_dependents();
    pdl_wait();
    double s = 0.;
    for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        const ClipTensor &t = tab.t[find_tensor(tab, c)];
        const int64_t per = chunk_elems(t.dtype), begin = (c - t.first) * per, end = min(begin + per, t.n);
        if (t.dtype == SSD_DTYPE_F32) s += chunk_squares((const float *)t.in, begin, end);
        else s += chunk_squares((const __nv_bfloat16 *)t.in, begin, end);
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// All chunks by a factor below fp32's normal numbers
template <int MAX> __device__ __noinline__ void scale_64(const ClipTable<MAX> &tab, double scale) {
    for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        const ClipTensor &t = tab.t[find_tensor(tab, c)];
        const int64_t per = chunk_elems(t.dtype), begin = (c - t.first) * per, end = min(begin + per, t.n);
        for (int64_t at = begin + threadIdx.x; at < end; at += CL_THREADS) {
            if (t.dtype == SSD_DTYPE_F32) ((float *)t.out)[at] = (float)((double)((const float *)t.in)[at] * scale);
            else ((__nv_bfloat16 *)t.out)[at] = __float2bfloat16_rn((float)((double)__bfloat162float(((const __nv_bfloat16 *)t.in)[at]) * scale));
        }
    }
}

template <int MAX>
__global__ void __launch_bounds__(CL_THREADS, CL_SCALE) k_clip_scale(const __grid_constant__ ClipTable<MAX> tab, const double *part, int nparts, float max_norm, float *norm) {
    __shared__ double red[CL_THREADS / 32];
    pdl_launch_dependents();
    pdl_wait();
    double s = 0.;
    for (int i = threadIdx.x; i < nparts; i += CL_THREADS) s += part[i];
    const double wide = sqrt(block_sum(s, red));
    const float n = (float)wide;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
    const float scale = n > max_norm && isfinite(wide) ? max_norm / n : 1.f;
    if (scale < FLT_MIN && max_norm > 0.f) {
        scale_64(tab, max_norm / wide);
        return;
    }
    for (int c = tab.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const ClipTensor &t = tab.t[find_tensor(tab, c)];
        if (scale == 1.f && t.in == t.out) continue;
        const int64_t per = chunk_elems(t.dtype), begin = (c - t.first) * per, end = min(begin + per, t.n);
        if (t.dtype == SSD_DTYPE_F32) chunk_scale((const float *)t.in, (float *)t.out, begin, end, scale);
        else chunk_scale((const __nv_bfloat16 *)t.in, (__nv_bfloat16 *)t.out, begin, end, scale);
    }
}

template <int MAX> cudaError_t clip_part(int n, const void *const *in, void *const *out, const int64_t *numel, const int32_t *dtypes, int pass, double *part,
                                         int ntables, float max_norm, float *norm, cudaStream_t st) {
    ClipTable<MAX> tab;
    tab.n = 0;
    tab.chunks = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const int64_t per = chunk_elems(dtypes[i]);
        tab.t[tab.n++] = ClipTensor{in[i], out[i], numel[i], dtypes[i], tab.chunks};
        tab.chunks += (int32_t)((numel[i] + per - 1) / per);
    }
    // one table: as many sums as chunks where these are fewer; several: the same number for each
    const int ctas = ntables > 1 || tab.chunks > kClipCtas ? kClipCtas : tab.chunks > 0 ? tab.chunks : 1;
    if (pass == 0) return launch_pdl(k_clip_norm<MAX>, dim3(ctas), dim3(CL_THREADS), 0, st, tab, part);
    return launch_pdl(k_clip_scale<MAX>, dim3(ctas < kNumSMs * CL_SCALE ? ctas : kNumSMs * CL_SCALE), dim3(CL_THREADS), 0, st, tab, part, ntables > 1 ? ntables * kClipCtas : ctas, max_norm, norm);
}

}  // namespace

int clip_tables(int n) { return n <= CL_MIDDLE ? 1 : (n + CL_LARGE - 1) / CL_LARGE; }
int64_t clip_chunks(int64_t numel, int dtype) { return (numel + chunk_elems(dtype) - 1) / chunk_elems(dtype); }

cudaError_t launch_clip(int n, const void *const *in, void *const *out, const int64_t *numel, const int32_t *dtypes, int pass, int table, double *part,
                        float max_norm, float *norm, cudaStream_t st) {
    const int ntables = clip_tables(n);
    if (n <= CL_SMALL) return clip_part<CL_SMALL>(n, in, out, numel, dtypes, pass, part, ntables, max_norm, norm, st);
    if (n <= CL_MIDDLE) return clip_part<CL_MIDDLE>(n, in, out, numel, dtypes, pass, part, ntables, max_norm, norm, st);
    const int a = table * CL_LARGE, k = n - a < CL_LARGE ? n - a : CL_LARGE;
    return clip_part<CL_LARGE>(k, in + a, out + a, numel + a, dtypes + a, pass, part + (pass == 0 ? table * kClipCtas : 0), ntables, max_norm,
                               table == 0 ? norm : nullptr, st);
}

}  // namespace ssd
