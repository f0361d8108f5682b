// One token of each running sequence, with the sequences' states in slots of a cache: row b of the inputs belongs to slot slots[b] (null:
// slot b).  A row whose slot is negative or not below nslots is empty, and so is one whose slot an earlier row has too: nothing of it is
// read or written.  The slots are device memory, so that a captured graph serves a changing batch.
//   k_decode_slots   h <- e^{dt A} h + dt x B^T ,  y = C h + D x          (Eq. 1, one step)
//   k_conv_step      out = SiLU(bias + w . (last three inputs, u)) , the last inputs moved on by one
#include "ssd_internal.h"
#include "ssd_conv_math.cuh"

namespace ssd {

namespace {

// Slot of row b, -1 for an empty row.  Whole warps call it; every lane gets the answer.  The comparison with the rows before takes one
// load per 32 of them, from the same few cache lines in every warp, beside the state's own loads: rows of 8 heads, N = 64, 48 us with slots and 42
// without for 1024 of them, 213 and 158 for 4096, 1840 and 620 for 16384; quadratic, which is why rows end at 65535.
__device__ __forceinline__ int slot_of(const int *slots, long long b, int nslots) {
    if (!slots) return (int)b;
    const int s = __ldg(slots + b);
    return (unsigned)s < (unsigned)nslots ? s : -1;
}
__device__ __forceinline__ bool taken_before(const int *slots, long long b, int s) {
    if (!slots) return false;
    bool hit = false;
    for (long long i = threadIdx.x & 31; i < b; i += 32) hit |= __ldg(slots + i) == s;
    return __any_sync(0xffffffffu, hit);
}

template <typename T> __device__ __forceinline__ float ldf(const T *p);
template <> __device__ __forceinline__ float ldf<float>(const float *p) { return __ldg(p); }
template <> __device__ __forceinline__ float ldf<__nv_bfloat16>(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
template <typename T> __device__ __forceinline__ void stf(T *p, float v);
template <> __device__ __forceinline__ void stf<float>(float *p, float v) { *p = v; }
template <> __device__ __forceinline__ void stf<__nv_bfloat16>(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
template <typename T> __device__ __forceinline__ void ld4(const T *p, float *f);
template <> __device__ __forceinline__ void ld4<float>(const float *p, float *f) {
    const float4 v = __ldg(reinterpret_cast<const float4 *>(p));
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}
template <> __device__ __forceinline__ void ld4<__nv_bfloat16>(const __nv_bfloat16 *p, float *f) {
    const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v.y));
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}

constexpr int DS_WARPS = 4;

// A row of the state (one p of one head) is held by N/4 lanes, 16 bytes each; a warp takes ROWS rows of one head, all their loads in
// flight together.  The sums over a row's lanes meet in a transposing butterfly.  Bound by the state's traffic, read and written once: 186 of 193 rows of
// 64 heads, 780 MB, 119 us (6.6 TB/s, a copy's rate); a row of 80 heads 2.8 us, the launch.
template <typename T, int N, int ROWS>
__global__ void __launch_bounds__(DS_WARPS * 32) k_decode_slots(SlotParams p, long long groups) {
    constexpr int LPR = N / 4, RPW = 32 / LPR, NL = ROWS / RPW;   // lanes per row, rows per load, loads
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, sub = lane / LPR, col = (lane % LPR) * 4;
    const long long grp = (long long)blockIdx.x * DS_WARPS + (threadIdx.x >> 5);
    if (grp >= groups) return;
    const int per_head = 64 / ROWS;
    const int p0 = (int)(grp % per_head) * ROWS, hh = (int)(grp / per_head % p.H);
    const long long b = grp / per_head / p.H;
    const int slot = slot_of(p.slots, b, p.nslots);
    if (slot < 0) return;
    float *hp = p.state + (long long)slot * p.state_stride + ((long long)hh * 64 + p0 + sub) * N + col;
    float4 hv[NL];
#pragma unroll
    for (int k = 0; k < NL; ++k) hv[k] = *reinterpret_cast<const float4 *>(hp + k * RPW * N);
    const T *xp = (const T *)p.x + b * p.x_rs + hh * 64 + p0;
    float xv[NL], bv[4], cv[4];
#pragma unroll
    for (int k = 0; k < NL; ++k) xv[k] = ldf(xp + k * RPW + sub);
    const int g = hh / p.hpg;
    ld4((const T *)p.Bm + b * p.b_rs + g * N + col, bv);
    ld4((const T *)p.Cm + b * p.c_rs + g * N + col, cv);
    const float dtv = __ldg(p.dt + b * p.dt_rs + hh), decay = expf(dtv * __ldg(p.A + hh)), Dh = __ldg(p.D + hh);
    if (taken_before(p.slots, b, slot)) return;
    float acc[NL];
#pragma unroll
    for (int k = 0; k < NL; ++k) {
        const float dx = dtv * xv[k];
        float4 v = hv[k];
        v.x = fmaf(v.x, decay, dx * bv[0]);
        v.y = fmaf(v.y, decay, dx * bv[1]);
        v.z = fmaf(v.z, decay, dx * bv[2]);
        v.w = fmaf(v.w, decay, dx * bv[3]);
        acc[k] = fmaf(cv[3], v.w, fmaf(cv[2], v.z, fmaf(cv[1], v.y, cv[0] * v.x)));
        *reinterpret_cast<float4 *>(hp + k * RPW * N) = v;
    }
    int mine = 0, o = LPR / 2;
#pragma unroll
    for (int cnt = NL; cnt > 1; cnt >>= 1, o >>= 1) {
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int i = 0; i < cnt / 2; ++i) {
            const float send = up ? acc[i] : acc[i + cnt / 2], keep = up ? acc[i + cnt / 2] : acc[i];
            acc[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
        mine += up ? cnt / 2 : 0;
    }
#pragma unroll
    for (; o > 0; o >>= 1) acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], o);
    if ((lane % (LPR / NL)) == 0) {
        const int r = mine * RPW + sub;
        stf((T *)p.y + b * p.y_rs + hh * 64 + p0 + r, fmaf(Dh, ldf(xp + r), acc[0]));
    }
}

constexpr int CS_THREADS = 64;

// A thread has 16 bytes of adjacent channels of one row: 193 rows of 4352 channels in bf16 6.0 us, a chain of two loads (slot, state) and the launch.
template <typename T>
__global__ void __launch_bounds__(CS_THREADS) k_conv_step(const T *u, int64_t u_rs, const float *w, const float *bias, T *state, int nslots,
                                                          int64_t state_stride, const int *slots, T *out, int64_t out_rs, int C) {
    constexpr int V = 16 / sizeof(T);
    pdl_launch_dependents();
    pdl_wait();
    const long long b = blockIdx.y;
    const int slot = slot_of(slots, b, nslots), c = (blockIdx.x * CS_THREADS + threadIdx.x) * V;
    if (slot < 0) return;
    const bool on = c < C;
    T *sp = state + (long long)slot * state_stride + c;
    uint4 r[4] = {};
    ConvWeights<V> cw;
    if (on) {
#pragma unroll
        for (int k = 0; k < 3; ++k) r[k] = *reinterpret_cast<const uint4 *>(sp + (int64_t)k * C);
        r[3] = __ldg(reinterpret_cast<const uint4 *>(u + b * u_rs + c));
        cw.load(w, bias, c);
    }
    if (taken_before(slots, b, slot) || !on) return;
    float2 f[4][V / 2], o[V / 2];
#pragma unroll
    for (int k = 0; k < 4; ++k) conv_unpack<T>(r[k], f[k]);
    cw.template apply<sizeof(T) == 4>(f[0], f[1], f[2], f[3], o);
    *reinterpret_cast<uint4 *>(out + b * out_rs + c) = conv_pack<T>(o);
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4 *>(sp + (int64_t)k * C) = r[k + 1];
}

}  // namespace

cudaError_t launch_decode_slots(const SlotParams &p, cudaStream_t st) {
    // Eight rows per warp; few rows are spread over more warps, two rows each (as in the step without slots)
    const long long rows = p.rows * p.H * 64;
    const int per = rows >= 8ll * 148 * 16 ? 8 : 2;
    const long long groups = rows / per;
    const dim3 grid((unsigned)((groups + DS_WARPS - 1) / DS_WARPS)), block(DS_WARPS * 32);
#define SSD_SLOTS_CASE(T, N)                                                                      \
    do {                                                                                          \
        if (per == 8) return launch_pdl(k_decode_slots<T, N, 8>, grid, block, 0, st, p, groups);  \
        return launch_pdl(k_decode_slots<T, N, 2>, grid, block, 0, st, p, groups);                \
    } while (0)
    if (p.dtype == SSD_DTYPE_F32) {
        if (p.N == 128) SSD_SLOTS_CASE(float, 128); else SSD_SLOTS_CASE(float, 64);
    } else {
        if (p.N == 128) SSD_SLOTS_CASE(__nv_bfloat16, 128); else SSD_SLOTS_CASE(__nv_bfloat16, 64);
    }
#undef SSD_SLOTS_CASE
}

cudaError_t launch_conv_step(int dtype, long long rows, int C, const void *u, int64_t u_rs, const float *w, const float *bias, void *state, int nslots,
                             int64_t state_stride, const int *slots, void *out, int64_t out_rs, cudaStream_t st) {
    const int V = dtype == SSD_DTYPE_F32 ? 4 : 8;
    const dim3 grid((unsigned)((C / V + CS_THREADS - 1) / CS_THREADS), (unsigned)rows), block(CS_THREADS);
    if (dtype == SSD_DTYPE_F32)
        return launch_pdl(k_conv_step<float>, grid, block, 0, st, (const float *)u, u_rs, w, bias, (float *)state, nslots, state_stride, slots, (float *)out,
                          out_rs, C);
    return launch_pdl(k_conv_step<__nv_bfloat16>, grid, block, 0, st, (const __nv_bfloat16 *)u, u_rs, w, bias, (__nv_bfloat16 *)state, nslots, state_stride,
                      slots, (__nv_bfloat16 *)out, out_rs, C);
}

}  // namespace ssd
