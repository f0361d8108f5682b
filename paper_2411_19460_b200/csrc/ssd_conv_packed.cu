// The short causal convolution over packed prompts: sequences one behind the other in the rows of u and out, the three inputs in front of
// each and the last three of it in a slot of a cache.
//     out[t,c] = SiLU(bias[c] + sum_{k<4} w[c,k] u[t-3+k, c])
// A CTA takes a tile of rows of one sequence (64; 32, 16 or 8 in batches of up to 16384, 4096, 1024 rows: ssd_plan_make); a thread has 16 bytes of adjacent channels
// and walks the rows with the last three in registers.  Its 16 bytes of the next 16 rows are on their way into shared memory, where no other
// thread looks (so there is nothing to meet for): 23760 rows of 5376 channels in bf16 98 us (5.2 TB/s, 80% of a copy's rate), with loads to registers
// ahead of their use 128.  Bound by memory.  The tile with a sequence's first row is the only one that touches its slot:
// the thread that reads the old state writes the new one, from the last rows of u.
#include "ssd_conv_math.cuh"
#include "ssd_internal.h"
#include "ssd_packed.h"

namespace ssd {

namespace {

constexpr int CP_THREADS = 64, CP_ROUND = 4, CP_ROUNDS = 4;      // rows of a round, rounds under way

template <typename T>
__global__ void __launch_bounds__(CP_THREADS, 8) k_conv_packed(const ConvTile *tiles, const T *u, int64_t u_rs, const float *w, const float *bias, T *state,
                                                            int64_t state_stride, T *out, int64_t out_rs, int C) {
    constexpr int V = 16 / sizeof(T);
    pdl_launch_dependents();
    pdl_wait();
    const int c = (blockIdx.y * CP_THREADS + threadIdx.x) * V;
    if (c >= C) return;
    const ConvTile t = tiles[blockIdx.x];
    const T *up = u + t.row0 * u_rs + c;
    auto row = [&](int64_t r) { return __ldg(reinterpret_cast<const uint4 *>(up + r * u_rs)); };
    uint4 past[3] = {};
    if (t.before >= 3) {
#pragma unroll
        for (int k = 0; k < 3; ++k) past[k] = row(k - 3);
    } else if (t.slot >= 0) {          // the first tile of a sequence
        T *sp = state + t.slot * state_stride + c;
        if (t.carry) {
#pragma unroll
            for (int k = 0; k < 3; ++k) past[k] = *reinterpret_cast<const uint4 *>(sp + (int64_t)k * C);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int r = t.len - 3 + k;                // below zero: input 3 + r of the old state
            uint4 v = r >= 0 ? row(r) : past[0];
            if (r == -2) v = past[1];
            if (r == -1) v = past[2];
            *reinterpret_cast<uint4 *>(sp + (int64_t)k * C) = v;
        }
    }
    if (t.n == 0) return;
    ConvWeights<V> cw;
    __shared__ uint4 ring[CP_ROUNDS][CP_ROUND][CP_THREADS];
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&ring[0][0][threadIdx.x]);
    constexpr uint32_t ROW = CP_THREADS * 16;
    const T *src = up;
    int left = t.n;                                    // rows that are not yet on their way
    auto fetch = [&](int round) {
        const uint32_t dst = mine + (round % CP_ROUNDS) * (CP_ROUND * ROW);
#pragma unroll
        for (int j = 0; j < CP_ROUND; ++j) {
            if (j < left) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + j * ROW), "l"(src) : "memory");
            src += u_rs;
        }
        left -= CP_ROUND;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < CP_ROUNDS - 1; ++k) fetch(k);
    cw.load(w, bias, c);
    float2 x[3][V / 2];
#pragma unroll
    for (int k = 0; k < 3; ++k) conv_unpack<T>(past[k], x[k]);
    T *op = out + t.row0 * out_rs + c;
    auto step = [&](const uint4 *at, const float2 *x0, const float2 *x1, const float2 *x2, float2 *x3) {
        float2 o[V / 2];
        conv_unpack<T>(*at, x3);
        cw.template apply<sizeof(T) == 4>(x0, x1, x2, x3, o);
        *reinterpret_cast<uint4 *>(op) = conv_pack<T>(o);
        op += out_rs;
    };
    float2 x3[V / 2];
    static_assert(CP_ROUND == 4, "four rows turn the window once round");
    for (int r = 0, round = 0; r < t.n; r += CP_ROUND, ++round) {
        fetch(round + CP_ROUNDS - 1);                  // into the round before this one's place
        asm volatile("cp.async.wait_group %0;" ::"n"(CP_ROUNDS - 1) : "memory");
        const uint4(*now)[CP_THREADS] = ring[round % CP_ROUNDS];
        step(&now[0][threadIdx.x], x[0], x[1], x[2], x3);
        if (r + 1 < t.n) step(&now[1][threadIdx.x], x[1], x[2], x3, x[0]);
        if (r + 2 < t.n) step(&now[2][threadIdx.x], x[2], x3, x[0], x[1]);
        if (r + 3 < t.n) step(&now[3][threadIdx.x], x3, x[0], x[1], x[2]);
    }
}

}  // namespace

cudaError_t launch_conv_packed(int dtype, int ntiles, const ConvTile *tiles, int C, const void *u, int64_t u_rs, const float *w, const float *bias, void *state,
                               int64_t state_stride, void *out, int64_t out_rs, cudaStream_t st) {
    const int V = dtype == SSD_DTYPE_F32 ? 4 : 8;
    const dim3 grid((unsigned)ntiles, (unsigned)((C / V + CP_THREADS - 1) / CP_THREADS)), block(CP_THREADS);
    if (dtype == SSD_DTYPE_F32)
        return launch_pdl(k_conv_packed<float>, grid, block, 0, st, tiles, (const float *)u, u_rs, w, bias, (float *)state, state_stride, (float *)out, out_rs, C);
    return launch_pdl(k_conv_packed<__nv_bfloat16>, grid, block, 0, st, tiles, (const __nv_bfloat16 *)u, u_rs, w, bias, (__nv_bfloat16 *)state, state_stride,
                      (__nv_bfloat16 *)out, out_rs, C);
}

}  // namespace ssd
