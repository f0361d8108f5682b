// The scan of packed prompts: sequences of any lengths one behind the other in the rows of x, dt, B, C and y, the state in front of
// each and behind it in a slot of a cache.
//     h_t = e^{dt_t A} h_{t-1} + dt_t x_t B_t^T ,   y_t = C_t h_t + D x_t
// by chunks of 64 steps, cs the inclusive sums of dt A inside a chunk:
//     y_t = sum_{s<=t} (C_t.B_s) e^{cs_t-cs_s} dt_s x_s + e^{cs_t} C_t h_in + D x_t
//     h_out = e^{cs_last} h_in + sum_s e^{cs_last-cs_s} dt_s x_s B_s^T
// A CTA takes one head of one sequence from its first row to its last, the state in registers (fp32) all the way: nothing but the
// tensors of the call is moved.  The products are those of the split path (ssd_split.cuh): fp32 operands as three bf16 parts, so that
// states and outputs are fp32 results, infinities among them: fp32 tensors (bf16 ones: ssd_packed_tc.cu).  A last chunk that the sequence does not fill is
// filled with zeros, whatever the rows behind it hold.  cs in 64 bits: with strong decays it runs into the thousands, where 32 bits
// would leave 5e-4 of a difference.
//
// Bound by the latency of a chunk's chain (load, split, three products with a barrier behind each): 14.5 us a chunk of 64 rows with N = 64,
// two CTAs per SM, in which the bf16 products (six to an fp32 one) are 25 MFLOP: 8 x 2000 rows of 24 heads run them at 170 TFLOP/s.
#include "ssd_internal.h"
#include "ssd_packed.h"
#include "ssd_split.cuh"

namespace ssd {

namespace {

constexpr int PK_Q = 64, PK_THREADS = 256;
constexpr int PA = SplitParts<float>::n;

// C, B, x, and the state's parts, in whose place the masked tile and x' stand in turn: N = 64 takes 112 KB, so that two CTAs share an SM
// (eight of 2000 rows of 24 heads 463 us; with a place of their own, 140 KB and one CTA, 573)
template <int N> constexpr int packed_smem() { return (2 * (N / 64) * PA + PA + 3 * (N / 64)) * (int)sizeof(SplitTile); }

// 64 rows of 64 columns of a row-major matrix, zeros from row n on
__device__ __forceinline__ void load_rows(TileRegs<float> &r, const float *src, int64_t stride, int n) {
    using V = std::remove_reference_t<decltype(r.v[0])>;
#pragma unroll
    for (int k = 0; k < TileRegs<float>::N; ++k) {
        const int row = r.row(k);
        if (row < n) r.v[k] = __ldg(reinterpret_cast<const V *>(src + row * stride + r.col()));
        else r.v[k] = V{};
    }
}
// Accumulators as three parts: element pairs, rows as they are
__device__ __forceinline__ void put_acc(SplitTile *s, const Acc &a) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t w[3];
            const float2 v = a.get(j, half);
            split2(v.x, v.y, w);
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<uint32_t *>(&s[p].v[acc_row(half)][acc_col(j)]) = w[p];
        }
}

struct ChunkVecs {
    double cs[PK_Q];
    float dts[PK_Q], wS[PK_Q], eC[PK_Q];
};

// A CTA's work.  True where NaN came out without AGAIN: then it is run once more with it, for infinities (tile_mma), and writes its outputs a second time;
// the slot is replaced at the end, by whichever is the last.
template <int N, bool SUMS, bool AGAIN> __device__ __forceinline__ bool packed_unit(const PackedParams &p, ChunkVecs &vecs) {
    constexpr int NT = N / 64;
    extern __shared__ __align__(16) unsigned char pk_smem[];
    SplitTile *Cs = reinterpret_cast<SplitTile *>(pk_smem), *Bs = Cs + NT * PA, *Xs = Bs + NT * PA, *Hs = Xs + PA, *Ms = Hs;
    double *cs = vecs.cs;
    float *dts = vecs.dts, *wS = vecs.wS, *eC = vecs.eC;
    bool nan = false;
    // v times a decay, and c added.  A decay is above zero, so that an infinity stays one where the decay's fp32 value has become zero.
    auto decayed_plus = [](float v, float decay, float c) { return AGAIN && isinf(v) ? v + c : fmaf(v, decay, c); };
    const int h = blockIdx.y, g = h / p.hpg;
    const ScanUnit u = (SUMS ? p.sums : p.units)[blockIdx.x];
    const float Dh = __ldg(p.D + h);
    const double Ah = __ldg(p.A + h);
    const float *x = (const float *)p.x + u.row0 * p.x_rs + h * 64;
    const float *Bm = (const float *)p.Bm + u.row0 * p.b_rs + g * N, *Cm = (const float *)p.Cm + u.row0 * p.c_rs + g * N;
    const float *dt = p.dt + u.row0 * p.dt_rs + h;
    float *y = (float *)p.y + u.row0 * p.y_rs + h * 64;
    const int64_t HPN = (int64_t)p.H * 64 * N;
    float *st = u.slot < 0 ? nullptr : p.state + u.slot * p.state_stride + (int64_t)h * 64 * N;
    float *entry = p.entries + u.entry * HPN + (int64_t)h * 64 * N;        // of a cut sequence

    Acc hs[NT];                    // h[p][n]: rows p, columns n of 64-column tile i
#pragma unroll
    for (int i = 0; i < NT; ++i) hs[i].zero();
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half) f(i, j, half, acc_row(half) * N + i * 64 + acc_col(j));
    };
    if (u.range == 0) {
        if (u.carry) {
            const float *from = !SUMS && u.entry >= 0 ? entry : st;            // the slot may have been replaced by then
            each([&](int i, int j, int half, int at) { hs[i].set(j, half, *reinterpret_cast<const float2 *>(from + at)); });
            if (SUMS) each([&](int i, int j, int half, int at) { *reinterpret_cast<float2 *>(entry + at) = hs[i].get(j, half); });
        }
    } else if (!SUMS) {
        // the state behind range 0, then the sums of the ranges up to this one
        for (int k = 1; k <= u.range; ++k) {
            const float d = exp2f((float)p.decays[(int64_t)(u.entry + k) * p.H + h]);
            each([&](int i, int j, int half, int at) {
                const float2 v = *reinterpret_cast<const float2 *>(entry + k * HPN + at), o = hs[i].get(j, half);
                hs[i].set(j, half, make_float2(decayed_plus(o.x, d, v.x), decayed_plus(o.y, d, v.y)));
            });
        }
    }
    double decayed = 0.;
    for (int t0 = 0; t0 < u.n; t0 += PK_Q) {
        const int n = min(PK_Q, u.n - t0);
        {
            TileRegs<float> rc[NT], rb[NT], rx;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if (!SUMS) load_rows(rc[i], Cm + t0 * p.c_rs + i * 64, p.c_rs, n);
                load_rows(rb[i], Bm + t0 * p.b_rs + i * 64, p.b_rs, n);
            }
            load_rows(rx, x + t0 * p.x_rs, p.x_rs, n);
            if (threadIdx.x < 32) {
                const int a = 2 * threadIdx.x;
                const float d0 = a < n ? __ldg(dt + (t0 + a) * p.dt_rs) : 0.f, d1 = a + 1 < n ? __ldg(dt + (t0 + a + 1) * p.dt_rs) : 0.f;
                const double a0 = d0 * Ah, a1 = a0 + d1 * Ah;
                double s = a1;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double v = __shfl_up_sync(0xffffffffu, s, o);
                    if ((int)threadIdx.x >= o) s += v;
                }
                const double last = __shfl_sync(0xffffffffu, s, 31), before = s - a1;
                cs[a] = before + a0;
                cs[a + 1] = s;
                dts[a] = d0;
                dts[a + 1] = d1;
                wS[a] = d0 * expf((float)(last - (before + a0)));
                wS[a + 1] = d1 * expf((float)(last - s));
                eC[a] = expf((float)(before + a0));
                eC[a + 1] = expf((float)s);
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if (!SUMS) tile_store(Cs + i * PA, rc[i]);
                tile_store(Bs + i * PA, rb[i]);
                if (!SUMS) put_acc(Hs + 3 * i, hs[i]);
            }
            tile_store(Xs, rx);
        }
        __syncthreads();
        if constexpr (!SUMS) {
            Acc m, yi, yx;
            m.zero();
            yi.zero();
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                tile_mma<PA, PA, false, false, AGAIN>(m, Cs + i * PA, Bs + i * PA);
                tile_mma<PA, 3, false, false, AGAIN>(yi, Cs + i * PA, Hs + 3 * i);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = acc_row(i >> 1), s = acc_col(j) + (i & 1);
                    if (AGAIN && s <= t && isinf(m.m[j][i])) m.m[j][i] *= dts[s];
                    else m.m[j][i] = s <= t ? m.m[j][i] * (expf((float)(cs[t] - cs[s])) * dts[s]) : 0.f;
                }
            __syncthreads();                                  // every warp is through with the state's parts
            put_acc(Ms, m);
            __syncthreads();
            yx.zero();
            tile_mma<3, PA, false, true, AGAIN>(yx, Ms, Xs);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int t = acc_row(half);
                const float e = eC[t];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 a = yi.get(j, half), b = yx.get(j, half);
                    const float x0 = joined<PA>(Xs, t, acc_col(j)), x1 = joined<PA>(Xs, t, acc_col(j) + 1);
                    const float2 v = make_float2(fmaf(Dh, x0, decayed_plus(a.x, e, b.x)), fmaf(Dh, x1, decayed_plus(a.y, e, b.y)));
                    if (t < n) {
                        *reinterpret_cast<float2 *>(y + (t0 + t) * p.y_rs + acc_col(j)) = v;
                        if (!AGAIN) nan |= isnan(v.x) || isnan(v.y);
                    }
                }
            }
            __syncthreads();                                  // every warp is through with the masked tile
        }
        const float decay = eC[PK_Q - 1];
        decayed += cs[PK_Q - 1];
        for (int i = threadIdx.x; i < 64 * 32; i += PK_THREADS) {
            const int s = i >> 5, c = (i & 31) * 2;
            const float w = wS[s], x0 = joined<PA>(Xs, s, c), x1 = joined<PA>(Xs, s, c + 1);
            uint32_t q[3];
            split2(AGAIN && isinf(x0) ? dts[s] * x0 : w * x0, AGAIN && isinf(x1) ? dts[s] * x1 : w * x1, q);
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<uint32_t *>(&Ms[k].v[s][c]) = q[k];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!AGAIN || !isinf(hs[i].m[j][e])) hs[i].m[j][e] *= decay;
            tile_mma<3, PA, true, true, AGAIN>(hs[i], Ms, Bs + i * PA);
        }
        __syncthreads();                                  // the tiles are free
    }
    if constexpr (!AGAIN) {
#pragma unroll
        for (int i = 0; i < NT; ++i) nan |= hs[i].nan();
        if (__syncthreads_or(nan)) return true;
    }
    if (SUMS) {
        entry += (u.range + 1) * HPN;
        each([&](int i, int j, int half, int at) { *reinterpret_cast<float2 *>(entry + at) = hs[i].get(j, half); });
        if (threadIdx.x == 0) p.decays[(int64_t)(u.entry + u.range + 1) * p.H + h] = decayed * 1.4426950408889634;
    } else if (u.last && st && (u.n > 0 || !u.carry)) {
        each([&](int i, int j, int half, int at) { *reinterpret_cast<float2 *>(st + at) = hs[i].get(j, half); });
    }
    return false;
}

template <int N, bool SUMS> __global__ void __launch_bounds__(PK_THREADS, N == 64 ? 2 : 1) k_packed_split(const __grid_constant__ PackedParams p) {
    __shared__ ChunkVecs vecs;
    pdl_launch_dependents();
    pdl_wait();
    // no wait of this kernel can run out: the status word is cleared, by the call's first launch
    if ((SUMS || p.nsums == 0) && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = 0u;
    if (packed_unit<N, SUMS, false>(p, vecs)) packed_unit<N, SUMS, true>(p, vecs);
}

}  // namespace

cudaError_t launch_packed_fwd(const PackedParams &p, bool sums, cudaStream_t st) {
    if (p.tc) return launch_packed_tc(p, sums, st);
    const dim3 grid((unsigned)(sums ? p.nsums : p.nunits), (unsigned)p.H), block(PK_THREADS);
#define SSD_PACKED_RUN(N, S)                                                           \
    do {                                                                               \
        cudaError_t e = allow_smem<k_packed_split<N, S>>(packed_smem<N>());            \
        if (e != cudaSuccess) return e;                                                \
        return launch_pdl(k_packed_split<N, S>, grid, block, packed_smem<N>(), st, p); \
    } while (0)
    if (p.N == 128) {
        if (sums) SSD_PACKED_RUN(128, true);
        SSD_PACKED_RUN(128, false);
    }
    if (sums) SSD_PACKED_RUN(64, true);
    SSD_PACKED_RUN(64, false);
#undef SSD_PACKED_RUN
}

}  // namespace ssd
