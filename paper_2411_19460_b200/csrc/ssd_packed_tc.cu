// The scan of packed prompts on the tensor cores (tcgen05, tensor memory, TMA): bf16 tensors, blocks of T = 128 steps.  With cs the inclusive
// sums of dt A inside a block, per head:
//     G = C B^T ,  M = G o mask, mask[t][s] = e^{cs_t-cs_s} dt_s (s <= t)
//     y = M X + e^{cs} (C H) + D x          S^T = B^T X', X'[s] = dt_s e^{cs_last-cs_s} x_s          H <- e^{cs_last} H + S
// A CTA (one per SM) takes one head, or two heads of a group in turn, of one sequence through all its blocks; an item is one head of one
// block.  The state stays in registers (fp32), so that nothing but the call's tensors moves; two heads share B, C and G.
//
// The mask by row sub-tiles of 32 steps (m the middle one): e^{cs_t-cs_s} = e^{cs_t-cs_m} e^{cs_m-cs_s}, a factor of the row, which is left to the
// output, and one of the column.  Each is at most 2^40 where it counts, where neither half of the sub-tile decays by more; else the mask is made
// with the row's factor in it, on the diagonal element by element.  From the first row on instead of from the middle, half the decay was the
// limit, and heads that passed it took a quarter longer, a whole batch with them.
//
// What is rounded: X' to three bf16 parts (nothing is lost: the states are fp32 results).  M and H to two, 2^-16 of each of their terms in y, which
// is itself rounded to 2^-8; D x is added in fp32.  One part of each, 2^-8 of its terms, costs y 40% more error than its own rounding where the products
// are all of it (D = 0), and nothing where D x is most of it: 24 prompts took 305 us so, the second part of M 26 more, that of H 22.
// Sums are fp32 in tensor memory.  cs is summed in 64 bits and kept as two fp32 numbers: with strong decays it runs into the thousands.
//
// Products (cycles of the tensor pipe): G 512 a block; S 1150 (one part after the other onto the same sums, N = 64, which 48 cycles of reading
// shared memory bound; side by side, 768, they take 128 columns more and the states three times the loads), C H 770, M X 512 (M from tensor
// memory) an item.  Columns of tensor memory: G 128, M two halves of 64 steps times 64, M X 64, C H two times 64 in turn, S 64.
//
// Warps, meeting only through mbarriers (tests/test_packed_halves.py and test_packed_roles.py have a model of who waits for what):
//   0 G and M X   1 S and C H   2, 3 decays of even and odd items   4..11 parts of x'   12..15 outputs   16..23 mask, but for one without
//   a sub-tile: loads   24..31 states, half of p each four
// Bound by shared memory and the hand-overs between the roles: of 4150 cycles an item (two heads; 2.5 us at 1.65 GHz) the products' operands take 2430 at 128
// bytes a cycle, by count, loads and stores of threads keep its pipe busy for 1700 (41% of all cycles, by counter), and the tensor pipe works for 2690.
// 24 prompts, 23760 tokens, of 80 heads: 345 us (1.7 TB/s; its bytes alone 93 us), three of 4096 168 us, one of 49153 of 64 heads with 8 groups 800, 245 of
// them for its sums (a pass among others).  What it took: y over x and parts of x' in a ring of three times 32 steps instead of twice 64, and x ahead of
// C; factors of the mask from the middle row (for strong decays); short code, for the roles' loops together go through the instruction cache once per
// item; with two parts of M and H, C H in two places and the halves of M one by one (353 -> 343).  Four items' x instead of three make no difference,
// for the sums either.  Taken back, slower or no faster: scores ahead of M X, or what of the two is ready first; C H behind the next item's S; y by
// warps; the next block prefetched into L2; polls that sleep or stay; sums given back ahead of the last stores; C H of both parts of H side by side, N =
// 128, which reads C once but has one place (352).
#include "ssd_internal.h"
#include "ssd_packed.h"
#include "ssd_split.cuh"

namespace ssd {

using namespace sm100;

namespace {

constexpr int PT_THREADS = 1024, PT_REGS = 64;          // registers per thread at launch, shared out by role (sum 8 x 64)
constexpr int PT_R_ISSUE = 56, PT_R_X = 48, PT_R_OUT = 56, PT_R_MASK = 56, PT_R_STATE = 96;
static_assert(PT_R_ISSUE + PT_R_OUT + 2 * PT_R_X + 2 * PT_R_MASK + 2 * PT_R_STATE <= 8 * PT_REGS, "a split above the launch's registers would wait forever");

constexpr int PT_SLOTS = 3;                             // ring of B and C tiles, in turn
constexpr int PT_VECS = 3;                              // ring of the items' decays
constexpr int PT_XS = 3;                                // ring of the items' rows of x, in whose place y goes
constexpr int PT_PARTS = 3;                             // ring of the parts of x' of 32 steps
// per item: weights of x' | e^{cs_t} | the output's factor of M X | column factors of the row sub-tiles 0 .. 3 (32, 64, 96, 128 columns) |
// cs, first and second part | dt | e^{cs_last}
enum { PV_W = 0, PV_E = 128, PV_R = 256, PV_F = 384, PV_HI = 704, PV_LO = 832, PV_DT = 960, PV_DECAY = 1088, PV_FLOATS = 1120 };
template <int N> struct PtMem {
    static constexpr uint32_t TILE = 128 * N * 2;
    static constexpr uint32_t X = PT_SLOTS * TILE < 65536 ? 65536 : PT_SLOTS * TILE, XP = X + PT_XS * 16384, H = XP + PT_PARTS * 12288, VEC = H + 2 * N * 128;
    static constexpr uint32_t BYTES = VEC + PT_VECS * PV_FLOATS * 4;
};
static_assert(PtMem<128>::BYTES <= 232448 - 1024, "shared memory");

template <int R> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
__device__ __forceinline__ float pt_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Waits, in few instructions and without the suspend hint: on a phase that is complete the general form takes 240 cycles, this one 72, and
// an item's chain of hand-overs has a dozen.  Only the warp that loads looks at the clock (pt_wait_watched); it waits for every tile's
// readers and at last for all other warps, so that none of them waits for longer than it does: what it gives up it tells the others by the
// abort flag.  A clock of its own in every wait took 9 of 65 KB of code.
__device__ __forceinline__ void pt_wait(uint64_t *bar, uint32_t parity, volatile uint32_t *abortp) {
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        ".reg .u32 a;\n"
        "AGAIN:\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%0], %1;\n"
        "@p bra DONE;\n"
        "ld.volatile.shared.u32 a, [%2];\n"
        "setp.eq.u32 q, a, 0;\n"
        "@q bra AGAIN;\n"
        "DONE:\n"
        "}\n" ::"r"(smem_u32(bar)), "r"(parity), "r"(smem_u32((const void *)abortp))
        : "memory");
}
__device__ __forceinline__ bool pt_try(uint64_t *bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint32_t pt_clock_hi() {      // 2^32 cycles, about 2.3 s
    uint32_t c;
    asm volatile("mov.u32 %0, %%clock_hi;" : "=r"(c));
    return c;
}
__device__ __forceinline__ void pt_wait_watched(uint64_t *bar, uint32_t parity, volatile uint32_t *abortp) {
    const uint32_t start = pt_clock_hi();
    while (!pt_try(bar, parity))
        if (pt_clock_hi() - start >= 2u || *abortp) {   // 2.3 to 4.6 s
            *abortp = 1u;
            break;
        }
}
// A role's place in a ring of three (decays, parts of x'): slot, and whether its pass over the ring is an odd one
static_assert(PT_PARTS == PT_VECS, "rings of one length");
struct VecTurn {
    uint32_t slot = 0, odd = 0;
    __device__ __forceinline__ void next(uint32_t by = 1) {
        slot += by;
        if (slot >= PT_VECS) {
            slot -= PT_VECS;
            odd ^= 1u;
        }
    }
};
// Of cs at a sub-tile's first, middle and last row
__device__ __forceinline__ bool pt_mild(float first, float middle, float last) { return first - middle <= kMildDecay && middle - last <= kMildDecay; }
__device__ __forceinline__ uint32_t pt_pack(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 pt_unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
// Two bf16 parts of two values: rounded, and what that leaves out, rounded (2^-16 of the value at most)
__device__ __forceinline__ void pt_pack2(float a, float b, uint32_t &w, uint32_t &r) {
    w = pt_pack(a, b);
    const float2 f = pt_unpack(w);
    r = pt_pack(a - f.x, b - f.y);
}
// Products and their hand-over by one thread (`on`) of a warp that runs its loop together: in a branch of that thread alone every descriptor
// took two more instructions.  `acc` 0: the first of a sum.
__device__ __forceinline__ void pt_mma(uint32_t on, uint32_t acc, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "setp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(on)
        : "memory");
}
__device__ __forceinline__ void pt_mma_ta(uint32_t on, uint32_t acc, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc) {
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "setp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        "}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(on)
        : "memory");
}
__device__ __forceinline__ void pt_commit(uint32_t on, uint64_t *bar) {
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %1, 0;\n"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
        "}\n" ::"r"(smem_u32(bar)), "r"(on)
        : "memory");
}

}  // namespace

// SUMS: the first launch of a batch with cut sequences: S and H alone, of the ranges that are not a sequence's last (whole blocks)
template <int N, bool SUMS>
__global__ void __launch_bounds__(PT_THREADS, 1)
k_packed_tc(PackedParams p, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC,
            const __grid_constant__ CUtensorMap tmY) {
    using Mem = PtMem<N>;
    constexpr int KN = N / 16;                          // steps of a contraction over n
    constexpr uint32_t TM_G = 0, TM_M = 128, TM_Y = 256, TM_CH = 320, TM_S = 448;
    extern __shared__ __align__(1024) unsigned char smem[];          // swizzled tiles start on multiples of 1024
    __shared__ uint64_t tfull[PT_SLOTS], tempty[PT_SLOTS], xfull[PT_XS], xempty[PT_XS], xready[PT_XS];
    __shared__ uint64_t vfull[PT_VECS], vempty[PT_VECS];
    __shared__ uint64_t gfull, gfree, mfull[2], mempty[2], xpfull[PT_PARTS], xpempty[PT_PARTS], sdone, sfree, hfull, chdone[2], chfree[2], yfull, yfree, tailtx, tailfull, alldone;
    __shared__ uint32_t tmem_base, abort_flag;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < PT_SLOTS; ++i) {
            mbar_init(&tfull[i], 1);
            mbar_init(&tempty[i], SUMS ? 1 : 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&mempty[i], 1);
            mbar_init(&mfull[i], 7);
            mbar_init(&chdone[i], 1);
            mbar_init(&chfree[i], 4);
        }
        for (int i = 0; i < PT_VECS; ++i) {
            mbar_init(&vfull[i], 1);
            mbar_init(&vempty[i], SUMS ? 8 + N / 16 : 8 + 4 + 7 + N / 16);
        }
        for (int i = 0; i < PT_XS; ++i) {
            mbar_init(&xfull[i], 1);
            mbar_init(&xempty[i], SUMS ? 8 : 1);
            mbar_init(&xready[i], 8);
        }
        for (int i = 0; i < PT_PARTS; ++i) {
            mbar_init(&xpfull[i], 8);
            mbar_init(&xpempty[i], 1);
        }
        mbar_init(&gfull, 1);
        mbar_init(&gfree, 7);
        mbar_init(&sdone, 1);
        mbar_init(&sfree, N / 16);
        mbar_init(&hfull, N / 16);
        mbar_init(&yfull, 1);
        mbar_init(&yfree, 4);
        mbar_init(&tailtx, 2);
        mbar_init(&tailfull, 1);
        mbar_init(&alldone, PT_THREADS / 32 - 1);
        abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0) tmem_alloc(&tmem_base, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_launch_dependents();
    pdl_wait();
    if ((SUMS || p.nsums == 0) && blockIdx.x == 0 && tid == 0) *p.status = 0u;      // by the call's first launch
    const uint32_t tm = tmem_base;
    volatile uint32_t *abortp = &abort_flag;

    // unit (rows of a sequence) and heads of this CTA
    const int hs = blockIdx.x % p.head_sets;
    const ScanUnit u = (SUMS ? p.sums : p.units)[blockIdx.x / p.head_sets];
    const int spg = p.head_sets / p.G, g = hs / spg, h0 = g * p.hpg + (hs - g * spg) * p.per_cta, nh = min(p.per_cta, (g + 1) * p.hpg - h0);
    const int nb = (u.n + 127) >> 7, ni = nb * nh;
    const int tail = SUMS ? 0 : u.n & 127;              // rows of the last block, 0: all
    constexpr int PER = SUMS ? 1 : 2;                   // tiles per block: B, C
    auto vec = [&](const VecTurn &v) { return reinterpret_cast<float *>(smem + Mem::VEC) + v.slot * PV_FLOATS; };

    if (PT_R_ISSUE < PT_REGS && warp < 4) regs_down<PT_R_ISSUE>();
    if (warp < 2) {
        const uint32_t on = elect_one();
        const uint32_t sb = smem_u32(smem);
        const uint64_t dK = umma_desc_sw128(sb, 16, 1024), dM = umma_desc_sw128(sb, 16384, 1024);
        const uint32_t loK = (uint32_t)dK, hiK = (uint32_t)(dK >> 32), loM = (uint32_t)dM, hiM = (uint32_t)(dM >> 32);
        // tile k (B of block k / 2, or C) is in place
        auto wait_tile = [&](int k) {
            const bool last = tail && k >= 2 * nb - 2;
            pt_wait(last ? &tailfull : &tfull[k % PT_SLOTS], last ? 0 : (k / PT_SLOTS) & 1, abortp);
        };
        if (warp == 0) {
            // -------------------------------------------------------- G, M X
            if (!SUMS) {
                const uint32_t idG = umma_idesc_bf16(128, 128, false, false), idY = umma_idesc_bf16(128, 64, false, true);
                for (int i = -1, c = -1, j = nh - 1; i < ni; ++i) {
                    if (i >= 0) {
                        pt_wait(&xready[i % PT_XS], (i / PT_XS) & 1, abortp);
                        if (i) pt_wait(&yfree, (i - 1) & 1, abortp);
                        // 64 steps at a time, as their masks get ready; the smaller part first
#pragma unroll 1
                        for (int side = 0; side < 2; ++side) {
                            const uint32_t lX = loM + Mem::X / 16 + (i % PT_XS) * 1024 + side * 512, lM = tm + TM_M + side * 64;
                            pt_wait(&mfull[side], i & 1, abortp);
                            tc_fence_after_sync();
#pragma unroll
                            for (int n = 0; n < 8; ++n)
                                pt_mma_ta(on, side + n, tm + TM_Y, lM + (n < 4 ? 32 : 0) + 8 * (n & 3), umma_desc_words(lX + (n & 3) * 128, hiM), idY);
                            pt_commit(on, &mempty[side]);
                        }
                        pt_commit(on, &yfull);
                    }
                    if (j == nh - 1 && c + 1 < nb) {                 // the next block's scores
                        const int kb = 2 * c + 2, kc = kb + 1;
                        const uint32_t lB = loK + (kb % PT_SLOTS) * (Mem::TILE / 16), lC = loK + (kc % PT_SLOTS) * (Mem::TILE / 16);
                        wait_tile(kb);
                        wait_tile(kc);
                        if (c >= 0) pt_wait(&gfree, c & 1, abortp);
                        tc_fence_after_sync();
#pragma unroll
                        for (int k = 0; k < KN; ++k) {
                            const uint32_t o = (k >> 2) * 1024 + (k & 3) * 2;
                            pt_mma(on, k, tm + TM_G, umma_desc_words(lC + o, hiK), umma_desc_words(lB + o, hiK), idG);
                        }
                        pt_commit(on, &gfull);
                        pt_commit(on, &tempty[kb % PT_SLOTS]);
                        pt_commit(on, &tempty[kc % PT_SLOTS]);
                    }
                    if (++j == nh) {
                        j = 0;
                        ++c;
                    }
                }
            }
        } else {
            // -------------------------------------------------------- S, C H
            const uint32_t idS = umma_idesc_bf16(128, 64, true, true), idC = umma_idesc_bf16(128, 64, false, true);
            const uint32_t lP = loM + Mem::XP / 16, lH = loM + Mem::H / 16;
            VecTurn pt;
            for (int i = 0, c = 0, j = 0; i < ni; ++i) {
                const int kb = PER * c, kc = 2 * c + 1;
                const uint32_t lB = loM + (kb % PT_SLOTS) * (Mem::TILE / 16), lC = loK + (kc % PT_SLOTS) * (Mem::TILE / 16);
                if (j == 0) wait_tile(kb);
                if (i) pt_wait(&sfree, (i - 1) & 1, abortp);
                // 32 steps at a time, so that their parts are made while the ones before are multiplied; the smallest part first
#pragma unroll 1
                for (int part = 0; part < 4; ++part, pt.next()) {
                    pt_wait(&xpfull[pt.slot], pt.odd, abortp);
                    tc_fence_after_sync();
#pragma unroll
                    for (int n = 0; n < 6; ++n) {
                        const uint32_t o = (n % 2) * 128, q = (2 - n / 2) * 256;
                        pt_mma(on, part + n, tm + TM_S, umma_desc_words(lB + 256 * part + o, hiM), umma_desc_words(lP + 768 * pt.slot + q + o, hiM), idS);
                    }
                    pt_commit(on, &xpempty[pt.slot]);
                }
                pt_commit(on, &sdone);
                if (j == nh - 1) pt_commit(on, &tempty[kb % PT_SLOTS]);
                if constexpr (!SUMS) {
                    if (j == 0) wait_tile(kc);
                    pt_wait(&hfull, i & 1, abortp);
                    if (i >= 2) pt_wait(&chfree[i & 1], ((i >> 1) - 1) & 1, abortp);
                    tc_fence_after_sync();
#pragma unroll
                    for (int n = 0; n < 2 * KN; ++n) {               // the smaller part first
                        const uint32_t k = n % KN, o = (k >> 2) * 1024 + (k & 3) * 2;
                        pt_mma(on, n, tm + TM_CH + 64 * (i & 1), umma_desc_words(lC + o, hiK), umma_desc_words(lH + (n < KN ? N * 8 : 0) + k * 128, hiM), idC);
                    }
                    pt_commit(on, &chdone[i & 1]);
                    if (j == nh - 1) pt_commit(on, &tempty[kc % PT_SLOTS]);
                }
                if (++j == nh) {
                    j = 0;
                    ++c;
                }
            }
        }
    } else if (warp < 4) {
        // ------------------------------------------------------------ decays; a lane has four consecutive steps
        const int first = warp - 2;
        float next[4];
        auto fetch = [&](int i) {
            const int c = nh == 2 ? i >> 1 : i, h = nh == 2 ? h0 + (i & 1) : h0;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int t = c * 128 + lane * 4 + m;
                next[m] = t < u.n ? __ldg(p.dt + (u.row0 + t) * p.dt_rs + h) : 0.f;
            }
        };
        const double a2 = (double)__ldg(p.A + h0 + (nh == 2 ? first : 0)) * 1.4426950408889634;
        if (first < ni) fetch(first);
        VecTurn vt;
        vt.next(first);
        for (int i = first; i < ni; i += 2, vt.next(2)) {
            const float4 d = make_float4(next[0], next[1], next[2], next[3]);
            if (i + 2 < ni) fetch(i + 2);
            const double s0 = d.x * a2, s1 = s0 + d.y * a2, s2 = s1 + d.z * a2;
            double run = s2 + d.w * a2;
            const double own = run;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double v = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += v;
            }
            const double before = run - own;
            const double cd[4] = {before + s0, before + s1, before + s2, run};
            float hi[4], lo[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                hi[m] = (float)cd[m];
                lo[m] = (float)(cd[m] - hi[m]);
            }
            const float dd[4] = {d.x, d.y, d.z, d.w};
            if (i >= PT_VECS) pt_wait(&vempty[vt.slot], vt.odd ^ 1u, abortp);
            float *v = vec(vt) + lane * 4;
            auto put = [&](int at, const float (&f)[4]) { *reinterpret_cast<float4 *>(v + at) = make_float4(f[0], f[1], f[2], f[3]); };
            // 2^(cs there - cs here): the differences of the two parts apart
            auto power = [&](float h, float l, float (&f)[4], float sign) {
#pragma unroll
                for (int m = 0; m < 4; ++m) f[m] = pt_ex2(((h - hi[m]) + (l - lo[m])) * sign);
            };
            float f[4], r[4];
            const float hl = __shfl_sync(0xffffffffu, hi[3], 31), ll = __shfl_sync(0xffffffffu, lo[3], 31);
            power(hl, ll, f, 1.f);
#pragma unroll
            for (int m = 0; m < 4; ++m) f[m] *= dd[m];
            put(PV_W, f);
            if (lane == 31) v[PV_DECAY - 124] = pt_ex2(hi[3]) * fmaf(lo[3], 0.69314718f, 1.f);
            put(PV_HI, hi);
            put(PV_LO, lo);
            if constexpr (!SUMS) {
                power(0.f, 0.f, f, -1.f);
                put(PV_E, f);
                put(PV_DT, dd);
                // row sub-tile k, relative to its middle row, or to its first where it does not decay mildly: the columns in front of it and its own
#pragma unroll 1
                for (int k = 0; k < 4; ++k) {
                    const float start = __shfl_sync(0xffffffffu, hi[0], 8 * k), middle = __shfl_sync(0xffffffffu, hi[0], 8 * k + 4);
                    const bool mild = pt_mild(start, middle, __shfl_sync(0xffffffffu, hi[3], 8 * k + 7));
                    const float h = mild ? middle : start, l = __shfl_sync(0xffffffffu, lo[0], 8 * k + (mild ? 4 : 0));
                    power(h, l, f, 1.f);
#pragma unroll
                    for (int m = 0; m < 4; ++m) f[m] *= dd[m];
                    if (lane < 8 * (k + 1)) put(PV_F + 16 * k * (k + 1), f);
                    if (lane >> 3 == k) {
                        power(h, l, r, -1.f);
#pragma unroll
                        for (int m = 0; m < 4; ++m) r[m] = mild ? r[m] : 1.f;
                        put(PV_R, r);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&vfull[vt.slot]);
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------ parts of x'
        regs_down<PT_R_X>();
        const int th = tid - 128, r0 = th >> 3, ch = th & 7;
        const uint32_t off = r0 * 128 + ((ch ^ (r0 & 7)) << 4);      // rows 32 apart have the same swizzle
        VecTurn vt, pt;
        for (int i = 0; i < ni; ++i, vt.next()) {
            int left = u.n - (nh == 2 ? i >> 1 : i) * 128 - r0;
            unsigned char *xs = smem + Mem::X + (i % PT_XS) * 16384 + off;
            const float *w = vec(vt) + PV_W + r0;
            pt_wait(&vfull[vt.slot], vt.odd, abortp);
            pt_wait(&xfull[i % PT_XS], (i / PT_XS) & 1, abortp);
#pragma unroll 1
            for (int part = 0; part < 4; ++part, pt.next()) {
                uint4 xr = *reinterpret_cast<const uint4 *>(xs);
                const float wr = *w;
                if (left <= 0) *reinterpret_cast<uint4 *>(xs) = xr = make_uint4(0, 0, 0, 0);
                const uint32_t e[4] = {xr.x, xr.y, xr.z, xr.w};
                uint32_t o[4][3];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float2 f = __fmul2_rn(pt_unpack(e[m]), make_float2(wr, wr));
                    split2(f.x, f.y, o[m]);
                }
                if (part == 3 || i) pt_wait(&xpempty[pt.slot], pt.odd ^ 1u, abortp);      // the parts before have been read
                unsigned char *xp = smem + Mem::XP + pt.slot * 12288 + off;
#pragma unroll
                for (int s = 0; s < 3; ++s) *reinterpret_cast<uint4 *>(xp + s * 4096) = make_uint4(o[0][s], o[1][s], o[2][s], o[3][s]);
                xs += 4096, w += 32, left -= 32;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&xpfull[pt.slot]);
            }
            if (lane == 0) {
                if (SUMS) mbar_arrive(&xempty[i % PT_XS]);
                else mbar_arrive(&xready[i % PT_XS]);
                mbar_arrive(&vempty[vt.slot]);
            }
        }
    } else if (warp < 16) {
        // ------------------------------------------------------------ outputs, a row per thread, in the place of its row of x and from there by TMA:
        // rows of 128 bytes one by one kept the memory pipe so busy that the other roles' loads from shared and tensor memory took 2000 cycles
        regs_down<PT_R_OUT>();
        const int q = warp & 3, r = q * 32 + lane, th = tid - 384;
        const uint32_t tl = tm + ((uint32_t)(q * 32) << 16);
        VecTurn vt;
        for (int i = 0, c = 0, j = 0; i < (SUMS ? 0 : ni); ++i, vt.next()) {
            const float Dh = __ldg(p.D + h0 + j);
            pt_wait(&vfull[vt.slot], vt.odd, abortp);
            const float et = vec(vt)[PV_E + r], rt = vec(vt)[PV_R + r];
            __syncwarp();
            if (lane == 0) mbar_arrive(&vempty[vt.slot]);
            unsigned char *xs = smem + Mem::X + (i % PT_XS) * 16384;
            const float2 e2 = make_float2(et, et), r2 = make_float2(rt, rt), D2 = make_float2(Dh, Dh);
            pt_wait(&chdone[i & 1], (i >> 1) & 1, abortp);
            pt_wait(&yfull, i & 1, abortp);              // so x has been read by all others: by the product, which came behind its parts
            tc_fence_after_sync();
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                float a[16], b[16];
                uint4 xv[2];
                tmem_ld16_nowait(tl + TM_CH + 64 * (i & 1) + 16 * k, a);
                tmem_ld16_nowait(tl + TM_Y + 16 * k, b);
#pragma unroll
                for (int n = 0; n < 2; ++n) xv[n] = *reinterpret_cast<const uint4 *>(xs + r * 128 + (((2 * k + n) ^ (r & 7)) << 4));
                tmem_ld_wait16(a);
                tmem_ld_wait16(b);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint32_t xe[4] = {xv[n].x, xv[n].y, xv[n].z, xv[n].w};
                    uint32_t w[4];
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const int f = 8 * n + 2 * m;
                        const float2 s = __ffma2_rn(make_float2(b[f], b[f + 1]), r2, __fmul2_rn(pt_unpack(xe[m]), D2));
                        const float2 y = __ffma2_rn(make_float2(a[f], a[f + 1]), e2, s);
                        w[m] = pt_pack(y.x, y.y);
                    }
                    *reinterpret_cast<uint4 *>(xs + r * 128 + (((2 * k + n) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            tc_fence_before_sync();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&yfree), mbar_arrive(&chfree[i & 1]);
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const int left = u.n - c * 128, row = u.row0 + c * 128;
            if (left >= 128) {
                if (th == 0) {
                    tma_store_3d(&tmY, xs, (h0 + j) * 64, row, 0);
                    tma_store_commit();
                    tma_store_wait_read();
                    mbar_arrive(&xempty[i % PT_XS]);
                }
            } else {                                     // the last block: its rows of x are followed by no others
                for (int o = th; o < left * 8; o += 128)
                    *reinterpret_cast<uint4 *>((__nv_bfloat16 *)p.y + (row + (o >> 3)) * p.y_rs + (h0 + j) * 64 + (o & 7) * 8) =
                        *reinterpret_cast<const uint4 *>(xs + (o >> 3) * 128 + (((o & 7) ^ ((o >> 3) & 7)) << 4));
            }
            if (++j == nh) {
                j = 0;
                ++c;
            }
        }
        if (th == 0) tma_store_wait_all();
    } else if (warp < 24) {
        if (PT_R_MASK < PT_REGS) regs_down<PT_R_MASK>();
        const int q = warp & 3, half = (warp - 16) >> 2, t = q * 32 + lane;
        const uint32_t tl = tm + ((uint32_t)(q * 32) << 16);
        {
            uint32_t z[16];
#pragma unroll
            for (int m = 0; m < 16; ++m) z[m] = 0u;
            for (int k = half; k < 4; k += 2)
                if (k > q) {                                         // above the diagonal, for good
                    tmem_st16(tl + TM_M + 64 * (k >> 1) + 16 * half, z);
                    tmem_st16(tl + TM_M + 64 * (k >> 1) + 16 * half + 32, z);
                }
            tmem_st_wait();
            tc_fence_before_sync();
        }
        if (warp == 20) {
            // -------------------------------------------------------- loads
            for (int c = 0, k = 0; c < nb; ++c) {
                const bool part = tail && c == nb - 1;
#pragma unroll 1
                for (int n = 0; n < PER + nh; ++n) {                 // B, x of the first head, C, x of the second: C's place is free last
                    const bool tile = n == 0 || (!SUMS && n == 2);
                    const int j = n == 1 ? 0 : 1, i = c * nh + j, slot = tile ? k % PT_SLOTS : i % PT_XS;
                    uint64_t *bar = tile ? &tfull[slot] : &xfull[slot];
                    const CUtensorMap *map = !tile ? &tmX : n ? &tmC : &tmB;
                    if (tile ? k >= PT_SLOTS : i >= PT_XS)
                        pt_wait_watched(tile ? &tempty[slot] : &xempty[slot], tile ? (k / PT_SLOTS - 1) & 1 : (i / PT_XS - 1) & 1, abortp);
                    if (tile && part) bar = &tailtx;
                    if (elect_one())
                        tma_load_tile(smem + (tile ? slot * Mem::TILE : Mem::X + slot * 16384), map, bar, tile ? N / 64 : 1, tile ? g * N : (h0 + j) * 64,
                                      u.row0 + c * 128);
                    __syncwarp();
                    k += tile;
                    if (!part || n != 2) continue;
                    // The last block's B and C: zeros from the sequence's end on.  Ahead of the second head's x, which waits for products that come
                    // behind this block's scores.
                    pt_wait_watched(&tailtx, 0, abortp);
                    for (int m = k - 2; m < k; ++m)
                        for (int b = 0; b < N / 64; ++b)
                            for (int o = tail * 8 + lane; o < 128 * 8; o += 32)
                                *reinterpret_cast<uint4 *>(smem + (m % PT_SLOTS) * Mem::TILE + b * 16384 + o * 16) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&tailfull);
                }
            }
            pt_wait_watched(&alldone, 0, abortp);
        } else if (!SUMS) {
            // -------------------------------------------------------- mask.  Warp (q, half): rows 32 q .., column sub-tiles half and half + 2
            VecTurn vt;
            for (int i = 0, c = 0, j = 0; i < ni; ++i, vt.next()) {
                const float *v = vec(vt);
                pt_wait(&vfull[vt.slot], vt.odd, abortp);
                const bool mild = pt_mild(v[PV_HI + q * 32], v[PV_HI + q * 32 + 16], v[PV_HI + q * 32 + 31]);
                const float *F = v + PV_F + 16 * q * (q + 1);        // column factors of row sub-tile q
                if (j == 0) pt_wait(&gfull, c & 1, abortp);
                tc_fence_after_sync();
                // a sub-tile of each half of the columns, 16 at a time
#pragma unroll 1
                for (int side = 0; side < 2; ++side) {
                    const int sub = 2 * side + half;
                    if (i) pt_wait(&mempty[side], (i - 1) & 1, abortp);
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int k = 2 * sub; k < 2 * sub + 2 && sub <= q; ++k) {
                        const uint32_t to = tl + TM_M + 64 * side + 8 * (k & 3);
                        float a[16];
                        __syncwarp();
                        tmem_ld16(tl + TM_G + 16 * k, a);
                        if (mild) {
#pragma unroll
                            for (int m = 0; m < 16; m += 4) {
                                const float4 f = *reinterpret_cast<const float4 *>(F + 16 * k + m);
                                const float2 x0 = __fmul2_rn(make_float2(a[m], a[m + 1]), make_float2(f.x, f.y));
                                const float2 x1 = __fmul2_rn(make_float2(a[m + 2], a[m + 3]), make_float2(f.z, f.w));
                                a[m] = x0.x; a[m + 1] = x0.y; a[m + 2] = x1.x; a[m + 3] = x1.y;
                            }
                        } else {                                         // with the row's factor, on the diagonal element by element
                            const float hi = v[PV_HI + t], lo = v[PV_LO + t];
                            const float rf = pt_ex2((hi - v[PV_HI + q * 32]) + (lo - v[PV_LO + q * 32]));
#pragma unroll
                            for (int m = 0; m < 16; m += 4) {
                                const int s = 16 * k + m;
                                float4 f;
                                if (k < 2 * q) {
                                    f = *reinterpret_cast<const float4 *>(F + s);
                                    f.x *= rf, f.y *= rf, f.z *= rf, f.w *= rf;
                                } else {
                                    const float4 sh = *reinterpret_cast<const float4 *>(v + PV_HI + s), sl = *reinterpret_cast<const float4 *>(v + PV_LO + s);
                                    f = *reinterpret_cast<const float4 *>(v + PV_DT + s);
                                    f.x *= pt_ex2((hi - sh.x) + (lo - sl.x)), f.y *= pt_ex2((hi - sh.y) + (lo - sl.y));
                                    f.z *= pt_ex2((hi - sh.z) + (lo - sl.z)), f.w *= pt_ex2((hi - sh.w) + (lo - sl.w));
                                }
                                a[m] *= f.x, a[m + 1] *= f.y, a[m + 2] *= f.z, a[m + 3] *= f.w;
                            }
                        }
                        if (k >= 2 * q) {
#pragma unroll
                            for (int m = 0; m < 16; ++m) a[m] = 16 * k + m <= t ? a[m] : 0.f;
                        }
                        uint32_t o[8], r[8];
#pragma unroll
                        for (int m = 0; m < 8; ++m) pt_pack2(a[2 * m], a[2 * m + 1], o[m], r[m]);
                        __syncwarp();
                        tmem_st8(to, o);
                        tmem_st8(to + 32, r);
                    }
                    tmem_st_wait();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&mfull[side]);
                }
                if (lane == 0) {
                    if (j == nh - 1) mbar_arrive(&gfree);
                    mbar_arrive(&vempty[vt.slot]);
                }
                if (++j == nh) {
                    j = 0;
                    ++c;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ states; a thread has 32 of p of one n, of each head
        regs_up<PT_R_STATE>();
        const int q = warp & 3, half = (warp - 24) >> 2, n = q * 32 + lane;
        if (n < N) {
            const uint32_t tl = tm + ((uint32_t)(q * 32) << 16) + TM_S + 32 * half;
            float *st = u.slot < 0 ? nullptr : p.state + u.slot * p.state_stride + (int64_t)(h0 * 64 + 32 * half) * N + n;
            const int64_t HPN = (int64_t)p.H * 64 * N;
            float *entry = p.entries + u.entry * HPN + (int64_t)(h0 * 64 + 32 * half) * N + n;      // of a cut sequence
            const double *dec = p.decays + (int64_t)u.entry * p.H + h0;
            float h[2][32];
            double decayed[2] = {0., 0.};
            const float *from = !SUMS && u.entry >= 0 ? entry : st;      // the slot may have been replaced by then
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    h[j][k] = u.range == 0 && u.carry && j < nh ? from[(j * 64 + k) * N] : 0.f;
                    if (SUMS && u.range == 0 && u.carry && j < nh) entry[(j * 64 + k) * N] = h[j][k];
                }
            if (!SUMS) {
                // the state behind range 0, then the sums of the ranges up to this one
#pragma unroll 1
                for (int k = 1; k <= u.range; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (j >= nh) break;
                        const float d = exp2f((float)dec[k * p.H + j]);
                        const float *e = entry + k * HPN + j * 64 * N;
#pragma unroll
                        for (int m = 0; m < 32; ++m) h[j][m] = fmaf(h[j][m], d, e[m * N]);
                    }
            }
            unsigned char *hp = smem + Mem::H + n * 128;
            VecTurn vt;
            auto step = [&](float (&s)[32], double &dl, int i) {
                if constexpr (!SUMS) {
                    if (i) pt_wait(&chdone[(i - 1) & 1], ((i - 1) >> 1) & 1, abortp);        // the state of the item before has been read
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t w[4], r[4];
#pragma unroll
                        for (int m = 0; m < 4; ++m) pt_pack2(s[8 * k + 2 * m], s[8 * k + 2 * m + 1], w[m], r[m]);
                        unsigned char *to = hp + (((4 * half + k) ^ (n & 7)) << 4);
                        *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(to + N * 128) = make_uint4(r[0], r[1], r[2], r[3]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&hfull);
                }
                pt_wait(&vfull[vt.slot], vt.odd, abortp);
                const float2 d2 = make_float2(vec(vt)[PV_DECAY], vec(vt)[PV_DECAY]);
                if (SUMS) dl += (double)vec(vt)[PV_HI + 127] + vec(vt)[PV_LO + 127];
                pt_wait(&sdone, i & 1, abortp);
                tc_fence_after_sync();
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a[16];
                    tmem_ld16(tl + 16 * k, a);
#pragma unroll
                    for (int m = 0; m < 8; ++m) {
                        const float2 r = __ffma2_rn(make_float2(s[16 * k + 2 * m], s[16 * k + 2 * m + 1]), d2, make_float2(a[2 * m], a[2 * m + 1]));
                        s[16 * k + 2 * m] = r.x;
                        s[16 * k + 2 * m + 1] = r.y;
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sfree);
                    mbar_arrive(&vempty[vt.slot]);
                }
                vt.next();
            };
            for (int i = 0; i < ni; ++i) {
                step(h[0], decayed[0], i);
                if (nh == 2) step(h[1], decayed[1], ++i);
            }
            float *to = SUMS ? entry + (u.range + 1) * HPN : u.last && (nb > 0 || !u.carry) ? st : nullptr;
            if (to) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (j < nh) to[(j * 64 + k) * N] = h[j][k];
            }
            if (SUMS && n < nh && half == 0) p.decays[(int64_t)(u.entry + u.range + 1) * p.H + h0 + n] = n ? decayed[1] : decayed[0];
        }
    }
    __syncwarp();
    if (warp != 20 && lane == 0) mbar_arrive(&alldone);
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tm, 512);
    if (tid == 0 && abort_flag) {
        atomicExch(p.status, 1u);
        for (const long long start = clock64(); clock64() - start < kWaitAbortedClk;) {}     // copies that are still under way land in this CTA's memory
    }
}

// The split of registers by role adds up to what 64 per thread at launch leave; fewer, and the kernel would wait for them for good.
template <auto K> static cudaError_t has_regs() {
    static std::atomic<int> regs{0};
    if (!regs.load(std::memory_order_relaxed)) {
        cudaFuncAttributes a;
        const cudaError_t e = cudaFuncGetAttributes(&a, K);
        if (e != cudaSuccess) return e;
        regs.store(a.numRegs, std::memory_order_relaxed);
    }
    return regs.load(std::memory_order_relaxed) == PT_REGS ? cudaSuccess : cudaErrorInvalidConfiguration;
}

cudaError_t launch_packed_tc(const PackedParams &p, bool sums, cudaStream_t st) {
    const dim3 grid((unsigned)((sums ? p.nsums : p.nunits) * p.head_sets)), block(PT_THREADS);
    CUtensorMap x, b, c, y;
    if (!tc_rows_map(&x, p.x, (uint64_t)p.H * 64, p.rows, p.x_rs) || !tc_rows_map(&b, p.Bm, (uint64_t)p.G * p.N, p.rows, p.b_rs) ||
        !tc_rows_map(&c, p.Cm, (uint64_t)p.G * p.N, p.rows, p.c_rs) || !tc_rows_map(&y, p.y, (uint64_t)p.H * 64, p.rows, p.y_rs))
        return cudaErrorInvalidValue;
#define SSD_PACKED_RUN(N, S)                                                                \
    do {                                                                                    \
        cudaError_t e = allow_smem<k_packed_tc<N, S>>(PtMem<N>::BYTES);                     \
        if (e == cudaSuccess) e = has_regs<k_packed_tc<N, S>>();                            \
        if (e != cudaSuccess) return e;                                                     \
        return launch_pdl(k_packed_tc<N, S>, grid, block, PtMem<N>::BYTES, st, p, x, b, c, y); \
    } while (0)
#define SSD_PACKED_TC(N)                 \
    do {                                 \
        if (sums) SSD_PACKED_RUN(N, true); \
        SSD_PACKED_RUN(N, false);        \
    } while (0)
    if (p.N == 128) SSD_PACKED_TC(128); else SSD_PACKED_TC(64);
#undef SSD_PACKED_TC
#undef SSD_PACKED_RUN
}

}  // namespace ssd
