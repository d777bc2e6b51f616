// The gated feed-forward sub-layer  Y = (act(X Wg^T) * (X Wu^T)) Wd^T (+ R)  and its gradients.
//
// Hidden units are taken 64 at a time (a block).  G and U of a block are one product of 128 columns, for Wg's and Wu's
// rows stand one behind the other in shared memory; the activations are formed in registers, rounded to bf16 and go back
// into tensor memory as the A operand of the next product, so no hidden value reaches global memory in any direction.
//
// glu_fwd_kernel    per 256-row tile, per block:  G|U = X [Wg; Wu]^T,   Y += (act(G) * U) Wd^T
// glu_dx_kernel     per 256-row tile, per block:  G|U again, dA = dY Wd,   dX += dG Wg + dU Wu
//                   with  dU = dA act(G),  dG = dA U act'(G)
// glu_dw_kernel     a CTA keeps one block and walks 128-row tiles:  G|U, dA again,   [dWg | dWu]^T += X^T [dG | dU],
//                   dWd += dY^T (act(G) * U),   accumulated in tensor memory (192 columns of fp32)
// glu_reduce_kernel sums the accumulators of the CTAs that share a block, in a fixed order
//
// Wg and Wu, 128 bytes of a row at a time, serve as K-major operands of the first products and, the same bytes read
// MN-major, of dX; Wd likewise.  X and dY tiles likewise in glu_dw_kernel.  Nothing is transposed in memory.
//
// The gradients compute G, U and dA twice, in eleven products instead of eight: the weights' accumulators of a row tile's
// whole width (768 KB for d_ff = 512) fit no SM, dX of one block would have to be summed over all of them, and the hidden
// gradients through memory are 3 KB a row each way (950 us for a million rows; glu_dw_kernel takes 830 to 890).
//
// Rounding: the hidden values (act(G) U; dG, dU) go into the second products in bf16, the type of the operands they meet, off
// by at most 2^-8 of themselves; everything else (products, activations, sums over rows and blocks) is held in 32 bits.
//
// 1.01M rows, d_ff = 512, SiLU, back to back: forward 405 to 413 us (980 TFLOP/s, 58 % of the measured burst rate), gradients 1 475 to
// 1 490 us; the board is at its 1 kW then and the clock at 1.5 to 1.65 of 1.97 GHz.  In short runs on 208 384 rows 76 us forward,
// 112 for dX and 172 for the weights (back to back 84, 128 and 185).  d_ff = 2048 on 101 000 rows: 120 to 123 us (1 300 TFLOP/s).

#include <cuda.h>

#include <atomic>

#include "dg4_internal.h"
#include "dg4_launch.cuh"
#include "dg4_pairs.cuh"
#include "dg4_sm100.cuh"

using namespace sm100;

namespace {

constexpr int kTileM = 128;
constexpr int kBlock = 64;                         // hidden units at a time
constexpr int kHalfBytes = kTileM * 128;           // 64 columns of a 128-row tile
constexpr int kTileBytes = 2 * kHalfBytes;
constexpr int kEpiWarps = 16;                      // four per scheduler: some compute while others wait for tensor memory
constexpr int kEl = 16;                            // a block's values of a row that an epilogue thread takes, by its warp
constexpr int kCtrlWarps = 4;                      // warp 0, 2, 3: loads, warp 1: products
constexpr int kThreads = (kCtrlWarps + kEpiWarps) * 32;
constexpr int kSetWarps = kEpiWarps / 2;           // forward and dX: half of the epilogue warps take every other block
constexpr int kSmemLimit = 232448;                 // what one CTA may hold
constexpr int kMaxDff = 8192;                      // 128 blocks: glu_dw_kernel has a CTA for each at least

// A place in a ring of n and the parity of its present round.
struct Turn {
    int at = 0;
    uint32_t odd = 0;
    __device__ __forceinline__ void next(int n) {
        if (++at == n) { at = 0; odd ^= 1u; }
    }
};

__device__ __forceinline__ void st_shared_v4(uint32_t addr, const uint32_t* r) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void ld_shared_v4(uint32_t addr, uint32_t* r) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ld_global_v4(const void* p, uint32_t* r) {
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void st_global_v4(void* p, const uint32_t* r) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t pk;
    asm("cvt.rn.bf16x2.f32 %0, %2, %1;" : "=r"(pk) : "f"(lo), "f"(hi));
    return pk;
}
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float ex2_small(float x) { float y; asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }   // below 2^-126 too
__device__ __forceinline__ float min_or_nan(float x, float y) { float z; asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y)); return z; }
__device__ __forceinline__ float relu(float x) { float y; asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// SiLU x * sigmoid(x), GELU by its tanh form x * sigmoid(2 sqrt(2/pi) (x + 0.044715 x^3)), ReLU max(0, x).
constexpr float kLog2e = 1.4426950408889634f, kGelu1 = 1.5957691216057308f, kGelu3 = 0.07135481282052f;
// sigmoid(p(g)) of eight values.  The special-function unit is what would bound the epilogues (an exponential and a reciprocal
// per value: 1024 clocks per block and SM, the products of the forward pass 768), so four values share a reciprocal:
// 1/x = y / (xy).  Where the product of the four is too large for that (2^126; four gates near -22, or one below -87), and for
// NaN, which would reach the other values, each has its own, from t = exp(p): t / (1 + t) keeps subnormal values, which a gate of
// -90 makes normal numbers of again.
template <int ACT>
__device__ __forceinline__ void sigmoid8(const float* g, float* s) {
    float e[8];
    bool each = false;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        Pair d[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const Pair x = pair(g[i + 2 * j], g[i + 2 * j + 1]);
            Pair p;
            if (ACT == DG4_ACT_SILU) p = mul2(x, pair(-kLog2e, -kLog2e));
            else p = mul2(x, fma2(mul2(x, x), pair(-kLog2e * kGelu3, -kLog2e * kGelu3), pair(-kLog2e * kGelu1, -kLog2e * kGelu1)));
            split(p, e[i + 2 * j], e[i + 2 * j + 1]);
            d[j] = add2(pair(ex2(e[i + 2 * j]), ex2(e[i + 2 * j + 1])), pair(1.f, 1.f));
        }
        float d0, d1, d2, d3;
        split(d[0], d0, d1);
        split(d[1], d2, d3);
        const float d01 = d0 * d1, d23 = d2 * d3, all = d01 * d23, r = rcp(all);
        each = each || !(all <= 0x1p126f);
        const float r01 = r * d23, r23 = r * d01;
        s[i] = r01 * d1; s[i + 1] = r01 * d0; s[i + 2] = r23 * d3; s[i + 3] = r23 * d2;
    }
    if (each) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = ex2_small(min_or_nan(-e[i], 126.f));
            s[i] = t * rcp(1.f + t);
        }
    }
}
// Sixteen values act(g) * u as eight pairs of bf16.
template <int ACT>
__device__ __forceinline__ void gated(const uint32_t* g_bits, const uint32_t* u_bits, uint32_t* out) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float *g = reinterpret_cast<const float*>(g_bits) + 8 * c, *u = reinterpret_cast<const float*>(u_bits) + 8 * c;
        float s[8];
        if (ACT != DG4_ACT_RELU) sigmoid8<ACT>(g, s);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            Pair x = pair(g[i], g[i + 1]);
            if (ACT == DG4_ACT_RELU) x = pair(relu(g[i]), relu(g[i + 1]));
            else x = mul2(x, pair(s[i], s[i + 1]));
            float lo, hi;
            split(mul2(x, pair(u[i], u[i + 1])), lo, hi);
            out[4 * c + i / 2] = pack_bf16(lo, hi);
        }
    }
}
// The same backward, for h = dL/d(act(g) u):  dg = h u act'(g),  du = h act(g),  a = act(g) u (not asked for: null), with
// act'(g) = s + g s (1 - s) p'(g), s = sigmoid(p(g)).  ReLU's dg is taken and not multiplied: zero behind a closed gate
// whatever h and u are, and not a number where the gate is none.
template <int ACT, bool VALUES>
__device__ __forceinline__ void gated_bwd(const uint32_t* g_bits, const uint32_t* u_bits, const uint32_t* h_bits, uint32_t* dg,
                                          uint32_t* du, uint32_t* a) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float *g = reinterpret_cast<const float*>(g_bits) + 8 * c, *u = reinterpret_cast<const float*>(u_bits) + 8 * c,
                    *h = reinterpret_cast<const float*>(h_bits) + 8 * c;
        float s[8];
        if (ACT != DG4_ACT_RELU) sigmoid8<ACT>(g, s);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const Pair uu = pair(u[i], u[i + 1]), hh = pair(h[i], h[i + 1]);
            Pair act, slope;
            if (ACT == DG4_ACT_RELU) {
                act = pair(relu(g[i]), relu(g[i + 1]));
            } else {
                const Pair x = pair(g[i], g[i + 1]), ss = pair(s[i], s[i + 1]);
                act = mul2(x, ss);
                const Pair rest = fma2(ss, pair(-1.f, -1.f), pair(1.f, 1.f));
                if (ACT == DG4_ACT_GELU) {
                    // beyond |g| = 1000 s or 1 - s is zero: p' is kept finite there
                    float x0, x1;
                    split(mul2(x, x), x0, x1);
                    const Pair dp = fma2(pair(fminf(x0, 1e6f), fminf(x1, 1e6f)), pair(3.f * kGelu3, 3.f * kGelu3), pair(kGelu1, kGelu1));
                    slope = fma2(mul2(act, rest), dp, ss);
                } else {
                    slope = fma2(act, rest, ss);
                }
            }
            float lo, hi;
            split(mul2(hh, act), lo, hi);
            du[4 * c + i / 2] = pack_bf16(lo, hi);
            if (ACT == DG4_ACT_RELU) {
                split(mul2(hh, uu), lo, hi);
                lo = g[i] > 0.f ? lo : relu(g[i]);
                hi = g[i + 1] > 0.f ? hi : relu(g[i + 1]);
            } else {
                split(mul2(mul2(hh, uu), slope), lo, hi);
            }
            dg[4 * c + i / 2] = pack_bf16(lo, hi);
            if (VALUES) {
                split(mul2(act, uu), lo, hi);
                a[4 * c + i / 2] = pack_bf16(lo, hi);
            }
        }
    }
}

struct Params {
    int32_t n, d_ff, n_tiles, n_blocks;
    int32_t splits;                          // pairs of CTAs that share a tile's blocks: 1, 2 or 4
    const __nv_bfloat16* R; int64_t ldr;     // forward: nullable residual
    __nv_bfloat16* out; int64_t ldo;         // Y, or dX
    int32_t* status;
    uint32_t poll_limit;
};

template <class Bars>
__device__ __forceinline__ void raise_timeout(Bars* bars, int32_t* status) {
    atomicExch(&bars->abort_flag, 1u);
    if (status) atomicCAS(status, 0, (int)DG4_ERR_TIMEOUT);
}

// Whether a phase has completed, for a converged warp: a third of a waiting instruction's time, of which the loops below would
// spend more than the products take.
__device__ __forceinline__ bool has_come(uint32_t bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_test(bar, parity) ? 1 : 0) != 0;
}
template <class Bars>
__device__ __forceinline__ bool await(Bars* bars, uint32_t bar, uint32_t parity, uint32_t limit) {
    if (has_come(bar, parity)) return true;
    if (__any_sync(0xffffffffu, *(volatile uint32_t*)&bars->abort_flag != 0)) return false;
    return mbar_wait_relaxed_warp(bar, parity, limit);
}

// The pair's form: the other CTA's roles are told too.
template <class Bars>
__device__ __forceinline__ void raise_timeout_pair(Bars* bars, int32_t* status, uint32_t in_cluster) {
    raise_timeout(bars, status);
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(smem_u32(&bars->abort_flag), in_cluster ^ 1u)), "r"(1u) : "memory");
}

// Few rows: the pairs of a cluster share a tile, each with every `splits`-th block, and their sums are joined through
// distributed shared memory, each pair finishing 128 / splits of the columns.  The epilogue warps send the others' columns of
// the sum (tensor memory, columns 0..127) into the first 64 KB of their CTAs' shared memory, which nothing uses any more
// (`send`); behind a barrier of the cluster each pair adds the parts up in the order of the pairs (`collect`).
struct Split {
    int splits, split, part, quad, lane;                         // part: 32 of the 128 columns
    uint32_t tmem, base, rank;
    __device__ __forceinline__ int owner() const { return part * splits / 4; }
    // 128 rows of 32 columns in fp32, the 16-byte pieces of a row swizzled
    __device__ __forceinline__ uint32_t slot(int from, int piece) const {
        const int row = quad * 32 + lane, at = from * (4 / splits) + part % (4 / splits);
        return base + (uint32_t)(at * 16384 + row * 128 + ((piece ^ (row & 7)) << 4));
    }
    __device__ __forceinline__ void load(uint32_t* y) const {
        tmem_ld_32x32(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(part * 32), y);
        tmem_ld_wait();
    }
    __device__ __forceinline__ void send() const {
        if (owner() == split) return;
        uint32_t y[32];
        load(y);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            asm volatile("st.shared::cluster.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(cluster_addr(slot(split, i), (uint32_t)owner() * 2 + rank)),
                         "r"(y[4 * i]), "r"(y[4 * i + 1]), "r"(y[4 * i + 2]), "r"(y[4 * i + 3]) : "memory");
    }
    // `row`: this lane's row of the tensors, -1 if there is none.  R (nullable): its 32 values are fetched by `residual`.
    __device__ __forceinline__ void residual(uint32_t* r, int64_t row, const __nv_bfloat16* R, int64_t ldr) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) r[i] = 0u;
        if (owner() != split || row < 0 || !R) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) ld_global_v4(R + row * ldr + part * 32 + i * 8, r + 4 * i);
    }
    __device__ __forceinline__ void collect(int64_t row, const uint32_t* r, __nv_bfloat16* out, int64_t ldo) const {
        if (owner() != split) return;
        uint32_t own[32];
        load(own);
        if (row < 0) return;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {                             // eight columns
            float f[8] = {};
            for (int q = 0; q < splits; ++q) {
                uint32_t v[8];
                if (q != split) {
                    ld_shared_v4(slot(q, i), v);
                    ld_shared_v4(slot(q, i + 1), v + 4);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] += __uint_as_float(q != split ? v[e] : own[4 * i + e]);
            }
            const int64_t col = part * 32 + i * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[2 * e] += __uint_as_float(r[2 * i + e] << 16);
                f[2 * e + 1] += __uint_as_float(r[2 * i + e] & 0xffff0000u);
            }
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = pack_bf16(f[2 * e], f[2 * e + 1]);
            st_global_v4(out + row * ldo + col, o);
        }
    }
};

// One block's Wg and Wu: two panels of 64 inputs, each 64 rows of Wg and 64 of Wu.
__device__ __forceinline__ void load_gu(const CUtensorMap* wg, const CUtensorMap* wu, uint32_t dst, int block, uint32_t bar) {
    for (int h = 0; h < 2; ++h) {
        tma_load_2d(dst + h * kHalfBytes, wg, h * 64, block * kBlock, bar);
        tma_load_2d(dst + h * kHalfBytes + kBlock * 128, wu, h * 64, block * kBlock, bar);
    }
}
__device__ __forceinline__ void load_tile(const CUtensorMap* map, uint32_t dst, int row0, uint32_t bar) {
    for (int h = 0; h < 2; ++h) tma_load_2d(dst + h * kHalfBytes, map, h * 64, row0, bar);
}
__device__ __forceinline__ void prefetch_tile(const CUtensorMap* map, int row0) {
    for (int h = 0; h < 2; ++h)
        asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(h * 64), "r"(row0) : "memory");
}
constexpr uint64_t kStepMn = 2048 >> 4;            // sixteen K of an MN-major operand, in descriptor units

// ---------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------
// A pair of CTAs takes 256 rows.  Each fetches half of every block's weights (one Wg, the other Wu, and each half of Wd's
// outputs), and the products read both halves: half the traffic from L2 and half the reads of shared memory per product,
// which bound a CTA alone (48 KB of weights in, 80 KB of operands read per block: 1000 clocks, where the products take 768).
// The CTA of rank 0 issues the products for both; rank 1's warp 1 passes on which of its loads have come.
//
// Tensor memory (each CTA its rows): Y in columns 0..127, three G|U buffers behind it, so that the products of two blocks
// run ahead of the epilogue of a third.  The activations of a block overwrite its G, 16 values in 8 of the columns they were
// computed from.
namespace fwd {
constexpr int kStages = 5, kBufs = 3;
constexpr int kGuBytes = kBlock * 256, kWdBytes = 64 * 128;       // this CTA's half of [Wg; Wu], and of Wd
constexpr int kStageBytes = kGuBytes + kWdBytes, kOffW = 2 * kTileBytes, kOffR = kOffW + kStages * kStageBytes, kOffBars = kOffR + kTileBytes;
struct Bars {
    uint64_t x_full[2], x_empty[2], r_full[2], r_empty[2], w_full[kStages], w_empty[kStages];
    // rank 0's, both CTAs arrive: a block's weights have come (for a tile's first block X too), its activations are there, Y
    // has been read
    uint64_t ready[kStages], a_ready[kBufs], y_empty;
    uint64_t acc_full[kBufs];
    uint64_t y_full[2], drain;                                    // those of two tiles in turn: a set of warps may see every other one
    uint32_t tmem_base, abort_flag;
};
constexpr int kSmem = kOffBars + (int)sizeof(Bars) + 1024;        // 1024: the base is aligned by hand
static_assert(kSmem <= kSmemLimit, "shared memory");
}  // namespace fwd

template <int ACT>
__global__ void __launch_bounds__(kThreads, 1)
glu_fwd_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_wg,
               const __grid_constant__ CUtensorMap map_wu, const __grid_constant__ CUtensorMap map_wd,
               const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_y, Params p) {
    using namespace fwd;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    Bars* bars = reinterpret_cast<Bars*>(smem_raw + (base - smem_u32(smem_raw)) + kOffBars);
    const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t in_cluster = cluster_rank(), rank = in_cluster & 1u, lead = in_cluster & ~1u, mask = 3u << lead;
    const int splits = p.splits, split = (int)(in_cluster >> 1), nb = (p.n_blocks - split + splits - 1) / splits;   // this pair's blocks
    auto unit_of = [&](int b) { return (b * splits + split) * kBlock; };                                           // and their first units
    volatile uint32_t* abort_flag = &bars->abort_flag;
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(bar(bars->x_full[i]), 1); mbar_init(bar(bars->x_empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(bar(bars->r_full[i]), 1); mbar_init(bar(bars->r_empty[i]), kSetWarps); }
        for (int i = 0; i < kStages; ++i) { mbar_init(bar(bars->w_full[i]), 1); mbar_init(bar(bars->w_empty[i]), 1); mbar_init(bar(bars->ready[i]), 2); }
        for (int i = 0; i < kBufs; ++i) { mbar_init(bar(bars->acc_full[i]), 1); mbar_init(bar(bars->a_ready[i]), 2 * kSetWarps); }
        mbar_init(bar(bars->y_full[0]), 1); mbar_init(bar(bars->y_full[1]), 1); mbar_init(bar(bars->y_empty), 2 * kSetWarps); mbar_init(bar(bars->drain), 1);
        bars->abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&map_x); tma_prefetch_desc(&map_wg); tma_prefetch_desc(&map_wu);
        tma_prefetch_desc(&map_wd); tma_prefetch_desc(&map_y);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&bars->tmem_base), 512);
    let_next_begin();
    wait_for_previous();
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                  // the other CTA's barriers are there too
    tc_fence_after();
    const uint32_t tmem = uniform(bars->tmem_base);
    const int pairs = (int)gridDim.x / (2 * splits), pair0 = (int)blockIdx.x / (2 * splits);
    const int tiles = (p.n_tiles - pair0 + pairs - 1) / pairs, total = tiles * nb;
    auto row_of = [&](int t) { return (pair0 + t * pairs) * 2 * kTileM + (int)rank * kTileM; };
    const uint32_t limit = p.poll_limit;
    const bool has_res = p.R != nullptr && splits == 1;          // through shared memory

    if (warp == 0) {
        // ------------------------------------------------------------------ weights: Wg or Wu, half of Wd's outputs
        if (lane == 0) {
            const CUtensorMap* map = rank == 0 ? &map_wg : &map_wu;
            Turn w;
            int c = 0, b = 0;
            for (; c < total && !*abort_flag; ++c, w.next(kStages)) {
                if (c >= kStages && !mbar_wait_relaxed(bar(bars->w_empty[w.at]), w.odd ^ 1u, limit)) { raise_timeout_pair(bars, p.status, in_cluster); break; }
                const uint32_t dst = base + kOffW + w.at * kStageBytes, full = bar(bars->w_full[w.at]);
                mbar_expect_tx(full, kStageBytes);
                for (int h = 0; h < 2; ++h) tma_load_2d(dst + h * kBlock * 128, map, h * 64, unit_of(b), full);
                tma_load_2d(dst + kGuBytes, &map_wd, unit_of(b), (int)rank * 64, full);
                if (++b == nb) b = 0;
            }
            // leave with no copy still landing in shared memory (these waits keep the default limit)
            for (int i = max(0, c - kStages); i < c; ++i) mbar_wait(bar(bars->w_full[i % kStages]), (uint32_t)(i / kStages) & 1u);
        }
    } else if (warp == 2) {
        // ------------------------------------------------------------------ tells rank 0 what has come
        if (lane == 0) {
            const uint32_t ready0 = cluster_addr(bar(bars->ready[0]), lead);
            Turn x, w;
            bool ok = true;
            for (int c = 0, b = 0; c < total && ok && !*abort_flag; ++c, w.next(kStages)) {
                if (b == 0) {
                    ok = mbar_wait_relaxed(bar(bars->x_full[x.at]), x.odd, limit);
                    x.next(2);
                }
                ok = ok && mbar_wait_relaxed(bar(bars->w_full[w.at]), w.odd, limit);
                if (ok) mbar_arrive_cluster(ready0 + w.at * 8);
                if (++b == nb) b = 0;
            }
            if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
        }
    } else if (warp == 3) {
        // ------------------------------------------------------------------ X, and the residual of the tile before
        if (lane == 0) {
            int armed_x = 0, armed_r = 0;
            bool ok = true;
            for (int t = 0; t <= tiles && ok && !*abort_flag; ++t) {
                if (t < tiles) {
                    ok = t < 2 || mbar_wait_relaxed(bar(bars->x_empty[t & 1]), (uint32_t)(t / 2 - 1) & 1u, limit);
                    if (ok) {
                        mbar_expect_tx(bar(bars->x_full[t & 1]), kTileBytes);
                        load_tile(&map_x, base + (t & 1) * kTileBytes, row_of(t), bar(bars->x_full[t & 1]));
                        armed_x = t + 1;
                    }
                }
                if (ok && t >= 1 && has_res) {                     // its place is free when the rows before have been stored
                    ok = t < 2 || mbar_wait_relaxed(bar(bars->r_empty[t & 1]), (uint32_t)(t / 2 - 1) & 1u, limit);
                    if (ok) {
                        const uint32_t full = bar(bars->r_full[(t - 1) & 1]);
                        mbar_expect_tx(full, kTileBytes);
                        load_tile(&map_r, base + kOffR, row_of(t - 1), full);
                        armed_r = t;
                    }
                }
            }
            if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
            for (int i = max(0, armed_x - 2); i < armed_x; ++i) mbar_wait(bar(bars->x_full[i & 1]), (uint32_t)(i >> 1) & 1u);
            if (armed_r > 0) mbar_wait(bar(bars->r_full[(armed_r - 1) & 1]), (uint32_t)((armed_r - 1) >> 1) & 1u);
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------ rank 0: issues the products
        // The tensor cores hold some sixteen products of a pair in waiting; what this warp does between them is hidden as long
        // as a block's issue takes less than its products, so it waits for as few barriers as can be.
        const uint32_t idesc = idesc_bf16_f32(256, 128), elected = elect_one(), high = desc_high(smem_desc_sw128(0));
        const uint32_t low_x = desc_low(smem_desc_sw128(base)), low_w = desc_low(smem_desc_sw128(base + kOffW));
        Turn x, w1, w2, buf1, buf2;
        int b1 = 0, b2 = 0;                              // blocks within their tiles
        uint32_t y_odd = 1;
        bool ok = true;
        const int ahead = 2;                             // first products run two blocks ahead of second ones
        auto second = [&]() {                            // Y += activations Wd^T of the next block
            if (b2 == 0) {
                ok = await(bars, bar(bars->y_empty), y_odd, limit);
                y_odd ^= 1u;
                if (!ok) return;
            }
            tc_fence_after();
            const uint32_t wd = low_w + ((w2.at * kStageBytes + kGuBytes) >> 4), a = tmem + 128 + buf2.at * 128;
            if (elected) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) mma_pair_ta(tmem, a + ks * 16, wd + ks * 2, high, idesc, (b2 | ks) ? 1u : 0u);
                if (b2 + 1 == nb) mma_commit_pair(bar(bars->y_full[y_odd]), mask);
                mma_commit_pair(bar(bars->w_empty[w2.at]), mask);
            }
            __syncwarp();
            w2.next(kStages); buf2.next(kBufs);
            if (++b2 == nb) b2 = 0;
        };
        for (int c = 0; c < total + ahead && ok; ++c) {
            // both of the barriers in one go where both have completed, as they mostly have
            const bool r1 = mbar_test(bar(bars->ready[w1.at]), w1.odd), r2 = mbar_test(bar(bars->a_ready[buf2.at]), buf2.odd);
            const uint32_t come = __reduce_and_sync(0xffffffffu, (r1 ? 1u : 0u) | (r2 ? 2u : 0u));
            // a tile's first second product waits for the tile before to be read: what can go before it goes before it
            const bool early = c >= ahead && (come & 2u) && b2 != 0;
            if (early) second();
            if (c < total) {
                if (!(come & 1u)) ok = await(bars, bar(bars->ready[w1.at]), w1.odd, limit);
                if (!ok) break;
                tc_fence_after();
                const uint32_t dx = low_x + x.at * (kTileBytes >> 4), dw = low_w + w1.at * (kStageBytes >> 4), to = tmem + 128 + buf1.at * 128;
                if (elected) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        mma_pair(to, dx + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4), high,
                                 dw + (((ks >> 2) * kBlock * 128 + (ks & 3) * 32) >> 4), high, idesc, ks > 0 ? 1u : 0u);
                    mma_commit_pair(bar(bars->acc_full[buf1.at]), mask);
                    if (b1 + 1 == nb) mma_commit_pair(bar(bars->x_empty[x.at]), mask);
                }
                __syncwarp();
                w1.next(kStages); buf1.next(kBufs);
                if (++b1 == nb) { b1 = 0; x.next(2); }
            }
            if (c >= ahead && !early) {
                if (!(come & 2u)) ok = await(bars, bar(bars->a_ready[buf2.at]), buf2.odd, limit);
                if (ok) second();
            }
        }
        if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
        if (elected) mma_commit_pair(bar(bars->drain), mask);  // tensor memory is freed below: every product must be done
        __syncwarp();
        mbar_wait_warp(bar(bars->drain), 0);
    } else if (warp >= kCtrlWarps) {
        // ------------------------------------------------------------------ epilogue
        // Two sets of warps take the blocks in turn, so that one computes while the other waits.  A warp has 32 rows and 32 of
        // a block's 64 columns.  A tile's Y is taken by the set that has the next tile's first block, after that block: its
        // last product has long been done then.
        const int ew = warp - kCtrlWarps, quad = warp & 3, set = ew / kSetWarps, part = (ew >> 2) & 1;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t stage = base + kOffR + part * kHalfBytes + quad * 4096;
        const uint32_t a_ready0 = cluster_addr(bar(bars->a_ready[0]), lead), y_empty0 = cluster_addr(bar(bars->y_empty), lead);
        Turn buf;
        bool ok = true;
        int turn = set;                                              // 0: the next block is this set's
        // Y of tile t, with the residual's rows where there are some, staged in their place
        auto finish = [&](int t) {
            if (!await(bars, bar(bars->y_full[t & 1]), (uint32_t)(t >> 1) & 1u, limit)) return false;
            tc_fence_after();
            uint32_t y[64];
            tmem_ld_32x32(tmem + lanes + (uint32_t)(part * 64), y);
            tmem_ld_32x32(tmem + lanes + (uint32_t)(part * 64 + 32), y + 32);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(y_empty0);
            if (has_res ? !await(bars, bar(bars->r_full[t & 1]), (uint32_t)(t >> 1) & 1u, limit)
                          : t > 0 && !await(bars, bar(bars->r_empty[(t - 1) & 1]), (uint32_t)((t - 1) >> 1) & 1u, limit)) return false;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t r[16] = {};
                if (has_res) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ld_shared_v4(stage + sw128_offset(lane, c * 4 + i), r + 4 * i);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = pack_bf16(__uint_as_float(y[c * 32 + 8 * i + 2 * e]) + __uint_as_float(r[4 * i + e] << 16),
                                         __uint_as_float(y[c * 32 + 8 * i + 2 * e + 1]) + __uint_as_float(r[4 * i + e] & 0xffff0000u));
                    st_shared_v4(stage + sw128_offset(lane, c * 4 + i), o);
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            const int row0 = row_of(t) + quad * 32;
            if (lane == 0 && row0 < p.n) {
                tma_store_2d(&map_y, part * 64, row0, stage);
                bulk_commit();
            }
            return true;
        };
        int owed = -1;                                               // the tile whose rows have not yet left their place
        auto leave = [&]() {
            if (owed >= 0 && lane == 0) {
                bulk_wait_read0();
                mbar_arrive(bar(bars->r_empty[owed & 1]));
            }
            owed = -1;
        };
        for (int t = 0; t < tiles && ok; ++t) {
            leave();
            bool open = t > 0 && turn == 0;                          // the tile before is this set's to finish
            for (int b = 0; b < nb; ++b, buf.next(kBufs), turn ^= 1) {
                if (turn) continue;
                ok = await(bars, bar(bars->acc_full[buf.at]), buf.odd, limit);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = tmem + lanes + (uint32_t)(128 + buf.at * 128 + part * 32);
                uint32_t g[32], u[32];
                tmem_ld_32x32(at, g);
                tmem_ld_32x32(at + 64, u);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t a[kEl / 2];
                    gated<ACT>(g + c * kEl, u + c * kEl, a);
                    const int valid = p.d_ff - unit_of(b) - part * 32 - c * kEl;   // hidden units past the last: zero
                    if (valid < kEl) {
#pragma unroll
                        for (int i = 0; i < kEl / 2; ++i) if (2 * i >= valid) a[i] = 0u;
                    }
                    tmem_st_32x8(at + c * kEl, a);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(a_ready0 + buf.at * 8);
                leave();
                if (open) {
                    open = false;
                    ok = finish(t - 1);
                    if (!ok) break;
                    owed = t - 1;
                }
            }
        }
        leave();
        if (ok && turn == 0 && splits == 1) ok = finish(tiles - 1);
        if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
        if (lane == 0) bulk_wait_all();
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1 && rank == 1) mbar_wait_warp(bar(bars->drain), 0);   // the last arrival that rank 0's products send here
    cluster_sync();                                  // no product reads this CTA's memory any more, no arrival is on its way
    if (splits > 1) {                                // uniform: all CTAs of the cluster go through its barriers
        const int ew = warp - kCtrlWarps, row = row_of(0) + (warp & 3) * 32 + lane;
        const Split s = {splits, split, ew >> 2, warp & 3, lane, tmem, base, rank};
        uint32_t r[16];
        tc_fence_after();
        if (ew >= 0) {
            s.residual(r, row < p.n ? row : -1, p.R, p.ldr);
            s.send();
        }
        __syncwarp();
        cluster_sync();
        if (ew >= 0) s.collect(row < p.n ? row : -1, r, p.out, p.ldo);
        __syncwarp();
        tc_fence_before();
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// ---------------------------------------------------------------------------------------------------
// backward: dX
// ---------------------------------------------------------------------------------------------------
// Pairs of CTAs as in the forward kernel.  Of a block each fetches Wg or Wu (for G|U), its half of the inputs of both (for
// dX) and its half of the hidden units of Wd (for dA).
// Tensor memory: dX in columns 0..127, two buffers of G | U | dA behind it.  dG and dU overwrite dA, 16 values of each in the
// 16 columns of dA they were computed from; G and U are free for the next product once they have been read.
namespace dx {
constexpr int kStages = 4, kBufs = 2, kBufCols = 192;
constexpr int kGuBytes = kBlock * 256, kInBytes = 2 * kBlock * 128, kWdBytes = kTileM * 64;
constexpr int kStageBytes = kGuBytes + kInBytes + kWdBytes;
constexpr int kOffW = 2 * kTileBytes, kOffBars = kOffW + kStages * kStageBytes;
struct Bars {
    uint64_t x_full, x_empty, dy_full, dy_empty, w_full[kStages], w_empty[kStages];
    // rank 0's, both CTAs arrive: a block's weights (and X) have come, dY has, G and U have been read, dG and dU are there, dX
    // has been read
    uint64_t ready[kStages], dy_ready, gu_read[kBufs], a_ready[kBufs], y_empty;
    uint64_t acc_full[kBufs], y_full[2], drain;
    uint32_t tmem_base, abort_flag;
};
constexpr int kSmem = kOffBars + (int)sizeof(Bars) + 1024;
static_assert(kSmem <= kSmemLimit, "shared memory");
}  // namespace dx

template <int ACT>
__global__ void __launch_bounds__(kThreads, 1)
glu_dx_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_dy,
              const __grid_constant__ CUtensorMap map_wg, const __grid_constant__ CUtensorMap map_wu,
              const __grid_constant__ CUtensorMap map_wd, Params p) {
    using namespace dx;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    Bars* bars = reinterpret_cast<Bars*>(smem_raw + (base - smem_u32(smem_raw)) + kOffBars);
    const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t in_cluster = cluster_rank(), rank = in_cluster & 1u, lead = in_cluster & ~1u, mask = 3u << lead;
    const int splits = p.splits, split = (int)(in_cluster >> 1), nb = (p.n_blocks - split + splits - 1) / splits;   // this pair's blocks
    auto unit_of = [&](int b) { return (b * splits + split) * kBlock; };                                           // and their first units
    volatile uint32_t* abort_flag = &bars->abort_flag;
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };

    if (threadIdx.x == 0) {
        mbar_init(bar(bars->x_full), 1); mbar_init(bar(bars->x_empty), 1);
        mbar_init(bar(bars->dy_full), 1); mbar_init(bar(bars->dy_empty), 1); mbar_init(bar(bars->dy_ready), 2);
        for (int i = 0; i < kStages; ++i) { mbar_init(bar(bars->w_full[i]), 1); mbar_init(bar(bars->w_empty[i]), 1); mbar_init(bar(bars->ready[i]), 2); }
        for (int i = 0; i < kBufs; ++i) { mbar_init(bar(bars->acc_full[i]), 1); mbar_init(bar(bars->gu_read[i]), 2 * kSetWarps); mbar_init(bar(bars->a_ready[i]), 2 * kSetWarps); }
        mbar_init(bar(bars->y_full[0]), 1); mbar_init(bar(bars->y_full[1]), 1); mbar_init(bar(bars->y_empty), 2 * kSetWarps); mbar_init(bar(bars->drain), 1);
        bars->abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&map_x); tma_prefetch_desc(&map_dy); tma_prefetch_desc(&map_wg); tma_prefetch_desc(&map_wu);
        tma_prefetch_desc(&map_wd);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&bars->tmem_base), 512);
    wait_for_previous();
    let_next_begin();                                // glu_dw_kernel needs nothing of this one: few rows leave SMs for it
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = uniform(bars->tmem_base);
    const int pairs = (int)gridDim.x / (2 * splits), pair0 = (int)blockIdx.x / (2 * splits);
    const int tiles = (p.n_tiles - pair0 + pairs - 1) / pairs, total = tiles * nb;
    auto row_of = [&](int t) { return (pair0 + t * pairs) * 2 * kTileM + (int)rank * kTileM; };
    const uint32_t limit = p.poll_limit;

    if (warp == 0) {
        // ------------------------------------------------------------------ weights
        if (lane == 0) {
            const CUtensorMap* map = rank == 0 ? &map_wg : &map_wu;
            Turn w;
            int c = 0, b = 0;
            for (; c < total && !*abort_flag; ++c, w.next(kStages)) {
                if (c >= kStages && !mbar_wait_relaxed(bar(bars->w_empty[w.at]), w.odd ^ 1u, limit)) { raise_timeout_pair(bars, p.status, in_cluster); break; }
                const uint32_t dst = base + kOffW + w.at * kStageBytes, full = bar(bars->w_full[w.at]);
                mbar_expect_tx(full, kStageBytes);
                for (int h = 0; h < 2; ++h) tma_load_2d(dst + h * kBlock * 128, map, h * 64, unit_of(b), full);
                tma_load_2d(dst + kGuBytes, &map_wg, (int)rank * 64, unit_of(b), full);
                tma_load_2d(dst + kGuBytes + kBlock * 128, &map_wu, (int)rank * 64, unit_of(b), full);
                tma_load_2d(dst + kGuBytes + kInBytes, &map_wd, unit_of(b) + (int)rank * 32, 0, full);
                if (++b == nb) b = 0;
            }
            for (int i = max(0, c - kStages); i < c; ++i) mbar_wait(bar(bars->w_full[i % kStages]), (uint32_t)(i / kStages) & 1u);
        }
    } else if (warp == 3) {
        // ------------------------------------------------------------------ X and dY
        if (lane == 0) {
            int armed_x = 0, armed_dy = 0;
            bool ok = true;
            for (int t = 0; t < tiles && ok && !*abort_flag; ++t) {
                ok = t == 0 || mbar_wait_relaxed(bar(bars->x_empty), (uint32_t)(t - 1) & 1u, limit);
                if (!ok) break;
                mbar_expect_tx(bar(bars->x_full), kTileBytes);
                load_tile(&map_x, base, row_of(t), bar(bars->x_full));
                armed_x = t + 1;
                ok = t == 0 || mbar_wait_relaxed(bar(bars->dy_empty), (uint32_t)(t - 1) & 1u, limit);
                if (!ok) break;
                mbar_expect_tx(bar(bars->dy_full), kTileBytes);
                load_tile(&map_dy, base + kTileBytes, row_of(t), bar(bars->dy_full));
                armed_dy = t + 1;
                if (t + 1 < tiles) {                                 // the next tile's rows into L2 meanwhile
                    prefetch_tile(&map_x, row_of(t + 1));
                    prefetch_tile(&map_dy, row_of(t + 1));
                }
            }
            if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
            if (armed_x > 0) mbar_wait(bar(bars->x_full), (uint32_t)(armed_x - 1) & 1u);
            if (armed_dy > 0) mbar_wait(bar(bars->dy_full), (uint32_t)(armed_dy - 1) & 1u);
        }
    } else if (warp == 2) {
        // ------------------------------------------------------------------ tells rank 0 what has come
        if (lane == 0) {
            const uint32_t ready0 = cluster_addr(bar(bars->ready[0]), lead), dy_ready0 = cluster_addr(bar(bars->dy_ready), lead);
            Turn w;
            uint32_t x_odd = 0;
            bool ok = true;
            for (int c = 0, b = 0; c < total && ok && !*abort_flag; ++c, w.next(kStages)) {
                if (b == 0) {
                    ok = mbar_wait_relaxed(bar(bars->x_full), x_odd, limit);
                    x_odd ^= 1u;
                }
                ok = ok && mbar_wait_relaxed(bar(bars->w_full[w.at]), w.odd, limit);
                if (ok) mbar_arrive_cluster(ready0 + w.at * 8);
                if (b == 0) {
                    ok = ok && mbar_wait_relaxed(bar(bars->dy_full), x_odd ^ 1u, limit);
                    if (ok) mbar_arrive_cluster(dy_ready0);
                }
                if (++b == nb) b = 0;
            }
            if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------ rank 0: issues the products
        const uint32_t id_gu = idesc_bf16_f32(256, 128), id_da = idesc_bf16_f32(256, 64) | kIdescBMn,
                       id_dx = idesc_bf16_f32(256, 128) | kIdescBMn, elected = elect_one();
        const uint32_t high = desc_high(smem_desc_sw128(0)), high_wd = desc_high(smem_desc_sw64_mn(0));
        const uint32_t low_x = desc_low(smem_desc_sw128(base)), low_dy = low_x + (kTileBytes >> 4), low_gu = desc_low(smem_desc_sw128(base + kOffW)),
                       low_in = desc_low(smem_desc_sw128_mn(base + kOffW + kGuBytes, kHalfBytes)), low_wd = desc_low(smem_desc_sw64_mn(base + kOffW + kGuBytes + kInBytes));
        Turn w1, w2, buf1, buf2;
        int b1 = 0, b2 = 0;
        uint32_t y_odd = 1, dy_odd = 0;
        bool ok = true;
        // Per block: G|U as soon as the epilogue has read the block before the last out of this buffer, then dX's product of that
        // block, then this one's dA in the place of that one's dG and dU.  (With G|U behind dX's product too, a block's
        // products wait for the whole epilogue of the block before the last: 119 us instead of 113 on 208 384 rows.)
        for (int c = 0; c < total + 2 && ok; ++c) {
            const bool r1 = mbar_test(bar(bars->ready[w1.at]), w1.odd) && mbar_test(bar(bars->gu_read[buf1.at]), buf1.odd ^ 1u);
            const bool r2 = mbar_test(bar(bars->a_ready[buf2.at]), buf2.odd);
            const uint32_t come = __reduce_and_sync(0xffffffffu, (r1 ? 1u : 0u) | (r2 ? 2u : 0u));
            const uint32_t w = w1.at * (kStageBytes >> 4), d = tmem + 128 + buf1.at * kBufCols;
            if (c < total) {
                if (!(come & 1u)) ok = await(bars, bar(bars->ready[w1.at]), w1.odd, limit) && await(bars, bar(bars->gu_read[buf1.at]), buf1.odd ^ 1u, limit);
                if (!ok) break;
                tc_fence_after();
                if (elected) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        mma_pair(d, low_x + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4), high,
                                 low_gu + w + (((ks >> 2) * kBlock * 128 + (ks & 3) * 32) >> 4), high, id_gu, ks > 0 ? 1u : 0u);
                    if (b1 + 1 == nb) mma_commit_pair(bar(bars->x_empty), mask);
                }
                __syncwarp();
            }
            if (c >= 2) {
                if (!(come & 2u)) ok = await(bars, bar(bars->a_ready[buf2.at]), buf2.odd, limit);
                if (ok && b2 == 0) { ok = await(bars, bar(bars->y_empty), y_odd, limit); y_odd ^= 1u; }
                if (!ok) break;
                tc_fence_after();
                const uint32_t in = low_in + w2.at * (kStageBytes >> 4), a = tmem + 128 + buf2.at * kBufCols + 128;
                if (elected) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)                   // dX += [dG | dU] [Wg; Wu]: their rows run along K
                        mma_pair_ta(tmem, a + (ks & 3) * 16 + (ks >> 2) * 8, in + ks * (2048 >> 4), high, id_dx, (b2 | ks) ? 1u : 0u);
                    if (b2 + 1 == nb) mma_commit_pair(bar(bars->y_full[y_odd]), mask);
                    mma_commit_pair(bar(bars->w_empty[w2.at]), mask);
                }
                __syncwarp();
                w2.next(kStages); buf2.next(kBufs);
                if (++b2 == nb) b2 = 0;
            }
            if (c < total) {
                if (b1 == 0) {
                    ok = await(bars, bar(bars->dy_ready), dy_odd, limit);
                    dy_odd ^= 1u;
                    if (!ok) break;
                    tc_fence_after();
                }
                if (elected) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)                   // dA = dY Wd: Wd's rows run along K
                        mma_pair(d + 128, low_dy + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4), high,
                                 low_wd + w + ks * (1024 >> 4), high_wd, id_da, ks > 0 ? 1u : 0u);
                    mma_commit_pair(bar(bars->acc_full[buf1.at]), mask);
                    if (b1 + 1 == nb) mma_commit_pair(bar(bars->dy_empty), mask);
                }
                __syncwarp();
                w1.next(kStages); buf1.next(kBufs);
                if (++b1 == nb) b1 = 0;
            }
        }
        if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
        if (elected) mma_commit_pair(bar(bars->drain), mask);
        __syncwarp();
        mbar_wait_warp(bar(bars->drain), 0);
    } else if (warp >= kCtrlWarps) {
        // ------------------------------------------------------------------ epilogue
        // as in the forward kernel: two sets of warps, dX of a tile after the next one's first block
        const int ew = warp - kCtrlWarps, quad = warp & 3, set = ew / kSetWarps, part = (ew >> 2) & 1;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t a_ready0 = cluster_addr(bar(bars->a_ready[0]), lead), gu_read0 = cluster_addr(bar(bars->gu_read[0]), lead),
                       y_empty0 = cluster_addr(bar(bars->y_empty), lead);
        Turn buf;
        bool ok = true;
        int turn = set;
        auto finish = [&](int t) {
            if (!await(bars, bar(bars->y_full[t & 1]), (uint32_t)(t >> 1) & 1u, limit)) return false;
            tc_fence_after();
            uint32_t y[64];
            tmem_ld_32x32(tmem + lanes + (uint32_t)(part * 64), y);
            tmem_ld_32x32(tmem + lanes + (uint32_t)(part * 64 + 32), y + 32);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(y_empty0);
            const int row = row_of(t) + quad * 32 + lane;
            if (row < p.n) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = pack_bf16(__uint_as_float(y[8 * i + 2 * e]), __uint_as_float(y[8 * i + 2 * e + 1]));
                    st_global_v4(p.out + (int64_t)row * p.ldo + part * 64 + i * 8, o);
                }
            }
            __syncwarp();
            return true;
        };
        for (int t = 0; t < tiles && ok; ++t) {
            bool open = t > 0 && turn == 0;
            for (int b = 0; b < nb; ++b, buf.next(kBufs), turn ^= 1) {
                if (turn) continue;
                ok = await(bars, bar(bars->acc_full[buf.at]), buf.odd, limit);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t at = tmem + lanes + (uint32_t)(128 + buf.at * kBufCols + part * 32 + c * kEl);
                    uint32_t g[kEl], u[kEl], h[kEl], dg[kEl / 2], du[kEl / 2];
                    tmem_ld_32x16(at, g);
                    tmem_ld_32x16(at + 64, u);
                    tmem_ld_32x16(at + 128, h);
                    tmem_ld_wait();
                    if (c == 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(gu_read0 + buf.at * 8);
                    }
                    gated_bwd<ACT, false>(g, u, h, dg, du, nullptr);
                    const int valid = p.d_ff - unit_of(b) - part * 32 - c * kEl;
                    if (valid < kEl) {
#pragma unroll
                        for (int i = 0; i < kEl / 2; ++i) if (2 * i >= valid) dg[i] = du[i] = 0u;
                    }
                    tmem_st_32x8(at + 128, dg);
                    tmem_st_32x8(at + 136, du);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(a_ready0 + buf.at * 8);
                if (open) {
                    open = false;
                    ok = finish(t - 1);
                    if (!ok) break;
                }
            }
        }
        if (ok && turn == 0 && splits == 1) ok = finish(tiles - 1);
        if (!ok) raise_timeout_pair(bars, p.status, in_cluster);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1 && rank == 1) mbar_wait_warp(bar(bars->drain), 0);
    cluster_sync();
    if (splits > 1) {                                // uniform: all CTAs of the cluster go through its barriers
        const int ew = warp - kCtrlWarps, row = row_of(0) + (warp & 3) * 32 + lane;
        const Split s = {splits, split, ew >> 2, warp & 3, lane, tmem, base, rank};
        uint32_t r[16];
        tc_fence_after();
        if (ew >= 0) {
            s.residual(r, row < p.n ? row : -1, nullptr, 0);
            s.send();
        }
        __syncwarp();
        cluster_sync();
        if (ew >= 0) s.collect(row < p.n ? row : -1, r, p.out, p.ldo);
        __syncwarp();
        tc_fence_before();
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// ---------------------------------------------------------------------------------------------------
// backward: the weights
// ---------------------------------------------------------------------------------------------------
// Tensor memory: [dWg | dWu]^T in columns 0..127 (lane = input, column = hidden unit of the block), dWd in 128..191 (lane =
// output, column = hidden unit), G | U | dA in 192..383.  The epilogue takes its 96 values into registers at once, and the
// next tile's first products run while it computes.
// Shared memory: the block's weights, two stages of X and dY, and the bf16 values dG | dU | act(G) U as MN-major operands.
namespace dw {
constexpr int kStages = 2;
constexpr int kOffX = kTileBytes + kHalfBytes, kOffA = kOffX + kStages * 2 * kTileBytes, kOffBars = kOffA + 3 * kHalfBytes;
constexpr int kPart = 3 * kBlock * 128;            // fp32 values of a CTA's accumulators: dWg, dWu, dWd^T, [unit][128] each
struct Bars {
    uint64_t w_full, x_full[kStages], x_empty[kStages], dy_full[kStages], dy_empty[kStages];
    uint64_t acc_full, acc_empty, a_full, a_empty, w_done;
    uint64_t drain;
    uint32_t tmem_base, abort_flag;
};
constexpr int kSmem = kOffBars + (int)sizeof(Bars) + 1024;
static_assert(kSmem <= kSmemLimit, "shared memory");
}  // namespace dw

struct DwOut {
    int32_t beside_dx;                             // the kernel before is dX's, which has waited for what came before it
    float* part;                                   // [groups][blocks][kPart], or null: one group, straight to bf16
    __nv_bfloat16 *wg, *wu, *wd;
};

template <int ACT>
__global__ void __launch_bounds__(kThreads, 1)
glu_dw_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_dy,
              const __grid_constant__ CUtensorMap map_wg, const __grid_constant__ CUtensorMap map_wu,
              const __grid_constant__ CUtensorMap map_wd, Params p, DwOut out) {
    using namespace dw;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    Bars* bars = reinterpret_cast<Bars*>(smem_raw + (base - smem_u32(smem_raw)) + kOffBars);
    const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int block = blockIdx.x, group = blockIdx.y, groups = gridDim.y;
    volatile uint32_t* abort_flag = &bars->abort_flag;
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };

    if (threadIdx.x == 0) {
        mbar_init(bar(bars->w_full), 1);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(bar(bars->x_full[i]), 1); mbar_init(bar(bars->x_empty[i]), 1);
            mbar_init(bar(bars->dy_full[i]), 1); mbar_init(bar(bars->dy_empty[i]), 1);
        }
        mbar_init(bar(bars->acc_full), 1); mbar_init(bar(bars->acc_empty), kEpiWarps);
        mbar_init(bar(bars->a_full), kEpiWarps); mbar_init(bar(bars->a_empty), 1);
        mbar_init(bar(bars->w_done), 1); mbar_init(bar(bars->drain), 1);
        bars->abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&map_x); tma_prefetch_desc(&map_dy);
    }
    if (warp == 1) tmem_alloc(smem_u32(&bars->tmem_base), 512);
    if (!out.beside_dx) wait_for_previous();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(bars->tmem_base);
    const int tiles = (p.n_tiles - group + groups - 1) / groups;     // at least one: groups <= n_tiles
    const uint32_t limit = p.poll_limit;

    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------------ X (with the block's weights), dY
        if (lane == 0) {
            const bool dy = warp == 2;
            const CUtensorMap* map = dy ? &map_dy : &map_x;
            uint64_t *full = dy ? bars->dy_full : bars->x_full, *empty = dy ? bars->dy_empty : bars->x_empty;
            if (!dy) {
                mbar_expect_tx(bar(bars->w_full), kTileBytes + kHalfBytes);
                load_gu(&map_wg, &map_wu, base, block, bar(bars->w_full));
                tma_load_2d(base + kTileBytes, &map_wd, block * kBlock, 0, bar(bars->w_full));
            }
            Turn x;
            int t = 0;
            for (; t < tiles && !*abort_flag; ++t, x.next(kStages)) {
                if (t >= kStages && !mbar_wait(bar(empty[x.at]), x.odd ^ 1u, limit)) { raise_timeout(bars, p.status); break; }
                const int row0 = (group + t * groups) * kTileM;
                mbar_expect_tx(bar(full[x.at]), kTileBytes);
                load_tile(map, base + kOffX + (2 * x.at + (dy ? 1 : 0)) * kTileBytes, row0, bar(full[x.at]));
                // the rows of two tiles on into L2: every block's CTA of the group wants them, one asks
                if (t + 2 < tiles && t % (int)gridDim.x == block) prefetch_tile(map, row0 + 2 * groups * kTileM);
            }
            if (!dy) mbar_wait(bar(bars->w_full), 0);
            for (int i = max(0, t - kStages); i < t; ++i) mbar_wait(bar(full[i % kStages]), (uint32_t)(i / kStages) & 1u);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        const uint32_t id_gu = idesc_bf16_f32(128, 128), id_da = idesc_bf16_f32(128, 64) | kIdescBMn,
                       id_w = idesc_bf16_f32(128, 128) | kIdescAMn | kIdescBMn, id_wd = idesc_bf16_f32(128, 64) | kIdescAMn | kIdescBMn,
                       elected = elect_one();
        const uint64_t desc_gu = smem_desc_sw128(base), desc_wd = smem_desc_sw128_mn(base + kTileBytes, kHalfBytes),
                       desc_a = smem_desc_sw128_mn(base + kOffA, kHalfBytes);
        Turn x1, x2;
        uint32_t acc_odd = 1, a_odd = 0, polls = 0;
        bool ok = mbar_wait_relaxed_warp(bar(bars->w_full), 0, limit);
        // Whichever can go first: the next tile's first products (its rows have come, the epilogue has taken its values) or
        // this tile's second ones.  With a fixed order the tensor cores would wait for rows that can only come when second
        // products have left a stage.  X leaves its place before dY, and G|U begins before dY has come.
        bool half = false;                                           // G|U of tile t1 has been issued, dA not yet
        for (int t1 = 0, t2 = 0; t2 < tiles && ok;) {
            if (t2 < t1 && has_come(bar(bars->a_full), a_odd)) {
                a_odd ^= 1u;
                tc_fence_after();
                const uint64_t x = smem_desc_sw128_mn(base + kOffX + x2.at * 2 * kTileBytes, kHalfBytes), dy = x + (kTileBytes >> 4);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)                       // sixteen rows at a time
                    mma_bf16_by(elected, tmem, x + ks * kStepMn, desc_a + ks * kStepMn, id_w, t2 > 0 || ks > 0 ? 1u : 0u);
                mma_commit_by(elected, bar(bars->x_empty[x2.at]));
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    mma_bf16_by(elected, tmem + 128, dy + ks * kStepMn, desc_a + (2 * kHalfBytes >> 4) + ks * kStepMn, id_wd, t2 > 0 || ks > 0 ? 1u : 0u);
                mma_commit_by(elected, bar(bars->dy_empty[x2.at]));
                mma_commit_by(elected, bar(bars->a_empty));
                x2.next(kStages);
                ++t2;
                polls = 0;
            } else if (!half && t1 < tiles && has_come(bar(bars->x_full[x1.at]), x1.odd) && has_come(bar(bars->acc_empty), acc_odd)) {
                acc_odd ^= 1u;
                tc_fence_after();
                const uint64_t x = smem_desc_sw128(base + kOffX + x1.at * 2 * kTileBytes);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const uint64_t off = (uint64_t)(((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4);
                    mma_bf16_by(elected, tmem + 192, x + off, desc_gu + off, id_gu, ks > 0 ? 1u : 0u);
                }
                half = true;
                polls = 0;
            } else if (half && has_come(bar(bars->dy_full[x1.at]), x1.odd)) {
                tc_fence_after();
                const uint64_t dy = smem_desc_sw128(base + kOffX + (x1.at * 2 + 1) * kTileBytes);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    mma_bf16_by(elected, tmem + 320, dy + (uint64_t)(((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4), desc_wd + ks * kStepMn, id_da, ks > 0 ? 1u : 0u);
                mma_commit_by(elected, bar(bars->acc_full));
                half = false;
                x1.next(kStages);
                ++t1;
                polls = 0;
            } else {
                ok = !__any_sync(0xffffffffu, *abort_flag != 0) && ++polls <= limit;
                if (polls > 64) __nanosleep(40);
            }
        }
        if (ok) mma_commit_by(elected, bar(bars->w_done));
        else raise_timeout(bars, p.status);
        mma_commit_by(elected, bar(bars->drain));
        mbar_wait_warp(bar(bars->drain), 0);
    } else if (warp >= kCtrlWarps) {
        // ------------------------------------------------------------------ epilogue
        const int quad = warp & 3, part = (warp - kCtrlWarps) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const int valid = p.d_ff - block * kBlock - part * kEl;      // hidden units of this warp's 16 that exist
        uint32_t odd = 0;
        bool ok = true;
        for (int t = 0; t < tiles && ok; ++t, odd ^= 1u) {
            const bool in = (group + t * groups) * kTileM + quad * 32 + lane < p.n;
            ok = await(bars, bar(bars->acc_full), odd, limit);
            if (!ok) break;
            tc_fence_after();
            const uint32_t at = tmem + lanes + (uint32_t)(192 + part * kEl);
            uint32_t g[kEl], u[kEl], h[kEl], v[3][kEl / 2];
            tmem_ld_32x16(at, g);
            tmem_ld_32x16(at + 64, u);
            tmem_ld_32x16(at + 128, h);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(bars->acc_empty));
            gated_bwd<ACT, true>(g, u, h, v[0], v[1], v[2]);
            // a row past the last (its X and dY read as zero) and a unit past the last add nothing, whatever the weights
            // hold: 0 * infinity would
            if (!in || valid < kEl) {
#pragma unroll
                for (int i = 0; i < kEl / 2; ++i) if (!in || 2 * i >= valid) v[0][i] = v[1][i] = v[2][i] = 0u;
            }
            ok = await(bars, bar(bars->a_empty), odd ^ 1u, limit);
            if (!ok) break;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t off = base + kOffA + sw128_offset(quad * 32 + lane, part * 2 + c);
#pragma unroll
                for (int m = 0; m < 3; ++m) st_shared_v4(off + m * kHalfBytes, v[m] + 4 * c);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(bars->a_full));
        }
        ok = ok && mbar_wait_relaxed_warp(bar(bars->w_done), 0, limit);
        let_next_begin();                            // glu_reduce_kernel, which waits
        if (ok) {
            tc_fence_after();
            const int col = quad * 32 + lane;                        // an input (dWg, dWu) or an output (dWd)
            float* sums = out.part ? out.part + ((int64_t)group * gridDim.x + block) * kPart : nullptr;
#pragma unroll 1
            for (int m = 0; m < 3; ++m) {
                uint32_t w[kEl];
                tmem_ld_32x16(tmem + lanes + (uint32_t)(m * 64 + part * kEl), w);
                tmem_ld_wait();
                if (sums) {
#pragma unroll
                    for (int i = 0; i < kEl; ++i) sums[(m * kBlock + part * kEl + i) * 128 + col] = __uint_as_float(w[i]);
                } else if (m < 2) {
                    __nv_bfloat16* to = (m == 0 ? out.wg : out.wu) + (int64_t)(block * kBlock + part * kEl) * 128 + col;
#pragma unroll
                    for (int i = 0; i < kEl; ++i) if (i < valid) to[i * 128] = __float2bfloat16(__uint_as_float(w[i]));
                } else {                                             // d_ff is a multiple of 8, and so are the units that exist
#pragma unroll
                    for (int i = 0; i < kEl; i += 8) {
                        uint32_t o[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = pack_bf16(__uint_as_float(w[i + 2 * e]), __uint_as_float(w[i + 2 * e + 1]));
                        if (i < valid) st_global_v4(out.wd + (int64_t)col * p.d_ff + block * kBlock + part * kEl + i, o);
                    }
                }
            }
            tc_fence_before();
        } else {
            raise_timeout(bars, p.status);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0) wait_for_previous();       // glu_dx_kernel ends before this one does
}

// One CTA per hidden unit and matrix, one thread per input or output: the groups' sums in the order of the groups.
__global__ void glu_reduce_kernel(DwOut out, int d_ff, int n_blocks, int groups) {
    const int unit = blockIdx.x, m = blockIdx.y, col = threadIdx.x;
    let_next_begin();
    wait_for_previous();
    const float* src = out.part + (int64_t)(unit / kBlock) * dw::kPart + (m * kBlock + unit % kBlock) * 128 + col;
    float f = 0.f;
    for (int g = 0; g < groups; ++g) f += src[(int64_t)g * n_blocks * dw::kPart];
    if (m == 2) out.wd[(int64_t)col * d_ff + unit] = __float2bfloat16(f);
    else (m == 0 ? out.wg : out.wu)[(int64_t)unit * 128 + col] = __float2bfloat16(f);
}

// ---------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------
#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

dg4_status sm_count(int dev, int* out) {
    static std::atomic<int> known[64];
    if (dev < 0 || dev >= 64) DG4_FAIL(DG4_ERR_UNSUPPORTED, "device ordinal %d is out of range", dev);
    int sms = known[dev].load(std::memory_order_relaxed);
    if (sms == 0) {
        DG4_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        known[dev].store(sms, std::memory_order_relaxed);
    }
    *out = sms;
    return DG4_OK;
}

// the opt-in to more than 48 KB of shared memory, once per kernel and device
template <auto kKernel>
dg4_status allow_smem(int dev, int bytes) {
    static std::atomic<bool> done[64];
    if (dev < 0 || dev >= 64) DG4_FAIL(DG4_ERR_UNSUPPORTED, "device ordinal %d is out of range", dev);
    if (!done[dev].load(std::memory_order_relaxed)) {
        DG4_CUDA_TRY(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        done[dev].store(true, std::memory_order_relaxed);
    }
    return DG4_OK;
}

struct Maps { CUtensorMap x, dy, wg, wu, wd, r, y, wd_half; };

int blocks_of(int d_ff) { return (d_ff + kBlock - 1) / kBlock; }
// Row groups of glu_dw_kernel: as many as the device has SMs for, as many again where a group would have more than kMaxTiles
// tiles, and no more than there are tiles.  The tensor cores cut their sums off instead of rounding them, on sums of one sign
// by 0.74 to 0.82 * 2^-23 per 16 rows (measured; 1.2e-2 on 2 million rows at once), so a group has up to 131 072 rows: 2^-23 for each
// of their 8 192 additions is a quarter of what rounding to bf16 may cost, 2^-8.
constexpr int kMaxTiles = 1024;
int groups_of(const dg4_graph* g, int d_ff, int sms) {
    const int64_t tiles = ((int64_t)g->n + kTileM - 1) / kTileM, blocks = blocks_of(d_ff), most = sms > blocks ? sms / blocks : 1;
    return (int)(tiles < most ? tiles : most * ((tiles + most * kMaxTiles - 1) / (most * kMaxTiles)));
}

dg4_status check_weights(const void* wg, const void* wu, const void* wd, int32_t d_ff, int32_t act) {
    if (act != DG4_ACT_SILU && act != DG4_ACT_GELU && act != DG4_ACT_RELU) DG4_FAIL(DG4_ERR_UNSUPPORTED, "unknown activation %d", act);
    if (d_ff < 8 || d_ff > kMaxDff || d_ff % 8 != 0) DG4_FAIL(DG4_ERR_UNSUPPORTED, "d_ff = %d: must be a multiple of 8 up to %d", d_ff, kMaxDff);
    CHECK(dg4i_check_tensor("W_gate", wg, 128, 2, 128));
    CHECK(dg4i_check_tensor("W_up", wu, 128, 2, 128));
    CHECK(dg4i_check_tensor("W_down", wd, d_ff, 2, d_ff));
    return DG4_OK;
}

dg4_status weight_maps(Maps* m, const void* wg, const void* wu, const void* wd, int d_ff, int wd_rows) {
    CHECK(dg4i_make_row_map(&m->wg, wg, d_ff, 128, kBlock));
    CHECK(dg4i_make_row_map(&m->wu, wu, d_ff, 128, kBlock));
    CHECK(dg4i_make_map(&m->wd, wd, d_ff, 128, d_ff, wd_rows, 64));
    return DG4_OK;
}

// Pairs of CTAs that share a tile's blocks, for a kernel that works in pairs on tiles of 256 rows: two from `least` blocks on,
// four from twice as many, where the device holds that many at once on `sms` SMs.  A block costs one pair 0.58 us forward and
// 0.83 for dX; joining two pairs' sums costs 3.2 us, four pairs' 6.5 (most of it the launch of the larger cluster).  One row by
// one, two and four pairs, us: forward 9.2, 10.1, 11.4 for 8 blocks, 13.7, 12.5, 12.9 for 16, 22.9, 17.1, 15.2 for 32, 41.3, 26.4,
// 19.8 for 64; dX 11.0, 11.4, 12.0, then 17.6, 15.0, 14.2, then 31.0, 21.6, 17.5, then 57.7, 35.0, 24.2.
constexpr int kSplitFwd = 12, kSplitDx = 8;
template <auto kKernel>
dg4_status splits_of(int tiles, int n_blocks, int least, int smem, int sms, int* out) {
    *out = 1;
    for (int s = 4; s > 1; s /= 2) {
        int clusters;
        if (n_blocks < least * (s / 2) || (int64_t)tiles * 2 * s > sms) continue;
        CHECK(dg4i_resident_clusters<kKernel>(2 * s, kThreads, smem, &clusters));
        if (tiles <= clusters) {
            *out = s;
            break;
        }
    }
    return DG4_OK;
}
// `p` with n_tiles counting tiles of 256 rows
template <auto kKernel, class... Args>
dg4_status launch_pairs(Params p, int least, int smem, int sms, int free_sms, cudaStream_t st, const Args&... maps) {
    p.n_tiles = (p.n_tiles + 1) / 2;
    CHECK(splits_of<kKernel>(p.n_tiles, p.n_blocks, least, smem, free_sms, &p.splits));
    const int pairs = p.splits > 1 || p.n_tiles < sms / 2 ? p.n_tiles : sms / 2;
    return dg4i_launch_clusters(kKernel, dim3(2 * p.splits * pairs), 2 * p.splits, kThreads, smem, st, true, maps..., p);
}

template <int ACT>
dg4_status launch_fwd(const Maps& m, const Params& p, int dev, int sms, cudaStream_t st) {
    CHECK(allow_smem<glu_fwd_kernel<ACT>>(dev, fwd::kSmem));
    return launch_pairs<glu_fwd_kernel<ACT>>(p, kSplitFwd, fwd::kSmem, sms, sms, st, m.x, m.wg, m.wu, m.wd, m.r, m.y);
}

template <int ACT>
dg4_status launch_bwd(const Maps& m, const Params& p, const DwOut& out, int groups, int dev, int sms, cudaStream_t st) {
    if (p.out) {
        CHECK(allow_smem<glu_dx_kernel<ACT>>(dev, dx::kSmem));
        // The weights' kernel begins beside this one: where a pair to each tile fits on what it leaves, the tiles' blocks are
        // shared among no more pairs than fit there, and elsewhere it has to wait for SMs anyway.  Whether the weights'
        // gradients are asked for does not enter, or dX would be summed in another order without them.  Gradients of all
        // (and dX alone), us: (2000 rows, d_ff 512) 17.9 (12.6), where shared blocks would take 21.2 (11.9); (1500, 1024)
        // 25.9 (14.6), without shared blocks 30.3 (19.3).
        const int left = sms - p.n_blocks * groups, free_sms = (p.n_tiles + 1) / 2 * 2 <= left ? left : sms;
        CHECK(launch_pairs<glu_dx_kernel<ACT>>(p, kSplitDx, dx::kSmem, sms, free_sms, st, m.x, m.dy, m.wg, m.wu, m.wd_half));
    }
    if (out.wg) {
        CHECK(allow_smem<glu_dw_kernel<ACT>>(dev, dw::kSmem));
        CHECK(dg4i_launch(glu_dw_kernel<ACT>, dim3(p.n_blocks, groups), kThreads, dw::kSmem, st, true, m.x, m.dy, m.wg, m.wu, m.wd, p, out));
        if (out.part) CHECK(dg4i_launch(glu_reduce_kernel, dim3(p.d_ff, 3), 128, 0, st, true, out, p.d_ff, p.n_blocks, groups));
    }
    return DG4_OK;
}

Params make_params(const dg4_graph* g, int d_ff) {
    Params p = {};
    p.n = g->n; p.d_ff = d_ff; p.n_blocks = blocks_of(d_ff);
    p.n_tiles = (int)(((int64_t)g->n + kTileM - 1) / kTileM);
    p.status = g->dev_status; p.poll_limit = dg4i_poll_limit();
    return p;
}

}  // namespace

extern "C" dg4_status dg4_glu_fwd(const dg4_graph* g, const dg4_desc* desc, const void* X, int64_t ldx, const void* W_gate,
                                  const void* W_up, const void* W_down, int32_t d_ff, int32_t activation, const void* H_res,
                                  int64_t ldh, void* Y, int64_t ldy, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, true));
    CHECK(dg4i_check_tensor("X", X, ldx, 2, 128));
    CHECK(check_weights(W_gate, W_up, W_down, d_ff, activation));
    const bool res = (desc->flags & DG4_FLAG_RESIDUAL) && H_res;
    if (res) CHECK(dg4i_check_tensor("H_res", H_res, ldh, 2, 128));
    CHECK(dg4i_check_tensor("Y", Y, ldy, 2, 128));
    if ((Y == X && ldy != ldx) || (res && Y == H_res && ldy != ldh))
        DG4_FAIL(DG4_ERR_INVALID_ARG, "Y in the place of X or H_res has another leading dimension");
    int sms;
    CHECK(sm_count(g->device, &sms));
    Maps m;
    CHECK(weight_maps(&m, W_gate, W_up, W_down, d_ff, 64));
    CHECK(dg4i_make_row_map(&m.x, X, g->n, ldx, kTileM));
    CHECK(dg4i_make_row_map(&m.y, Y, g->n, ldy, 32));
    Params p = make_params(g, d_ff);
    p.R = res ? (const __nv_bfloat16*)H_res : nullptr; p.ldr = ldh;
    p.out = (__nv_bfloat16*)Y; p.ldo = ldy;
    m.r = m.x;
    if (res) CHECK(dg4i_make_row_map(&m.r, H_res, g->n, ldh, kTileM));
    const cudaStream_t st = (cudaStream_t)stream;
    if (activation == DG4_ACT_SILU) return launch_fwd<DG4_ACT_SILU>(m, p, g->device, sms, st);
    if (activation == DG4_ACT_GELU) return launch_fwd<DG4_ACT_GELU>(m, p, g->device, sms, st);
    return launch_fwd<DG4_ACT_RELU>(m, p, g->device, sms, st);
}

extern "C" size_t dg4_glu_bwd_workspace_bytes(const dg4_graph* g, const dg4_desc* desc, int32_t d_ff) {
    int sms;
    if (!g || dg4i_check_desc(desc, true) != DG4_OK || d_ff < 8 || d_ff > kMaxDff || sm_count(g->device, &sms) != DG4_OK) return 0;
    const int groups = groups_of(g, d_ff, sms);
    return groups > 1 ? (size_t)groups * blocks_of(d_ff) * dw::kPart * sizeof(float) : 0;
}

extern "C" dg4_status dg4_glu_bwd(const dg4_graph* g, const dg4_desc* desc, const void* X, int64_t ldx, const void* W_gate,
                                  const void* W_up, const void* W_down, int32_t d_ff, int32_t activation, const void* dY,
                                  int64_t lddy, void* dX, int64_t lddx, void* dW_gate, void* dW_up, void* dW_down,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, true));
    CHECK(dg4i_check_tensor("X", X, ldx, 2, 128));
    CHECK(check_weights(W_gate, W_up, W_down, d_ff, activation));
    CHECK(dg4i_check_tensor("dY", dY, lddy, 2, 128));
    if (dX) CHECK(dg4i_check_tensor("dX", dX, lddx, 2, 128));
    if (dX && ((dX == X && lddx != ldx) || (dX == dY && lddx != lddy)))
        DG4_FAIL(DG4_ERR_INVALID_ARG, "dX in the place of X or dY has another leading dimension");
    const bool weights = dW_gate || dW_up || dW_down;
    if (!dX && !weights) DG4_FAIL(DG4_ERR_INVALID_ARG, "neither dX nor the weights' gradients are asked for");
    int sms;
    CHECK(sm_count(g->device, &sms));
    DwOut out = {};
    out.beside_dx = dX != nullptr;
    const int groups = groups_of(g, d_ff, sms);
    if (weights) {
        CHECK(dg4i_check_tensor("dW_gate", dW_gate, 128, 2, 128));
        CHECK(dg4i_check_tensor("dW_up", dW_up, 128, 2, 128));
        CHECK(dg4i_check_tensor("dW_down", dW_down, d_ff, 2, d_ff));
        // the kernels of dX and of the weights run side by side, and each reads everything
        if (dX && (dX == X || dX == dY)) DG4_FAIL(DG4_ERR_INVALID_ARG, "dX must not be X or dY when the weights' gradients are asked for");
        const void *in[3] = {W_gate, W_up, W_down}, *made[3] = {dW_gate, dW_up, dW_down};
        for (int i = 0; i < 3; ++i)
            for (int j = 0; j < 3; ++j)
                if (made[i] == in[j] || (i < j && made[i] == made[j])) DG4_FAIL(DG4_ERR_INVALID_ARG, "a weight's gradient lies over a weight or another gradient");
        const size_t need = dg4_glu_bwd_workspace_bytes(g, desc, d_ff);
        if (need && (!workspace || workspace_bytes < need))
            DG4_FAIL(DG4_ERR_INVALID_ARG, "workspace too small: %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
        if (need && ((uintptr_t)workspace & 15u)) DG4_FAIL(DG4_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
        out.part = need ? (float*)workspace : nullptr;
        out.wg = (__nv_bfloat16*)dW_gate; out.wu = (__nv_bfloat16*)dW_up; out.wd = (__nv_bfloat16*)dW_down;
    }
    Maps m;
    CHECK(weight_maps(&m, W_gate, W_up, W_down, d_ff, 128));
    CHECK(dg4i_make_map(&m.wd_half, W_down, d_ff, 128, d_ff, 128, 32));
    CHECK(dg4i_make_row_map(&m.x, X, g->n, ldx, kTileM));
    CHECK(dg4i_make_row_map(&m.dy, dY, g->n, lddy, kTileM));
    Params p = make_params(g, d_ff);
    p.out = (__nv_bfloat16*)dX; p.ldo = lddx;
    const cudaStream_t st = (cudaStream_t)stream;
    if (activation == DG4_ACT_SILU) return launch_bwd<DG4_ACT_SILU>(m, p, out, groups, g->device, sms, st);
    if (activation == DG4_ACT_GELU) return launch_bwd<DG4_ACT_GELU>(m, p, out, groups, g->device, sms, st);
    return launch_bwd<DG4_ACT_RELU>(m, p, out, groups, g->device, sms, st);
}
