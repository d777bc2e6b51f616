// The norm of a residual sum, forward and backward:
//     Z = X + R,   xh = (Z - mean) * inv,   Y = xh * gamma + beta,      inv = 1 / sqrt(var + eps)
//     t = dY * gamma,   dZ = D_res + inv * (t - mean(t) - xh * mean(t * xh)),   dgamma = sum dY * xh,   dbeta = sum dY
// (root mean square: nothing is taken off, so mean and mean(t) are zero).  Rows of 128 elements as in dg4_norm_core.cuh;
// between a row's loads and its stores everything stays in registers in 32 bits, so both passes are bound by memory:
// a bf16 row costs 256 bytes per tensor.
//
// Backward the mean and variance are taken from Z again: six shuffles per four rows, where saved ones would cost 8 bytes
// per row in each pass and an argument.  A lane adds up the contributions of its 16 columns over all rows its warp walks;
// the four rows of a warp, the warps of a CTA (through shared memory) and the CTAs (norm_reduce_kernel) are added in a
// fixed order, so the sums do not depend on which warp came first.

#include "dg4_launch.cuh"
#include "dg4_norm_core.cuh"

using namespace normcore;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kFewRows = 32;               // up to here one CTA takes all rows at once and the sums need no second kernel
                                           // (128 rows: 5.2 us so, 4.9 us by two kernels)

struct FwdArgs {
    const void* X; int64_t ldx;            // bytes
    const void* R; int64_t ldr;            // R nullable
    void* Z; int64_t ldz;                  // Z nullable
    void* Y; int64_t ldy;
    const float *gamma, *beta;             // beta nullable (zero)
    int32_t n;
    float eps;
};

struct BwdArgs {
    const void* Z; int64_t ldz;            // bytes
    const void* dY; int64_t lddy;
    const void* D; int64_t ldd;            // nullable
    void* dZ; int64_t lddz;                // nullable
    const float* gamma;
    float *dgamma, *dbeta;                 // each nullable
    float* part;                           // [CTAs][2][128], or null: one CTA, straight to dgamma and dbeta
    int32_t n, sums;
    float eps;
};

// the vectors in the order the lanes read them: place i * 8 + sub holds quad_of(i, sub)
template <bool BF16>
__device__ __forceinline__ void stage_vec(float4* to, const float* v, float fill, int t) {
    to[t] = v ? reinterpret_cast<const float4*>(v)[quad_of<BF16>(t / kLanes, t & (kLanes - 1))] : make_float4(fill, fill, fill, fill);
}

template <bool BF16, bool RMS>
__global__ void __launch_bounds__(kThreads, 2) add_norm_kernel(FwdArgs a) {
    __shared__ float4 vec[2][32];
    const int lane = threadIdx.x & 31, sub = lane & (kLanes - 1), grp = lane / kLanes;
    let_next_begin();
    wait_for_previous();
    if (threadIdx.x < 64) stage_vec<BF16>(vec[threadIdx.x >> 5], threadIdx.x < 32 ? a.gamma : a.beta, 0.f, threadIdx.x & 31);
    __syncthreads();
    const uint32_t n = (uint32_t)a.n, step = gridDim.x * kWarps * kRows;
    uint32_t row = (blockIdx.x * kWarps + (threadIdx.x >> 5)) * kRows + grp;
    Raw<BF16> x_next, r_next;
    auto fetch = [&](uint32_t at) {
        if (at < n) {
            x_next.load((const char*)a.X + (int64_t)at * a.ldx, sub);
            if (a.R) r_next.load((const char*)a.R + (int64_t)at * a.ldr, sub);
        }
    };
    fetch(row);
    for (; row - grp < n; row += step) {                             // the whole warp
        Pair x[kPairs];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[i] = x_next.get(i);
        if (a.R) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[i] = add2(x[i], r_next.get(i));
        }
        fetch(row + step);
        if (a.Z && row < n) Raw<BF16>::store((char*)a.Z + (int64_t)row * a.ldz, sub, x);
        norm_row<RMS>(x, &vec[0][sub], &vec[1][sub], a.eps);
        if (row < n) Raw<BF16>::store((char*)a.Y + (int64_t)row * a.ldy, sub, x);
    }
}

template <bool BF16, bool RMS>
__global__ void __launch_bounds__(kThreads, 2) norm_bwd_kernel(BwdArgs a) {
    __shared__ float4 vec[32];
    __shared__ float4 sum[kWarps][2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane & (kLanes - 1), grp = lane / kLanes;
    let_next_begin();
    wait_for_previous();
    if (threadIdx.x < 32) stage_vec<BF16>(vec, a.gamma, 1.f, threadIdx.x);
    __syncthreads();
    const uint32_t n = (uint32_t)a.n, step = gridDim.x * kWarps * kRows;
    uint32_t row = (blockIdx.x * kWarps + warp) * kRows + grp;
    Raw<BF16> z_next, y_next;
    auto fetch = [&](uint32_t at) {
        if (at < n) {
            z_next.load((const char*)a.Z + (int64_t)at * a.ldz, sub);
            y_next.load((const char*)a.dY + (int64_t)at * a.lddy, sub);
        }
    };
    fetch(row);
    Pair dg[kPairs], db[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) dg[i] = db[i] = pair(0.f, 0.f);
    for (; row - grp < n; row += step) {                             // the whole warp
        Pair x[kPairs], t[kPairs];
        Raw<BF16> d;
        const bool in = row < n;
        if (a.D && in) d.load((const char*)a.D + (int64_t)row * a.ldd, sub);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) { x[i] = z_next.get(i); t[i] = y_next.get(i); }
        fetch(row + step);
        if (!RMS) {
            const float mean = row_sum(x) * (1.f / 128.f);
            const Pair m = pair(-mean, -mean);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[i] = add2(x[i], m);
        }
        Pair q[kPairs];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) q[i] = mul2(x[i], x[i]);
        const float inv = rsqrtf(row_sum(q) * (1.f / 128.f) + a.eps);
        const Pair s = pair(inv, inv);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[i] = mul2(x[i], s);
        if (in) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) { dg[i] = fma2(t[i], x[i], dg[i]); db[i] = add2(db[i], t[i]); }
        }
#pragma unroll
        for (int i = 0; i < kPairs; i += 2) {
            const float4 g = vec[i / 2 * kLanes + sub];
            t[i] = mul2(t[i], pair(g.x, g.y));
            t[i + 1] = mul2(t[i + 1], pair(g.z, g.w));
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) q[i] = mul2(t[i], x[i]);
        const float m2 = row_sum(q) * (-1.f / 128.f);
        const Pair p2 = pair(m2, m2);
        if (!RMS) {
            const float m1 = row_sum(t) * (-1.f / 128.f);
            const Pair p1 = pair(m1, m1);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) t[i] = add2(t[i], p1);
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            t[i] = fma2(x[i], p2, t[i]);
            t[i] = a.D ? fma2(t[i], s, d.get(i)) : mul2(t[i], s);
        }
        if (a.dZ && in) Raw<BF16>::store((char*)a.dZ + (int64_t)row * a.lddz, sub, t);
    }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < kPairs / 2; ++i) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float4 f;
            split(m ? db[2 * i] : dg[2 * i], f.x, f.y);
            split(m ? db[2 * i + 1] : dg[2 * i + 1], f.z, f.w);
#pragma unroll
            for (int o = kLanes; o < 32; o <<= 1) {
                f.x += __shfl_xor_sync(0xffffffffu, f.x, o); f.y += __shfl_xor_sync(0xffffffffu, f.y, o);
                f.z += __shfl_xor_sync(0xffffffffu, f.z, o); f.w += __shfl_xor_sync(0xffffffffu, f.w, o);
            }
            if (grp == 0) sum[warp][m][quad_of<BF16>(i, sub)] = f;
        }
    }
    __syncthreads();
    const int m = threadIdx.x >> 7, col = threadIdx.x & 127;
    float f = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) f += reinterpret_cast<const float*>(sum[w][m])[col];
    if (a.part) a.part[(int64_t)blockIdx.x * 256 + threadIdx.x] = f;
    else if (float* out = m ? a.dbeta : a.dgamma) out[col] = f;
}

// 32 of the 256 sums per CTA, a warp per 32nd CTA of norm_bwd_kernel.
__global__ void __launch_bounds__(1024) norm_reduce_kernel(const float* part, int ctas, float* dgamma, float* dbeta) {
    __shared__ float sum[32][33];
    let_next_begin();
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = blockIdx.x * 32 + lane;
    float f = 0.f;
#pragma unroll 4
    for (int c = warp; c < ctas; c += 32) f += part[(int64_t)c * 256 + at];
    sum[warp][lane] = f;
    __syncthreads();
    f = sum[lane][warp];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) f += __shfl_xor_sync(0xffffffffu, f, o);
    const int to = blockIdx.x * 32 + warp;
    if (lane == 0) {
        if (float* out = to < 128 ? dgamma : dbeta) out[to & 127] = f;
    }
}

#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

int ctas_of(int n, int resident) {
    const int needed = (int)(((int64_t)n + kWarps * kRows - 1) / (kWarps * kRows));
    return needed < resident ? needed : resident;
}

template <bool BF16, bool RMS>
dg4_status launch_fwd(const FwdArgs& a, cudaStream_t st) {
    int resident;
    CHECK((dg4i_resident_blocks<add_norm_kernel<BF16, RMS>>(kThreads, &resident)));
    return dg4i_launch(add_norm_kernel<BF16, RMS>, dim3(ctas_of(a.n, resident)), kThreads, 0, st, true, a);
}

// CTAs of the backward kernel: one where its sums are to be final, else as many as the device holds.
template <bool BF16, bool RMS>
dg4_status bwd_ctas(int n, int* out) {
    int resident;
    CHECK((dg4i_resident_blocks<norm_bwd_kernel<BF16, RMS>>(kThreads, &resident)));
    *out = n <= kFewRows ? 1 : ctas_of(n, resident);
    return DG4_OK;
}
dg4_status bwd_ctas(bool bf16, bool rms, int n, int* out) {
    if (bf16) return rms ? bwd_ctas<true, true>(n, out) : bwd_ctas<true, false>(n, out);
    return rms ? bwd_ctas<false, true>(n, out) : bwd_ctas<false, false>(n, out);
}

template <bool BF16, bool RMS>
dg4_status launch_bwd(const BwdArgs& a, int ctas, cudaStream_t st) {
    CHECK(dg4i_launch(norm_bwd_kernel<BF16, RMS>, dim3(ctas), kThreads, 0, st, true, a));
    if (a.part) CHECK(dg4i_launch(norm_reduce_kernel, dim3(8), 1024, 0, st, true, (const float*)a.part, ctas, a.dgamma, a.dbeta));
    return DG4_OK;
}

dg4_status check_eps(float eps) {
    if (!(eps >= 0.f) || eps > 3.0e38f) DG4_FAIL(DG4_ERR_INVALID_ARG, "eps is negative or not finite");
    return DG4_OK;
}

}  // namespace

extern "C" dg4_status dg4_add_norm_fwd(const dg4_graph* g, const dg4_desc* desc, const void* X, int64_t ldx, const void* R,
                                       int64_t ldr, const float* gamma, const float* beta, float eps, void* Z, int64_t ldz,
                                       void* Y, int64_t ldy, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, false));
    const int es = desc->dtype == DG4_BF16 ? 2 : 4;
    CHECK(dg4i_check_tensor("X", X, ldx, es, 128));
    if (R) CHECK(dg4i_check_tensor("R", R, ldr, es, 128));
    CHECK(check_vec("gamma", gamma, false));
    CHECK(check_vec("beta", beta, true));
    CHECK(check_eps(eps));
    if (Z) CHECK(dg4i_check_tensor("Z", Z, ldz, es, 128));
    CHECK(dg4i_check_tensor("Y", Y, ldy, es, 128));
    if (Z == Y) DG4_FAIL(DG4_ERR_INVALID_ARG, "Z and Y are the same buffer");
    if ((Z && Z == X && ldz != ldx) || (Z && Z == R && ldz != ldr) || (Y == X && ldy != ldx) || (Y == R && ldy != ldr))
        DG4_FAIL(DG4_ERR_INVALID_ARG, "an output in the place of X or R has another leading dimension");
    const FwdArgs a = {X, ldx * es, R, ldr * es, Z, ldz * es, Y, ldy * es, gamma, beta, g->n, eps};
    const bool rms = (desc->flags & DG4_FLAG_RMS_NORM) != 0;
    const cudaStream_t st = (cudaStream_t)stream;
    if (es == 2) return rms ? launch_fwd<true, true>(a, st) : launch_fwd<true, false>(a, st);
    return rms ? launch_fwd<false, true>(a, st) : launch_fwd<false, false>(a, st);
}

extern "C" size_t dg4_norm_bwd_workspace_bytes(const dg4_graph* g, const dg4_desc* desc) {
    int ctas = 0;
    if (!g || dg4i_check_desc(desc, false) != DG4_OK) return 0;
    DeviceGuard guard(g->device);                    // the size is the handle's, whichever device is current
    if (!guard.ok || bwd_ctas(desc->dtype == DG4_BF16, (desc->flags & DG4_FLAG_RMS_NORM) != 0, g->n, &ctas) != DG4_OK) return 0;
    return ctas > 1 ? (size_t)ctas * 256 * sizeof(float) : 0;
}

extern "C" dg4_status dg4_norm_bwd(const dg4_graph* g, const dg4_desc* desc, const void* Z, int64_t ldz, const float* gamma,
                                   float eps, const void* dY, int64_t lddy, const void* D_res, int64_t lddr, void* dZ,
                                   int64_t lddz, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, false));
    const int es = desc->dtype == DG4_BF16 ? 2 : 4;
    CHECK(dg4i_check_tensor("Z", Z, ldz, es, 128));
    CHECK(check_vec("gamma", gamma, false));
    CHECK(check_eps(eps));
    CHECK(dg4i_check_tensor("dY", dY, lddy, es, 128));
    if (D_res) CHECK(dg4i_check_tensor("D_res", D_res, lddr, es, 128));
    if (dZ) CHECK(dg4i_check_tensor("dZ", dZ, lddz, es, 128));
    CHECK(check_vec("dgamma", dgamma, true));
    CHECK(check_vec("dbeta", dbeta, true));
    const bool sums = dgamma || dbeta, rms = (desc->flags & DG4_FLAG_RMS_NORM) != 0;
    if (!dZ && !sums) DG4_FAIL(DG4_ERR_INVALID_ARG, "none of dZ, dgamma and dbeta is asked for");
    if (dZ && ((dZ == Z && lddz != ldz) || (dZ == dY && lddz != lddy) || (dZ == D_res && lddz != lddr)))
        DG4_FAIL(DG4_ERR_INVALID_ARG, "dZ in the place of Z, dY or D_res has another leading dimension");
    if (dgamma && dgamma == dbeta) DG4_FAIL(DG4_ERR_INVALID_ARG, "dgamma and dbeta are the same buffer");
    int ctas;
    CHECK(bwd_ctas(es == 2, rms, g->n, &ctas));
    const size_t need = sums && ctas > 1 ? (size_t)ctas * 256 * sizeof(float) : 0;
    if (need && (!workspace || workspace_bytes < need))
        DG4_FAIL(DG4_ERR_INVALID_ARG, "workspace too small: %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
    if (need && ((uintptr_t)workspace & 15u)) DG4_FAIL(DG4_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
    const BwdArgs a = {Z, ldz * es, dY, lddy * es, D_res, lddr * es, dZ, lddz * es, gamma, dgamma, dbeta,
                       need ? (float*)workspace : nullptr, g->n, sums ? 1 : 0, eps};
    const cudaStream_t st = (cudaStream_t)stream;
    if (es == 2) return rms ? launch_bwd<true, true>(a, ctas, st) : launch_bwd<true, false>(a, ctas, st);
    return rms ? launch_bwd<false, true>(a, ctas, st) : launch_bwd<false, false>(a, ctas, st);
}
