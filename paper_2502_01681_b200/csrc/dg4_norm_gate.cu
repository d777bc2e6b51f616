// Norms around a sub-layer in one pass over the rows:
//     R' = res_scale * R + gate * Norm_post(S),      Y = Norm_pre(R'),
// S the sub-layer's output, R the residual stream, the gate a vector per request.  Everything between the two loads
// and the two stores of a row stays in registers in 32 bits (Y is computed from the unrounded R'), so a bf16 row
// costs 512 bytes in and 512 out, which is the bound: the arithmetic is some 20 operations per element.
//
// 16 lanes per row, 8 elements per lane; a warp walks chunks of up to 32 consecutive rows, its two halves on
// alternate rows (fewer rows per chunk when there are not enough for every resident warp: two rows one after the
// other cost twice a row's latency).  The request of a chunk's first row is found by a 16-way search over the offsets (each step one load and one
// ballot), after that only when a row passes the end of its request.  Mean and variance are taken in two passes over
// the registers, so a large common offset of a row does not cancel in the variance.

#include "dg4_internal.h"
#include "dg4_kv8_core.cuh"

namespace {

constexpr int kMaxChunk = 32;              // rows a warp takes at a time, at most
constexpr int kEl = 8;

struct NormArgs {
    const void* S; int64_t lds;            // bytes
    const void* R; int64_t ldr;
    void* R_out; int64_t ldro;
    void* Y; int64_t ldy;                  // Y nullable
    const float* gate;                     // [n_gates, 128], nullable (one)
    const float *post_gamma, *post_beta, *pre_gamma, *pre_beta;   // betas nullable (zero)
    const int32_t *seg_ptr, *seg_id;       // nullable (one request: all rows, gate 0)
    int32_t n_gates, n_seg, n, chunk;
    float res_scale, eps;
};

__device__ __forceinline__ void load_vec(const float* p, int sub, float fill, float* f) {
    if (p) {
        const float4 a = *reinterpret_cast<const float4*>(p + sub * kEl), b = *reinterpret_cast<const float4*>(p + sub * kEl + 4);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < kEl; ++i) f[i] = fill;
    }
}

__device__ __forceinline__ float row_sum(float x, unsigned mask) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(mask, x, o);
    return x;
}

// x := Norm(x) * gamma + beta for the row that the 16 lanes hold
template <bool RMS>
__device__ __forceinline__ void norm_row(float* x, const float* gamma, const float* beta, float eps, unsigned mask) {
    if (!RMS) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kEl; ++i) s += x[i];
        const float mean = row_sum(s, mask) * (1.f / 128.f);
#pragma unroll
        for (int i = 0; i < kEl; ++i) x[i] -= mean;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < kEl; ++i) q = fmaf(x[i], x[i], q);
    const float inv = rsqrtf(row_sum(q, mask) * (1.f / 128.f) + eps);
#pragma unroll
    for (int i = 0; i < kEl; ++i) x[i] = fmaf(x[i] * inv, gamma[i], beta[i]);
}

// The request of a row: the last s with seg_ptr[s] <= row, -1 if there is none.  All 16 lanes of `mask` call it.
__device__ __forceinline__ int find_segment(const int32_t* seg_ptr, int n_seg, int row, int sub, unsigned mask) {
    int lo = 0, hi = n_seg;                // entries below lo are <= row, entries from hi on are > row
    while (lo < hi) {
        const int step = (hi - lo + 15) >> 4;
        const int64_t at = (int64_t)lo + (int64_t)(sub + 1) * step - 1;
        const bool below = at < hi && seg_ptr[at] <= row;
        const int c = __popc(__ballot_sync(mask, below) & mask);
        const int64_t next = (int64_t)lo + (int64_t)(c + 1) * step - 1;
        lo += c * step;
        hi = next < hi ? (int)next : hi;
    }
    return lo - 1;
}

template <bool BF16, bool RMS>
__global__ void __launch_bounds__(256) norm_gate_kernel(NormArgs a) {
    const int lane = threadIdx.x & 31, sub = lane & 15, half = lane >> 4;
    const unsigned mask = 0xffffu << (lane - sub);
    float post_g[kEl], post_b[kEl], pre_g[kEl], pre_b[kEl], gate[kEl];
    load_vec(a.post_gamma, sub, 1.f, post_g);
    load_vec(a.post_beta, sub, 0.f, post_b);
    load_vec(a.Y ? a.pre_gamma : nullptr, sub, 1.f, pre_g);
    load_vec(a.Y ? a.pre_beta : nullptr, sub, 0.f, pre_b);
    load_vec(a.seg_ptr ? nullptr : a.gate, sub, 1.f, gate);
    const int64_t chunks = ((int64_t)a.n + a.chunk - 1) / a.chunk;
    const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5);
    for (int64_t chunk = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; chunk < chunks; chunk += warps) {
        int end = a.seg_ptr ? -1 : a.n;    // rows below `end` belong to the request whose gate is held
        bool covered = true;
        for (int i = half; i < a.chunk; i += 2) {
            const int64_t row = chunk * a.chunk + i;
            if (row >= a.n) break;
            if (row >= end) {
                const int s = find_segment(a.seg_ptr, a.n_seg, (int)row, sub, mask);
                covered = s >= 0 && row < a.seg_ptr[s + 1];
                end = s + 1 <= a.n_seg ? a.seg_ptr[s + 1] : a.n;
                if (end <= row) end = a.n;                      // behind the last request: nothing more is written
                if (covered) {
                    const int id = a.seg_id[s];
                    load_vec((uint32_t)id < (uint32_t)a.n_gates && a.gate ? a.gate + (int64_t)id * 128 : nullptr, sub, 1.f, gate);
                }
            }
            if (!covered) continue;
            float x[kEl], r[kEl];
            kv8::load8<BF16>((const char*)a.S + row * a.lds, sub, x);
            kv8::load8<BF16>((const char*)a.R + row * a.ldr, sub, r);
            norm_row<RMS>(x, post_g, post_b, a.eps, mask);
#pragma unroll
            for (int e = 0; e < kEl; ++e) x[e] = fmaf(gate[e], x[e], a.res_scale * r[e]);
            kv8::store8<BF16>((char*)a.R_out + row * a.ldro, sub, x);
            if (a.Y) {
                norm_row<RMS>(x, pre_g, pre_b, a.eps, mask);
                kv8::store8<BF16>((char*)a.Y + row * a.ldy, sub, x);
            }
        }
    }
}

#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

dg4_status check_vec(const char* name, const void* p, bool optional) {
    if (!p && optional) return DG4_OK;
    if (!p) DG4_FAIL(DG4_ERR_INVALID_ARG, "%s is null", name);
    if (((uintptr_t)p & 15u) != 0) DG4_FAIL(DG4_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return DG4_OK;
}

template <bool BF16, bool RMS>
dg4_status launch(NormArgs a, cudaStream_t st) {
    int dev = 0, sms = 0, per_sm = 0;
    DG4_CUDA_TRY(cudaGetDevice(&dev));
    DG4_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    DG4_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, norm_gate_kernel<BF16, RMS>, 256, 0));
    const int64_t resident = (int64_t)sms * (per_sm > 0 ? per_sm : 1);
    const int64_t share = ((int64_t)a.n + 16 * resident - 1) / (16 * resident);      // rows of a half-warp
    a.chunk = (int32_t)(2 * share < kMaxChunk ? 2 * share : kMaxChunk);
    const int64_t needed = ((int64_t)a.n + 8 * a.chunk - 1) / (8 * a.chunk);
    norm_gate_kernel<BF16, RMS><<<(unsigned)(needed < resident ? needed : resident), 256, 0, st>>>(a);
    dg4i_count_launch();
    DG4_CUDA_TRY(cudaGetLastError());
    return DG4_OK;
}

}  // namespace

dg4_status dg4i_check_segments(const dg4_segments* seg) {
    if (seg->n_seg < 1) DG4_FAIL(DG4_ERR_INVALID_ARG, "the number of segments (%d) is below one", seg->n_seg);
    if (!seg->seg_ptr || !seg->seg_id) DG4_FAIL(DG4_ERR_INVALID_ARG, "the segments' arrays are null");
    if (((uintptr_t)seg->seg_ptr & 3u) || ((uintptr_t)seg->seg_id & 3u))
        DG4_FAIL(DG4_ERR_INVALID_ARG, "the segments' arrays are not 4-byte aligned");
    return DG4_OK;
}

extern "C" dg4_status dg4_norm_gate_fwd(const dg4_graph* g, const dg4_desc* desc, const void* S, int64_t lds,
                                        const void* R, int64_t ldr, float res_scale, const float* gate,
                                        int32_t n_gates, const dg4_segments* seg, const float* post_gamma,
                                        const float* post_beta, const float* pre_gamma, const float* pre_beta,
                                        float eps, void* R_out, int64_t ldro, void* Y, int64_t ldy, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, false));
    const int es = desc->dtype == DG4_BF16 ? 2 : 4;
    CHECK(dg4i_check_tensor("S", S, lds, es, 128));
    CHECK(dg4i_check_tensor("R", R, ldr, es, 128));
    CHECK(dg4i_check_tensor("R_out", R_out, ldro, es, 128));
    if (Y) CHECK(dg4i_check_tensor("Y", Y, ldy, es, 128));
    CHECK(check_vec("post_gamma", post_gamma, false));
    CHECK(check_vec("post_beta", post_beta, true));
    CHECK(check_vec("pre_gamma", pre_gamma, !Y));
    CHECK(check_vec("pre_beta", pre_beta, true));
    CHECK(check_vec("gate", gate, true));
    if (!(eps >= 0.f) || eps > 3.0e38f) DG4_FAIL(DG4_ERR_INVALID_ARG, "eps is negative or not finite");
    if (!(res_scale >= -3.0e38f && res_scale <= 3.0e38f)) DG4_FAIL(DG4_ERR_INVALID_ARG, "res_scale is not finite");
    if (gate && n_gates < 1) DG4_FAIL(DG4_ERR_INVALID_ARG, "the number of gates (%d) is below one", n_gates);
    if (gate && !seg && n_gates != 1) DG4_FAIL(DG4_ERR_INVALID_ARG, "%d gates but no segments to choose among them", n_gates);
    if (Y && Y == R_out) DG4_FAIL(DG4_ERR_INVALID_ARG, "Y and R_out are the same buffer");
    if (seg) CHECK(dg4i_check_segments(seg));
    NormArgs a;
    a.S = S; a.lds = lds * es; a.R = R; a.ldr = ldr * es; a.R_out = R_out; a.ldro = ldro * es; a.Y = Y; a.ldy = ldy * es;
    a.gate = gate; a.n_gates = gate ? n_gates : 0;
    a.post_gamma = post_gamma; a.post_beta = post_beta; a.pre_gamma = pre_gamma; a.pre_beta = pre_beta;
    a.seg_ptr = seg ? seg->seg_ptr : nullptr; a.seg_id = seg ? seg->seg_id : nullptr; a.n_seg = seg ? seg->n_seg : 0;
    a.n = g->n; a.chunk = kMaxChunk; a.res_scale = res_scale; a.eps = eps;
    const bool rms = (desc->flags & DG4_FLAG_RMS_NORM) != 0;
    const cudaStream_t st = (cudaStream_t)stream;
    if (es == 2) return rms ? launch<true, true>(a, st) : launch<true, false>(a, st);
    return rms ? launch<false, true>(a, st) : launch<false, false>(a, st);
}
