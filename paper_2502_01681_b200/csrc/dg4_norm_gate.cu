// Norms around a sub-layer in one pass over the rows:
//     R' = res_scale * R + gate * Norm_post(S),      Y = Norm_pre(R'),
// S the sub-layer's output, R the residual stream, the gate a vector per request.  Everything between the two loads
// and the two stores of a row stays in registers in 32 bits (Y is computed from the unrounded R'), so a bf16 row
// costs 512 bytes in and 512 out, which is the bound: 1.01M rows in 164 us in short runs,
// sustained 167 us, 6.2 TB/s (96 % of the measured copy rate); fp32 rows 334 us (96 %).
//
// 8 lanes per row, 16 elements per lane, four consecutive rows per warp: each sum over a row takes 3 shuffles for four
// rows at once, and the arithmetic runs on pairs (packed fp32 instructions).  The norm vectors lie in shared memory in
// the order the lanes read them, the gate in registers.  A warp walks chunks of up to 16 consecutive rows (chunks of 32:
// 168 us, of 8: 164, of 4: 167); the next four rows are loaded while four are worked on.  (16 lanes per row and the
// vectors in registers: 224 us; a warp per row: 230.)  The request of a row is found by a 32-way search over the offsets
// (each step one load and one ballot), only when the four rows leave the request last found; where they belong to
// several requests, each row's lanes search for their own.  Mean and variance are taken in two passes over the
// registers, so a large common offset of a row does not cancel in the variance.

#include "dg4_internal.h"
#include "dg4_launch.cuh"
#include "dg4_norm_core.cuh"

using namespace normcore;

namespace {

constexpr int kMaxChunk = 16;              // rows a warp takes at a time, at most

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

// The request of a row: the last s with seg_ptr[s] <= row, -1 if there is none.  The lanes of `mask` call it together,
// `ways` of them (a power of two), `me` counting them from 0.
__device__ __forceinline__ int find_segment(const int32_t* seg_ptr, int n_seg, int row, int me, int ways, unsigned mask) {
    int lo = 0, hi = n_seg;                // entries below lo are <= row, entries from hi on are > row
    while (lo < hi) {
        const int step = (int)(((uint32_t)(hi - lo) + ways - 1) / ways);
        const int64_t at = (int64_t)lo + (int64_t)(me + 1) * step - 1;
        const bool below = at < hi && seg_ptr[at] <= row;
        const int c = __popc(__ballot_sync(mask, below) & mask);
        const int64_t next = (int64_t)lo + (int64_t)(c + 1) * step - 1;
        lo += c * step;
        hi = next < hi ? (int)next : hi;
    }
    return lo - 1;
}

template <bool BF16, bool RMS>
__global__ void __launch_bounds__(256, 2) norm_gate_kernel(NormArgs a) {
    __shared__ float4 vec[4][32];
    const int lane = threadIdx.x & 31, sub = lane & (kLanes - 1), grp = lane / kLanes;
    if (threadIdx.x < 128) {                                         // place i * 8 + sub holds quad_of(i, sub)
        const int v = threadIdx.x >> 5, t = threadIdx.x & 31;
        const float* p = v == 0 ? a.post_gamma : v == 1 ? a.post_beta : v == 2 ? a.pre_gamma : a.pre_beta;
        const float fill = (v & 1) ? 0.f : 1.f;
        if (!a.Y && v >= 2) p = nullptr;
        vec[v][t] = p ? reinterpret_cast<const float4*>(p)[quad_of<BF16>(t / kLanes, t & (kLanes - 1))] : make_float4(fill, fill, fill, fill);
    }
    __syncthreads();
    Pair gate[kPairs];
    auto set_gate = [&](int id) {
        const float4* p = reinterpret_cast<const float4*>(a.gate) + (int64_t)id * 32;
        const bool has = a.gate && (uint32_t)id < (uint32_t)a.n_gates;
#pragma unroll
        for (int i = 0; i < kPairs / 2; ++i) {
            const float4 g = has ? p[quad_of<BF16>(i, sub)] : make_float4(1.f, 1.f, 1.f, 1.f);
            gate[2 * i] = pair(g.x, g.y);
            gate[2 * i + 1] = pair(g.z, g.w);
        }
    };
    const uint32_t step = gridDim.x * (blockDim.x >> 5) * a.chunk;
    uint32_t chunk = ((blockIdx.x * blockDim.x + threadIdx.x) >> 5) * a.chunk;
    uint32_t row0 = chunk;                                           // the first of the four rows
    const uint32_t n = (uint32_t)a.n;
    bool covered = true;                                             // this lane's row belongs to a request
    uint32_t end = n;                                                // rows below it have this `gate` and `covered`
    if (a.seg_ptr) end = 0;
    else set_gate(0);
    Raw<BF16> s_next, r_next;
    auto fetch = [&](uint32_t row) {
        if (row < n) {
            s_next.load((const char*)a.S + (int64_t)row * a.lds, sub);
            r_next.load((const char*)a.R + (int64_t)row * a.ldr, sub);
        }
    };
    fetch(row0 + grp);
    const Pair rs = pair(a.res_scale, a.res_scale);
    while (row0 < n) {                                               // the whole warp
        const uint32_t row = row0 + grp;
        Pair x[kPairs], r[kPairs];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) { x[i] = s_next.get(i); r[i] = r_next.get(i); }
        uint32_t next = row0 + kRows;
        if (next >= chunk + a.chunk) next = chunk += step;
        fetch(next + grp);
        if (min(row0 + kRows, n) > end) {
            int s = find_segment(a.seg_ptr, a.n_seg, (int)row0, lane, 32, 0xffffffffu);
            // between the end of request s and the beginning of the next non-empty one there may be rows of none
            const int to = a.seg_ptr[s + 1];
            end = to > (int)row0 ? (uint32_t)to : n;                 // behind the last request nothing is written
            covered = s >= 0 && to > (int)row0;
            if (min(row0 + kRows, n) > end) {                        // several requests: each row for itself, this once
                s = find_segment(a.seg_ptr, a.n_seg, (int)min(row, n - 1), sub, kLanes, 0xffu << (lane - sub));
                covered = s >= 0 && a.seg_ptr[s + 1] > (int)row;
                end = 0;
            }
            if (covered) set_gate(a.seg_id[s]);
        }
        norm_row<RMS>(x, &vec[0][sub], &vec[1][sub], a.eps);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[i] = fma2(gate[i], x[i], mul2(rs, r[i]));
        const bool writes = covered && row < n;
        if (writes) Raw<BF16>::store((char*)a.R_out + (int64_t)row * a.ldro, sub, x);
        if (a.Y) {
            norm_row<RMS>(x, &vec[2][sub], &vec[3][sub], a.eps);
            if (writes) Raw<BF16>::store((char*)a.Y + (int64_t)row * a.ldy, sub, x);
        }
        row0 = next;
    }
}

#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

template <bool BF16, bool RMS>
dg4_status launch(NormArgs a, cudaStream_t st) {
    int resident;
    CHECK((dg4i_resident_blocks<norm_gate_kernel<BF16, RMS>>(256, &resident)));
    const int64_t share = ((int64_t)a.n + 8 * (int64_t)resident - 1) / (8 * (int64_t)resident);        // rows of a warp
    a.chunk = (int32_t)(share < kMaxChunk ? (share + kRows - 1) / kRows * kRows : kMaxChunk);
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
