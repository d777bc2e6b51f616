// Rows of 128 elements in registers, eight lanes per row: how the norm kernels hold, load, store and sum them.
#pragma once

#include "dg4_attn_core.cuh"
#include "dg4_internal.h"
#include "dg4_pairs.cuh"

namespace normcore {

constexpr int kRows = 4;                    // rows of a warp at a time
constexpr int kLanes = 8;                   // lanes per row
constexpr int kEl = 128 / kLanes;           // elements per lane
constexpr int kPairs = kEl / 2;

// Which four elements of a row the i-th quadruple of a lane is (counted in quadruples): a lane's loads are 16 bytes, 8
// lanes side by side, so bf16 rows give it two neighbouring quadruples at a time and fp32 rows one.
template <bool BF16> __device__ __forceinline__ int quad_of(int i, int sub) {
    return BF16 ? 2 * (sub + kLanes * (i >> 1)) + (i & 1) : sub + kLanes * i;
}

// a lane's 16 elements of a row as they stand in memory, streamed
template <bool BF16> struct Raw {
    static constexpr int kPieces = BF16 ? 2 : 4;
    attn::Piece p[kPieces];
    __device__ __forceinline__ void load(const char* row, int sub) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) p[i] = attn::ld_piece_stream(row + (sub + kLanes * i) * 16);
    }
    __device__ __forceinline__ Pair get(int i) const {               // pair i of the lane's 8
        if (BF16) {
            const uint32_t w = p[i >> 2].w[i & 3];
            return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        }
        return pair(__uint_as_float(p[BF16 ? 0 : i >> 1].w[2 * (i & 1)]), __uint_as_float(p[BF16 ? 0 : i >> 1].w[2 * (i & 1) + 1]));
    }
    __device__ static __forceinline__ void store(char* row, int sub, const Pair* x) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            float f[8];
#pragma unroll
            for (int e = 0; e < kPairs / kPieces; ++e) split(x[i * (kPairs / kPieces) + e], f[2 * e], f[2 * e + 1]);
            attn::st_piece_stream(row + (sub + kLanes * i) * 16, attn::Elem<BF16>::pack(f));
        }
    }
};

__device__ __forceinline__ float row_sum(const Pair* x) {            // over the 8 lanes of a row
    const Pair t = add2(add2(add2(x[0], x[1]), add2(x[2], x[3])), add2(add2(x[4], x[5]), add2(x[6], x[7])));
    float a, b;
    split(t, a, b);
    a += b;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    return a;
}

// x := Norm(x) * gamma + beta; v: gamma and beta as this lane reads them, quadruple after quadruple
template <bool RMS>
__device__ __forceinline__ void norm_row(Pair* x, const float4* gamma, const float4* beta, float eps) {
    if (!RMS) {
        const float mean = row_sum(x) * (1.f / 128.f);
        const Pair m = pair(-mean, -mean);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[i] = add2(x[i], m);
    }
    Pair q[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) q[i] = mul2(x[i], x[i]);
    const float inv = rsqrtf(row_sum(q) * (1.f / 128.f) + eps);
    const Pair s = pair(inv, inv);
#pragma unroll
    for (int i = 0; i < kPairs; i += 2) {
        const float4 g = gamma[i / 2 * kLanes], b = beta[i / 2 * kLanes];
        x[i] = fma2(mul2(x[i], s), pair(g.x, g.y), pair(b.x, b.y));
        x[i + 1] = fma2(mul2(x[i + 1], s), pair(g.z, g.w), pair(b.z, b.w));
    }
}

// An fp32 vector of a norm's argument list.
inline dg4_status check_vec(const char* name, const void* p, bool optional) {
    if (!p && optional) return DG4_OK;
    if (!p) DG4_FAIL(DG4_ERR_INVALID_ARG, "%s is null", name);
    if (((uintptr_t)p & 15u) != 0) DG4_FAIL(DG4_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return DG4_OK;
}

}  // namespace normcore
