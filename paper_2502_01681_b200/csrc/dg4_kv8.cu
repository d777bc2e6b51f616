// The 8-bit K | V table: writing rows, reading them back, and sparse attention over it.
//
// Writing and reading are bound by HBM: 16 lanes per row (two rows per warp), 8 elements of K and of V per lane (see
// dg4_kv8_core.cuh for the row); each row passes through registers once, 512 + 288 bytes in bf16.  1.01M rows written
// and read back: 276 us in short runs, 280 sustained, 5.8 TB/s (89 % of the measured copy rate); 250 007 fp32 rows: 111
// and 114 us.
// The attention gathers 288 bytes per member instead of 512 and is bound by instructions (see there).

#include "dg4_internal.h"
#include "dg4_kv8_core.cuh"
#include "dg4_launch.cuh"

#include <type_traits>

namespace {

using namespace attn;
using namespace kv8;

struct CopyArgs {
    void* K; int64_t ldk;              // bytes
    void* V; int64_t ldv;
    uint8_t* T; int64_t ldt;
    const int32_t* nodes;              // nullable
    int32_t count, n;
    int32_t wide;                      // fp32 rows: bases and row distances are multiples of 32 bytes
};

// Largest magnitude bit pattern over the lanes of a head (LPH adjacent lanes): magnitudes of floats order like
// their bit patterns, infinities and NaNs above all numbers, so one integer maximum also finds non-finite slices.
template <int LPH>
__device__ __forceinline__ uint32_t slice_top(const float* f, unsigned mask) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kEl; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(mask, top, o));
    return top;
}

// 8 elements of K and of V as they stand in memory.  fp32 rows whose 32 bytes per lane are aligned to that move with one
// instruction (`wide`, the same for the whole launch).
template <bool BF16> struct RawKV {
    static constexpr int kPieces = BF16 ? 1 : 2;
    Piece k[kPieces], v[kPieces];
    __device__ __forceinline__ void load(const CopyArgs& a, int row, int sub) {
        const char* pk = (const char*)a.K + (int64_t)row * a.ldk + sub * 16 * kPieces;
        const char* pv = (const char*)a.V + (int64_t)row * a.ldv + sub * 16 * kPieces;
        if (BF16) {
            k[0] = ld_piece_stream(pk);
            v[0] = ld_piece_stream(pv);
        } else if (a.wide) {
            ld_pieces2_nc(pk, k[0], k[kPieces - 1]);
            ld_pieces2_nc(pv, v[0], v[kPieces - 1]);
        } else {
            k[0] = ld_piece_stream(pk); k[kPieces - 1] = ld_piece_stream(pk + 16);
            v[0] = ld_piece_stream(pv); v[kPieces - 1] = ld_piece_stream(pv + 16);
        }
    }
};

// The id of the row a slot stands for, -1 for none (ids outside the table are skipped)
__device__ __forceinline__ int row_of(const CopyArgs& a, uint32_t slot) {
    int v = -1;
    if (slot < (uint32_t)a.count) v = a.nodes ? a.nodes[slot] : (int)slot;
    return (uint32_t)v < (uint32_t)a.n ? v : -1;
}

// In both kernels the next row's loads are in flight while this row is worked on and stored.
template <bool BF16, int LPH>
__global__ void __launch_bounds__(256) kv8_write_kernel(CopyArgs a) {
    const int lane = threadIdx.x & 31, sub = lane & 15, grp = lane - sub;
    const unsigned mask = 0xffffu << grp;
    const uint32_t stride = gridDim.x * (blockDim.x / kLanes);
    uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) / kLanes;
    RawKV<BF16> raw;
    int row_next = row_of(a, slot);
    if (row_next >= 0) raw.load(a, row_next, sub);
    for (; slot < (uint32_t)a.count; slot += stride) {
        const int row = row_next;
        float k[kEl], w[kEl];
#pragma unroll
        for (int i = 0; i < RawKV<BF16>::kPieces; ++i) {
            Elem<BF16>::unpack(raw.k[i], k + 4 * i);
            Elem<BF16>::unpack(raw.v[i], w + 4 * i);
        }
        row_next = row_of(a, slot + stride);
        if (row_next >= 0) raw.load(a, row_next, sub);
        if (row < 0) continue;
        const uint32_t bk = scale_byte(slice_top<LPH>(k, mask)), bv = scale_byte(slice_top<LPH>(w, mask));
        Piece p;
        encode8(k, bk, p.w);
        encode8(w, bv, p.w + 2);
        uint8_t* t = a.T + (int64_t)row * a.ldt;
        *reinterpret_cast<Piece*>(t + sub * 16) = p;
        // lane l writes the pair of head l (held by the lanes of that head), the lanes beyond the heads write zero
        const uint32_t mine = bk | (bv << 8);
        const uint32_t pair = __shfl_sync(mask, mine, grp + ((sub * LPH) & 15));
        *reinterpret_cast<uint16_t*>(t + kCodeBytes + 2 * sub) = (uint16_t)(sub < 16 / LPH ? pair : 0u);
    }
}

template <bool BF16, int LPH>
__global__ void __launch_bounds__(256) kv8_read_kernel(CopyArgs a) {
    const int sub = threadIdx.x & 15;
    const uint32_t stride = gridDim.x * (blockDim.x / kLanes);
    uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) / kLanes;
    Piece p_next;
    uint32_t pair_next = 0;
    int row_next = -1;
    auto fetch = [&](uint32_t at) {
        row_next = row_of(a, at);
        if (row_next >= 0) {
            const uint8_t* t = a.T + (int64_t)row_next * a.ldt;
            p_next = ld_piece_stream(t + sub * 16);
            pair_next = ld_pair(t + kCodeBytes + 2 * (sub / LPH));
        }
    };
    fetch(slot);
    for (; slot < (uint32_t)a.count; slot += stride) {
        const int row = row_next;
        const Piece p = p_next;
        const uint32_t pair = pair_next;
        fetch(slot + stride);
        if (row < 0) continue;
        const float sk = scale_k(pair), sv = scale_v(pair);
        float k[kEl], w[kEl];
        decode4(p.w[0], k); decode4(p.w[1], k + 4);
        decode4(p.w[2], w); decode4(p.w[3], w + 4);
#pragma unroll
        for (int i = 0; i < kEl; ++i) { k[i] *= sk; w[i] *= sv; }
        char* pk = (char*)a.K + (int64_t)row * a.ldk;
        char* pv = (char*)a.V + (int64_t)row * a.ldv;
        if (!BF16 && a.wide) {
            st_pieces2_stream(pk + sub * 32, Elem<BF16>::pack(k), Elem<BF16>::pack(k + 4));
            st_pieces2_stream(pv + sub * 32, Elem<BF16>::pack(w), Elem<BF16>::pack(w + 4));
        } else {
            store8<BF16>(pk, sub, k);
            store8<BF16>(pv, sub, w);
        }
    }
}

struct AttnArgs {
    const void* Q; int64_t ldq;        // bytes
    const uint8_t* T; uint32_t ldt;
    void* O; int64_t ldo;
    const int32_t* nodes;              // nullable
    const int32_t* nbr_pad;            // fixed-width lists (two hops at most)
    const int32_t* nbr_ptr;            // CSR lists (wider cones)
    const int32_t* nbr_idx;
    int32_t count, n;
    float c;                           // scale * log2(e): scores are kept in log2 units
};

// Attention is bound by instructions, not by bytes: a member's 256 codes cost 128 conversions to pairs of fp16 and 256
// multiply-adds, whoever does them, and every lane that takes part pays the member's addresses, scales, exponential and
// sums on top.  So
//  - a row is spread over as few lanes as the heads allow: 8 lanes with two pieces (one 32-byte load) each for up to 8
//    heads (a lane then holds 16 elements; with 8 heads that is a head, and a score needs no shuffle), 16 lanes with
//    one piece each for 16;
//  - for bf16 rows the multiply-adds take the fp16 codes as they are (fp16 x fp16 + fp32), which saves the 256
//    conversions to fp32.  The query is brought to fp16 for that, times a power of two that puts the largest magnitude
//    of its head into [2^14, 2^15): a bf16 number then fits exactly down to 2^-25 of that magnitude, and what is
//    smaller is off by at most 2^-40 of it.  The weights are rounded to fp16 (off by at most 2^-11 of themselves,
//    an eighth of the output's own rounding); their sum is taken in fp32 before that rounding.  fp32 rows keep query
//    and weights in fp32.
// A member's weight on its codes is exp2(score - max score) * (V scale), of which the scales alone may span 2^247.
// Before it is rounded to fp16 it is therefore measured against the largest weight of the node and head, which is put
// near 2^14 by a power of two (the other end of fp16's range, 2^-24, is then so far below that it does not matter).
// exponent field of the power of two that puts a largest magnitude `top` into [2^14, 2^15), kept where that power and
// its inverse (field 254 - b) are normal numbers
__device__ __forceinline__ uint32_t lift(float top) { return min(268u - (__float_as_uint(top) >> 23), 253u); }

template <bool BF16, int LANES> struct Query {
    static constexpr int kN = 128 / LANES;
    uint32_t h[BF16 ? kN / 2 : 1];
    float f[BF16 ? 1 : kN];
    float c;                                   // what makes a dot product with codes times the K scale a score in log2 units
    // fp32 queries are brought down by a power of two, too, where their largest element is above 2^15 (what that takes from
    // their small ones is below 2^-140 of the largest), so that a dot product with codes is at most 2^31 for both types.
    template <int LPH>
    __device__ __forceinline__ void set(const float* q, float scale) {
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < kN; ++e) top = fmaxf(top, fabsf(q[e]));
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const uint32_t b = BF16 ? lift(top) : min(lift(top), 127u);
        const float up = __uint_as_float(b << 23);
        c = (BF16 ? 0.5f : 1.f) * scale * __uint_as_float((254u - b) << 23);
        if (BF16) {
#pragma unroll
            for (int e = 0; e < kN / 2; ++e) {
                const __half2 x = __floats2half2_rn(q[2 * e] * up, q[2 * e + 1] * up);
                h[e] = *reinterpret_cast<const uint32_t*>(&x);
            }
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) f[e] = q[e] * up;
        }
    }
    // Score from a dot product with codes and the K scale.  Up to |c| = 2^96 the product with c goes first: it does not
    // overflow (queries of 2^113 and more have a larger c).  Beyond, the product with the scale goes first: it overflows
    // only where the score does, and what it loses to underflow is below 2^-149 c <= 2^-36 of a score.  FAR: some lane
    // of the warp is beyond; each lane goes by its own c.
    __device__ __forceinline__ bool is_far() const { return fabsf(c) > 0x1p96f; }
    template <bool FAR> __device__ __forceinline__ float score(float dot, float k_scale) const {
        return FAR && is_far() ? dot * k_scale * c : dot * c * k_scale;
    }
};

__device__ __forceinline__ void fma_half2(uint32_t a, uint32_t b, float& lo, float& hi) {     // lo += a.lo b.lo, hi += a.hi b.hi
    asm("{\n\t.reg .b16 al, ah, bl, bh;\n\tmov.b32 {al, ah}, %2;\n\tmov.b32 {bl, bh}, %3;\n\t"
        "fma.rn.f32.f16 %0, al, bl, %0;\n\tfma.rn.f32.f16 %1, ah, bh, %1;\n\t}"
        : "+f"(lo), "+f"(hi) : "r"(a), "r"(b));
}

template <bool BF16, int LANES> struct Row {
    static constexpr int kPieces = 16 / LANES, kN = 8 * kPieces;

    Piece p[kPieces];
    uint32_t pair;
    // bf16 rows: twice the scale (two instructions fewer), put right in the query's factor and at the end
    __device__ static __forceinline__ float k_scale(uint32_t pair) { return BF16 ? twice_scale_k(pair) : scale_k(pair); }
    __device__ static __forceinline__ float v_scale(uint32_t pair) { return BF16 ? twice_scale_v(pair) : scale_v(pair); }
    // codes: T + this lane's pieces; exps: T + this lane's pair
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* exps, uint32_t row, uint32_t ldt) {
        // one wide multiply-add per address
        const uint64_t pc = (uint64_t)row * ldt + (uint64_t)codes, pe = (uint64_t)row * ldt + (uint64_t)exps;
        if (kPieces == 2) ld_pieces2_nc((const void*)pc, p[0], p[kPieces - 1]);
        else p[0] = ld_piece_nc((const void*)pc);
        pair = ld_pair((const void*)pe);
    }
    __device__ __forceinline__ float dot(const Query<BF16, LANES>& q) const {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i) {
            const uint32_t w = p[i >> 1].w[i & 1];
            if (BF16) {
                uint32_t k[2];
                decode4_half(w, k);
                fma_half2(k[0], q.h[2 * i], a, b);
                fma_half2(k[1], q.h[2 * i + 1], a, b);
            } else {
                float k[4];
                decode4(w, k);
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    a = fmaf(q.f[4 * i + e], k[e], a);
                    b = fmaf(q.f[4 * i + e + 1], k[e + 1], b);
                }
            }
        }
        return a + b;
    }
    __device__ __forceinline__ void add(float weight, float* acc) const {
        const __half2 w2 = __floats2half2_rn(weight, weight);
        const uint32_t wh = *reinterpret_cast<const uint32_t*>(&w2);
#pragma unroll
        for (int i = 0; i < 2 * kPieces; ++i) {
            const uint32_t w = p[i >> 1].w[2 + (i & 1)];
            float* o = acc + 4 * i;
            if (BF16) {
                uint32_t v[2];
                decode4_half(w, v);
                fma_half2(v[0], wh, o[0], o[1]);
                fma_half2(v[1], wh, o[2], o[3]);
            } else {
                float v[4];
                decode4(w, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(weight, v[e], o[e]);
            }
        }
    }
};
// this lane's part of a row as it stands in memory, so that a row fetched early costs no more registers than that
template <bool BF16, int LANES> struct RawRow {
    static constexpr int kPieces = (BF16 ? 1 : 2) * 16 / LANES;
    Piece p[kPieces];
    __device__ __forceinline__ void load(const void* row, int sub) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) p[i] = ld_piece_stream((const char*)row + (sub * kPieces + i) * 16);
    }
    __device__ __forceinline__ void unpack(float* f) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) Elem<BF16>::unpack(p[i], f + i * Elem<BF16>::kPerPiece);
    }
};
template <bool BF16, int LANES>
__device__ __forceinline__ void store_row(void* row, int sub, const float* f) {
#pragma unroll
    for (int i = 0; i < 16 / LANES; ++i) store8<BF16>(row, sub * (16 / LANES) + i, f + 8 * i);
}

// Lists of at most MAXN members from the fixed-width table.  A group of LANES lanes takes a node; the nodes in flight
// across the GPU are a contiguous range.  A member beyond a node's own list weighs zero (its filler is the node's own
// row, so no value enters that the node does not read anyway).  The scores come in two runs without a branch inside, the
// first three members and the others, so that their chains of dependent instructions overlap; the sums skip what lies
// beyond the longest list of the warp (1.01M two-hop cones: 216 us, under sustained load 243; with a branch at every
// member 244, with none 229 and 262; fp32 rows 291 and 332).
// The loads run ahead of the arithmetic: lists two nodes ahead, and a member's row of the next node goes into the
// registers of this node's as soon as that has been added up.
template <bool BF16, int LANES, int LPH, int MAXN>
__global__ void __launch_bounds__(256, LANES == 8 ? 2 : 3) sparse_attn_kv8_kernel(AttnArgs a) {
    constexpr int W = MAXN + 1, N = Row<BF16, LANES>::kN;
    const int lane = threadIdx.x & 31, sub = lane & (LANES - 1), grp = lane - sub;
    const uint32_t stride = gridDim.x * (blockDim.x / LANES);
    uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) / 32 * (32 / LANES) + lane / LANES;
    uint32_t base = slot - lane / LANES;                                      // the warp's first slot
    const uint8_t* codes = a.T + sub * (256 / LANES);
    const uint8_t* exps = a.T + kCodeBytes + 2 * (sub / LPH);
    auto node_of = [&](uint32_t s) {
        int v = -1;
        if (s < (uint32_t)a.count) v = a.nodes ? a.nodes[s] : (int)s;
        return (uint32_t)v < (uint32_t)a.n ? v : -1;                          // ids outside the graph are skipped
    };
    auto list_of = [&](int v) { return sub < W && v >= 0 ? a.nbr_pad[(size_t)v * W + sub] : 0; };
    Row<BF16, LANES> row[MAXN];
    RawRow<BF16, LANES> raw;
    int v = node_of(slot), pad = list_of(v);
    int v1 = node_of(slot + stride), pad1 = list_of(v1);
    raw.load((const char*)a.Q + (int64_t)max(v, 0) * a.ldq, sub);
#pragma unroll
    for (int j = 0; j < MAXN; ++j)
        row[j].load(codes, exps, (uint32_t)(j ? __shfl_sync(0xffffffffu, pad, grp + j) : max(v, 0)), a.ldt);
    for (; base < (uint32_t)a.count; base += stride, slot += stride) {
        const int cnt = __shfl_sync(0xffffffffu, pad, grp);
        const int most = __reduce_max_sync(0xffffffffu, cnt);                 // the longest list of the warp
        const bool more = base + stride < (uint32_t)a.count;                  // the warp has another round
        const int v2 = node_of(slot + 2 * stride), pad2 = list_of(v2);
        float acc[N];
        raw.unpack(acc);
        Query<BF16, LANES> q;
        q.template set<LPH>(acc, a.c);
        if (more) raw.load((const char*)a.Q + (int64_t)max(v1, 0) * a.ldq, sub);
        float s[MAXN], m = -INFINITY, z = 0.f, top = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.f;
        auto scores = [&](auto far) {
#pragma unroll
            for (int j = 0; j < MAXN; ++j) {
                s[j] = -INFINITY;
                if (j < 3 || most > 3) {
                    float dot = row[j].dot(q);
#pragma unroll
                    for (int o = LPH / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    if (j < cnt) s[j] = q.template score<decltype(far)::value>(dot, row[j].k_scale(row[j].pair));
                }
                if (j == 0 && cnt <= 1) s[0] = 0.f;                           // softmax over one member: weight exactly 1
                m = fmaxf(m, s[j]);
            }
        };
        scores(std::false_type());
        if (__any_sync(0xffffffffu, q.is_far())) {
            m = -INFINITY;
            scores(std::true_type());
        }
#pragma unroll
        for (int j = 0; j < MAXN; ++j) {
            const float p = fast_exp2(s[j] - m);
            z += p;
            s[j] = p * row[j].v_scale(row[j].pair);                           // from here on the weight on the codes
            top = fmaxf(top, s[j]);
        }
        const uint32_t b = BF16 ? lift(top) : 127u;
        const float up = __uint_as_float(b << 23), down = 0.5f * __uint_as_float((254u - b) << 23);
#pragma unroll
        for (int j = 0; j < MAXN; ++j) {
            if (j < most) row[j].add(BF16 ? s[j] * up : s[j], acc);
            const int u = j ? __shfl_sync(0xffffffffu, pad1, grp + j) : max(v1, 0);
            if (more) row[j].load(codes, exps, (uint32_t)u, a.ldt);
        }
        const float inv = cnt <= 1 ? 1.f : fast_rcp(z);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = BF16 ? acc[e] * inv * down : acc[e] * inv;
        if (v >= 0) store_row<BF16, LANES>((char*)a.O + (int64_t)v * a.ldo, sub, acc);
        v = v1; pad = pad1;
        v1 = v2; pad1 = pad2;
    }
}

// Wider cones (3 to 8 hops, lists of up to 511 members): one warp per node, its groups of LANES lanes take alternate
// members, UN in flight each; online softmax (running maximum and sum in 32 bits) per group, merged at the end.
// For bf16 rows the sums are measured against a running reference of their own, mw: the largest logarithm of a weight on
// the codes, which is put at 14.  These logarithms, score - m + log2(V scale), are relative to the scores' maximum m: so,
// however large the scores are, they are numbers of a few hundred wherever a weight matters, and what their rounding does
// (2^-17 in the exponent) is far below that of the fp16 weights.  (Against scores of 10^6 themselves an exponent would be
// off by 2^-5.)
// The loads run ahead of the arithmetic: the next batch of members (of this node, or the first one of the next node)
// goes into the registers of the present one as soon as that has been added up, the member ids a chunk of 32 ahead.
template <bool BF16, int LANES, int LPH>
__global__ void __launch_bounds__(256, 2) sparse_attn_kv8_wide_kernel(AttnArgs a) {
    constexpr int GROUPS = 32 / LANES, UN = 4, BATCH = GROUPS * UN, N = Row<BF16, LANES>::kN;
    static_assert(32 % BATCH == 0, "a batch lies in one chunk of member ids");
    const int lane = threadIdx.x & 31, sub = lane & (LANES - 1), grp = lane / LANES;
    const uint32_t warps = gridDim.x * (blockDim.x >> 5);
    const uint8_t* codes = a.T + sub * (256 / LANES);
    const uint8_t* exps = a.T + kCodeBytes + 2 * (sub / LPH);
    uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    // the node after next: id (-1: none), list bounds, first 32 members
    int v1 = -1, beg1 = 0, cnt1 = 0, u1 = 0;
    auto fetch = [&]() {
        v1 = -1;
        for (; slot < (uint32_t)a.count && v1 < 0; slot += warps) {
            const int v = a.nodes ? a.nodes[slot] : (int)slot;
            if ((uint32_t)v < (uint32_t)a.n) v1 = v;                          // ids outside the graph are skipped
        }
        if (v1 >= 0) {
            beg1 = a.nbr_ptr[v1];
            cnt1 = a.nbr_ptr[v1 + 1] - beg1;
            u1 = lane < cnt1 ? a.nbr_idx[beg1 + lane] : 0;
        }
    };
    // exp2(x - ref) where ref = -inf stands for "nothing seen yet": measured against 0 then, so that scores of -inf
    // weigh nothing instead of inf - inf
    auto finite = [](float ref) { return ref == -INFINITY ? 0.f : ref; };
    Row<BF16, LANES> row[UN];
    RawRow<BF16, LANES> raw;
    fetch();
    int v = v1, beg = beg1, cnt = cnt1, ids = u1;                             // ids: the chunk of 32 members being read
    if (v < 0) return;
    raw.load((const char*)a.Q + (int64_t)v * a.ldq, sub);
    // members past the end are stood in for by the last one, which is not added again
#pragma unroll
    for (int i = 0; i < UN; ++i)
        row[i].load(codes, exps, (uint32_t)__shfl_sync(0xffffffffu, ids, min(GROUPS * i + grp, min(cnt, 32) - 1)), a.ldt);
    fetch();
    while (v >= 0) {
        float acc[N], m = -INFINITY, mw = -INFINITY, z = 0.f;
        raw.unpack(acc);
        Query<BF16, LANES> q;
        q.template set<LPH>(acc, a.c);
        if (v1 >= 0) raw.load((const char*)a.Q + (int64_t)v1 * a.ldq, sub);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.f;
        const bool far = __any_sync(0xffffffffu, q.is_far());
        int ids_next = 32 + lane < cnt ? a.nbr_idx[beg + 32 + lane] : 0;      // the chunk after `ids`
        for (int t = 0; t < cnt; t += BATCH) {
            float s[UN], m_new = m;
            auto scores = [&](auto far) {
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    float dot = row[i].dot(q);
#pragma unroll
                    for (int o = LPH / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    dot = q.template score<decltype(far)::value>(dot, row[i].k_scale(row[i].pair));
                    s[i] = t + GROUPS * i + grp < cnt ? dot : -INFINITY;
                    if (i == 0 && cnt == 1 && grp == 0) s[0] = 0.f;           // softmax over one member: weight exactly 1
                    m_new = fmaxf(m_new, s[i]);
                }
            };
            scores(std::false_type());
            if (far) {
                m_new = m;
                scores(std::true_type());
            }
            const float ref = finite(m_new), shift = m - ref, keep = fast_exp2(shift);       // one rescale per batch; 0 for the first
            mw += shift;
            float lw[UN], mw_new = mw;
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                s[i] -= ref;
                if (BF16) mw_new = fmaxf(mw_new, lw[i] = s[i] + log2_scale_v(row[i].pair));
            }
            const float ref_w = finite(mw_new), keep_w = BF16 ? fast_exp2(mw - ref_w) : keep;
            z *= keep;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] *= keep_w;
            m = m_new;
            mw = mw_new;
            // where the next batch comes from
            int next = t + BATCH, from = ids, left = cnt;
            const bool same = next < cnt;
            if (same) {
                if ((next & 31) == 0) {
                    from = ids = ids_next;
                    ids_next = next + 32 + lane < cnt ? a.nbr_idx[beg + next + 32 + lane] : 0;
                }
                left = cnt - (next & ~31);
            } else {
                from = u1;
                left = cnt1;
                next = 0;
            }
            const bool more = same || v1 >= 0;
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                const float p = fast_exp2(s[i]);
                z += p;
                const float w = BF16 ? fast_exp2(lw[i] - (ref_w - 14.f)) : p * scale_v(row[i].pair);
                if (t + GROUPS * i + grp < cnt) row[i].add(w, acc);
                const int u = __shfl_sync(0xffffffffu, from, min((next & 31) + GROUPS * i + grp, min(left, 32) - 1) & 31);
                if (more) row[i].load(codes, exps, (uint32_t)u, a.ldt);
            }
        }
        // merge the groups: maxima first, then the sums, of which each step gives one half away and keeps the other, so
        // that a lane ends with the four elements it stores (101 000 nodes, cones of five hops: 168 us, fp32
        // rows 190; with all sums exchanged at both steps 181)
        float mm = m;
#pragma unroll
        for (int o = LANES; o < 32; o <<= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, o));
        const float shift = m - finite(mm), fit_z = fast_exp2(shift);
        mw += shift;
        float mmw = mw;
#pragma unroll
        for (int o = LANES; o < 32; o <<= 1) mmw = fmaxf(mmw, __shfl_xor_sync(0xffffffffu, mmw, o));
        const float fit = BF16 ? fast_exp2(mw - finite(mmw)) : fit_z;
        z *= fit_z;
#pragma unroll
        for (int o = LANES; o < 32; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] *= fit;
        int width = N;
#pragma unroll
        for (int o = 16; o >= LANES; o >>= 1) {
            width /= 2;
            const bool high = (lane & o) != 0;
#pragma unroll
            for (int e = 0; e < N / 2; ++e) {
                if (e < width) {
                    const float give = high ? acc[e] : acc[e + width], keep = high ? acc[e + width] : acc[e];
                    acc[e] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
        }
        // what stood at 14 goes back: a power of two up to some 2^150, put on in two halves
        const float inv = fast_rcp(z), half = BF16 ? fast_exp2(0.5f * (finite(mmw) - 14.f)) : 1.f;
        static_assert(N / GROUPS == 4, "a lane keeps four elements");
        float out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = BF16 ? acc[e] * half * inv * half : acc[e] * inv;
        // element offset of what is kept: bit 4 of the lane chose the half of N, the next bit the half of that
        int first = sub * N;
        if (LANES == 8) first += ((lane >> 4) & 1) * (N / 2) + ((lane >> 3) & 1) * (N / 4);
        else first += ((lane >> 4) & 1) * (N / 2);
        char* o_row = (char*)a.O + (int64_t)v * a.ldo;
        if (BF16) {
            const __nv_bfloat162 x = __floats2bfloat162_rn(out[0], out[1]), y = __floats2bfloat162_rn(out[2], out[3]);
            asm volatile("st.global.cs.v2.u32 [%0], {%1,%2};" ::"l"(o_row + first * 2), "r"(*reinterpret_cast<const uint32_t*>(&x)), "r"(*reinterpret_cast<const uint32_t*>(&y)) : "memory");
        } else {
            st_piece_stream(o_row + first * 4, Elem<false>::pack(out));
        }
        v = v1; beg = beg1; cnt = cnt1; ids = u1;
        fetch();
    }
}

// ---------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------
#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

template <auto kKernel, typename Args>
dg4_status launch(const Args& args, int64_t per_block, cudaStream_t st) {
    int resident;
    CHECK(dg4i_resident_blocks<kKernel>(256, &resident));
    const int64_t needed = ((int64_t)args.count + per_block - 1) / per_block;
    kKernel<<<(unsigned)(needed < resident ? needed : resident), 256, 0, st>>>(args);
    dg4i_count_launch();
    DG4_CUDA_TRY(cudaGetLastError());
    return DG4_OK;
}

dg4_status check_table(const dg4_desc* d, const void* T, int64_t ldt) {
    if (d->heads > 16) DG4_FAIL(DG4_ERR_UNSUPPORTED, "heads = %d: the 8-bit table has at most 16", d->heads);
    if (ldt > 0x7fffffff) DG4_FAIL(DG4_ERR_UNSUPPORTED, "the table's rows are %lld bytes apart: 2^31 - 1 at most", (long long)ldt);
    CHECK(dg4i_check_tensor("T", T, ldt, 1, DG4_KV8_ROW_BYTES));
    if ((((uintptr_t)T) | (uintptr_t)ldt) & 31u) DG4_FAIL(DG4_ERR_INVALID_ARG, "the table or its row distance is not a multiple of 32 bytes");
    return DG4_OK;
}

dg4_status check_nodes(const dg4_graph* g, const int32_t* nodes, int32_t count) {
    if (count < 0) DG4_FAIL(DG4_ERR_INVALID_ARG, "the number of nodes (%d) is negative", count);
    if (nodes && ((uintptr_t)nodes & 3u)) DG4_FAIL(DG4_ERR_INVALID_ARG, "the node list is not 4-byte aligned");
    if (!nodes && count != 0 && count != g->n)
        DG4_FAIL(DG4_ERR_INVALID_ARG, "%d nodes but no list of them: 0 or the graph's %d are possible", count, g->n);
    return DG4_OK;
}

#define DG4_KV8_HEADS(LAUNCH, BF16, ...)                                                     \
    switch (16 / desc->heads) {                                                              \
        case 1: return LAUNCH(BF16, 1, ##__VA_ARGS__);                                       \
        case 2: return LAUNCH(BF16, 2, ##__VA_ARGS__);                                       \
        case 4: return LAUNCH(BF16, 4, ##__VA_ARGS__);                                       \
        case 8: return LAUNCH(BF16, 8, ##__VA_ARGS__);                                       \
        default: return LAUNCH(BF16, 16, ##__VA_ARGS__);                                     \
    }

#define WRITE(BF16, LPH) launch<kv8_write_kernel<BF16, LPH>>(a, 256 / kLanes, st)
#define READ(BF16, LPH) launch<kv8_read_kernel<BF16, LPH>>(a, 256 / kLanes, st)
// LPH counts lanes of 8 elements: with two pieces per lane a head spans half as many
#define ATTN(BF16, LPH, MAXN) \
    launch<sparse_attn_kv8_kernel<BF16, LPH == 1 ? 16 : 8, LPH == 1 ? 1 : LPH / 2, MAXN>>(a, LPH == 1 ? 16 : 32, st)
#define ATTN_WIDE(BF16, LPH) launch<sparse_attn_kv8_wide_kernel<BF16, LPH == 1 ? 16 : 8, LPH == 1 ? 1 : LPH / 2>>(a, 8, st)

dg4_status copy_call(const dg4_graph* g, const dg4_desc* desc, const void* K, int64_t ldk, const void* V, int64_t ldv,
                     const void* T, int64_t ldt, const int32_t* nodes, int32_t count, bool write, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, false));
    CHECK(check_table(desc, T, ldt));
    const int es = desc->dtype == DG4_BF16 ? 2 : 4;
    CHECK(dg4i_check_tensor("K", K, ldk, es, 128));
    CHECK(dg4i_check_tensor("V", V, ldv, es, 128));
    CHECK(check_nodes(g, nodes, count));
    CopyArgs a;
    a.K = const_cast<void*>(K); a.ldk = ldk * es;
    a.V = const_cast<void*>(V); a.ldv = ldv * es;
    a.T = (uint8_t*)const_cast<void*>(T); a.ldt = ldt;
    a.nodes = nodes; a.count = nodes ? count : g->n; a.n = g->n;
    a.wide = (((uintptr_t)K | (uintptr_t)V | (uintptr_t)a.ldk | (uintptr_t)a.ldv) & 31u) == 0;
    if (a.count == 0) return DG4_OK;
    const cudaStream_t st = (cudaStream_t)stream;
    if (write) {
        if (es == 2) { DG4_KV8_HEADS(WRITE, true) }
        DG4_KV8_HEADS(WRITE, false)
    }
    if (es == 2) { DG4_KV8_HEADS(READ, true) }
    DG4_KV8_HEADS(READ, false)
}

}  // namespace

extern "C" dg4_status dg4_kv8_write(const dg4_graph* g, const dg4_desc* desc, const void* K, int64_t ldk, const void* V,
                                    int64_t ldv, void* T, int64_t ldt, const int32_t* nodes, int32_t count,
                                    void* stream) {
    return copy_call(g, desc, K, ldk, V, ldv, T, ldt, nodes, count, true, stream);
}

extern "C" dg4_status dg4_kv8_read(const dg4_graph* g, const dg4_desc* desc, const void* T, int64_t ldt, void* K,
                                   int64_t ldk, void* V, int64_t ldv, const int32_t* nodes, int32_t count,
                                   void* stream) {
    return copy_call(g, desc, K, ldk, V, ldv, T, ldt, nodes, count, false, stream);
}

extern "C" dg4_status dg4_sparse_attn_kv8_fwd(const dg4_graph* g, const dg4_desc* desc, const void* Q, int64_t ldq,
                                              const void* T, int64_t ldt, void* O, int64_t ldo, const int32_t* nodes,
                                              int32_t count, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, false));
    CHECK(check_table(desc, T, ldt));
    const int es = desc->dtype == DG4_BF16 ? 2 : 4;
    CHECK(dg4i_check_tensor("Q", Q, ldq, es, 128));
    CHECK(dg4i_check_tensor("O", O, ldo, es, 128));
    CHECK(check_nodes(g, nodes, count));
    if (nodes && O == Q) DG4_FAIL(DG4_ERR_INVALID_ARG, "O may not be Q for a list of nodes (one that is named twice would be read after it was written)");
    AttnArgs a;
    a.Q = Q; a.ldq = ldq * es; a.T = (const uint8_t*)T; a.ldt = (uint32_t)ldt; a.O = O; a.ldo = ldo * es;
    a.nodes = nodes; a.count = nodes ? count : g->n; a.n = g->n;
    a.nbr_pad = g->nbr_pad; a.nbr_ptr = g->nbr_ptr; a.nbr_idx = g->nbr_idx;
    a.c = desc->scale * 1.4426950408889634f;
    if (a.count == 0) return DG4_OK;
    const cudaStream_t st = (cudaStream_t)stream;
    if (g->wide) {
        if (es == 2) { DG4_KV8_HEADS(ATTN_WIDE, true) }
        DG4_KV8_HEADS(ATTN_WIDE, false)
    }
    if (g->max_class <= 3) {
        if (es == 2) { DG4_KV8_HEADS(ATTN, true, 3) }
        DG4_KV8_HEADS(ATTN, false, 3)
    }
    if (es == 2) { DG4_KV8_HEADS(ATTN, true, 7) }
    DG4_KV8_HEADS(ATTN, false, 7)
}
