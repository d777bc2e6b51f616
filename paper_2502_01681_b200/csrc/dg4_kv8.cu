// The 8-bit K | V table: writing rows, reading them back, and sparse attention over it.
//
// All three are bound by memory, so each row passes through registers once: 16 lanes per row (two rows per warp),
// 8 elements of K and of V per lane (see dg4_kv8_core.cuh for the row).  A written row costs 512 + 288 bytes in
// bf16; a gathered neighbour costs 288 bytes instead of 512.

#include "dg4_internal.h"
#include "dg4_kv8_core.cuh"

namespace {

using namespace attn;
using namespace kv8;

struct CopyArgs {
    void* K; int64_t ldk;              // bytes
    void* V; int64_t ldv;
    uint8_t* T; int64_t ldt;
    const int32_t* nodes;              // nullable
    int32_t count, n, heads;
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

template <bool BF16, int LPH>
__global__ void __launch_bounds__(256) kv8_write_kernel(CopyArgs a) {
    const int lane = threadIdx.x & 31, sub = lane & 15, grp = lane - sub;
    const unsigned mask = 0xffffu << grp;
    const uint32_t stride = gridDim.x * (blockDim.x / kLanes);
    for (uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) / kLanes; slot < (uint32_t)a.count; slot += stride) {
        const int v = a.nodes ? a.nodes[slot] : (int)slot;
        if ((uint32_t)v >= (uint32_t)a.n) continue;                 // ids outside the table are skipped
        float k[kEl], w[kEl];
        load8<BF16>((const char*)a.K + (int64_t)v * a.ldk, sub, k);
        load8<BF16>((const char*)a.V + (int64_t)v * a.ldv, sub, w);
        const uint32_t bk = scale_byte(slice_top<LPH>(k, mask)), bv = scale_byte(slice_top<LPH>(w, mask));
        Piece p;
        encode8(k, bk, p.w);
        encode8(w, bv, p.w + 2);
        uint8_t* row = a.T + (int64_t)v * a.ldt;
        *reinterpret_cast<Piece*>(row + sub * 16) = p;
        // lane l writes the pair of head l (held by the lanes of that head), the lanes beyond the heads write zero
        const uint32_t mine = bk | (bv << 8);
        const uint32_t pair = __shfl_sync(mask, mine, grp + ((sub * LPH) & 15));
        *reinterpret_cast<uint16_t*>(row + kCodeBytes + 2 * sub) = (uint16_t)(sub < 16 / LPH ? pair : 0u);
    }
}

template <bool BF16, int LPH>
__global__ void __launch_bounds__(256) kv8_read_kernel(CopyArgs a) {
    const int sub = threadIdx.x & 15;
    const uint32_t stride = gridDim.x * (blockDim.x / kLanes);
    for (uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) / kLanes; slot < (uint32_t)a.count; slot += stride) {
        const int v = a.nodes ? a.nodes[slot] : (int)slot;
        if ((uint32_t)v >= (uint32_t)a.n) continue;
        const uint8_t* row = a.T + (int64_t)v * a.ldt;
        const Piece p = ld_piece_stream(row + sub * 16);
        const uint32_t pair = ld_pair(row + kCodeBytes + 2 * (sub / LPH));
        const float sk = scale_of(pair & 255u), sv = scale_of(pair >> 8);
        float k[kEl], w[kEl];
        decode4(p.w[0], k); decode4(p.w[1], k + 4);
        decode4(p.w[2], w); decode4(p.w[3], w + 4);
#pragma unroll
        for (int i = 0; i < kEl; ++i) { k[i] *= sk; w[i] *= sv; }
        store8<BF16>((char*)a.K + (int64_t)v * a.ldk, sub, k);
        store8<BF16>((char*)a.V + (int64_t)v * a.ldv, sub, w);
    }
}

struct AttnArgs {
    const void* Q; int64_t ldq;        // bytes
    const uint8_t* T; int64_t ldt;
    void* O; int64_t ldo;
    const int32_t* nodes;              // nullable
    const int32_t* nbr_pad;            // fixed-width lists (two hops at most)
    const int32_t* nbr_ptr;            // CSR lists (wider cones)
    const int32_t* nbr_idx;
    int32_t count, n;
    float c;                           // scale * log2(e): scores are kept in log2 units
};

// q . (8 codes); the sum over a head's lanes and the slice's scale follow
__device__ __forceinline__ float dot8(const float* q, const Piece& p) {
    float k[kEl], acc = 0.f;
    decode4(p.w[0], k); decode4(p.w[1], k + 4);
#pragma unroll
    for (int i = 0; i < kEl; ++i) acc = fmaf(q[i], k[i], acc);
    return acc;
}
__device__ __forceinline__ void add8(float weight, const Piece& p, float* acc) {
    float w[kEl];
    decode4(p.w[2], w); decode4(p.w[3], w + 4);
#pragma unroll
    for (int i = 0; i < kEl; ++i) acc[i] = fmaf(weight, w[i], acc[i]);
}

// Lists of at most MAXN members from the fixed-width table; the walk and the prefetch of the next node's list are
// those of the 16-bit kernel (dg4_attn.cu).
template <bool BF16, int LPH, int MAXN>
__global__ void __launch_bounds__(256, 3) sparse_attn_kv8_kernel(AttnArgs a) {
    constexpr int W = MAXN + 1;
    const int lane = threadIdx.x & 31, sub = lane & 15, grp = lane - sub;
    const unsigned mask = 0xffffu << grp;
    const uint32_t stride = gridDim.x * (blockDim.x / kLanes);
    uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) / kLanes;
    int v_next = -1, pad_next = 0;
    if (slot < (uint32_t)a.count) {
        v_next = a.nodes ? a.nodes[slot] : (int)slot;
        if (sub < W && (uint32_t)v_next < (uint32_t)a.n) pad_next = a.nbr_pad[(size_t)v_next * W + sub];
    }
    for (; slot < (uint32_t)a.count; slot += stride) {
        const int v = v_next, pad = pad_next;
        {
            const uint32_t s2 = slot + stride;
            if (s2 < (uint32_t)a.count) {
                v_next = a.nodes ? a.nodes[s2] : (int)s2;
                if (sub < W && (uint32_t)v_next < (uint32_t)a.n) pad_next = a.nbr_pad[(size_t)v_next * W + sub];
            }
        }
        if ((uint32_t)v >= (uint32_t)a.n) continue;                 // ids outside the graph are skipped
        const int cnt = __shfl_sync(mask, pad, grp);
        Piece kv[MAXN];
        uint32_t pair[MAXN];
        int u[MAXN];
        u[0] = v;
#pragma unroll
        for (int j = 1; j < MAXN; ++j) u[j] = __shfl_sync(mask, pad, grp + j);
        float q[kEl];
        load8<BF16>((const char*)a.Q + (int64_t)v * a.ldq, sub, q);
        // the filler of a list repeats v, so every slot names a valid row and the loads need no predicate
#pragma unroll
        for (int j = 0; j < MAXN; ++j) {
            const uint8_t* row = a.T + (int64_t)u[j] * a.ldt;
            kv[j] = ld_piece_nc(row + sub * 16);
            pair[j] = ld_pair(row + kCodeBytes + 2 * (sub / LPH));
        }
        float acc[kEl];
#pragma unroll
        for (int i = 0; i < kEl; ++i) acc[i] = 0.f;
        if (cnt <= 1) {                                             // softmax over one member: weight exactly 1
            add8(scale_of(pair[0] >> 8), kv[0], acc);
        } else {
            float s[MAXN], m = -INFINITY, z = 0.f;
#pragma unroll
            for (int j = 0; j < MAXN; ++j) {
                float dot = j < cnt ? dot8(q, kv[j]) : 0.f;
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(mask, dot, o);
                s[j] = j < cnt ? dot * scale_of(pair[j] & 255u) * a.c : -INFINITY;
                m = fmaxf(m, s[j]);
            }
#pragma unroll
            for (int j = 0; j < MAXN; ++j) {
                if (j < cnt) {
                    const float p = fast_exp2(s[j] - m);
                    z += p;
                    add8(p * scale_of(pair[j] >> 8), kv[j], acc);
                }
            }
            const float inv = fast_rcp(z);
#pragma unroll
            for (int i = 0; i < kEl; ++i) acc[i] *= inv;
        }
        store8<BF16>((char*)a.O + (int64_t)v * a.ldo, sub, acc);
    }
}

// Wider cones (3 to 8 hops, lists of up to 511 members): one warp per node, the half-warps take alternate members,
// four in flight each; online softmax (running maximum and sum in 32 bits) per half, merged at the end.
template <bool BF16, int LPH>
__global__ void __launch_bounds__(256, 3) sparse_attn_kv8_wide_kernel(AttnArgs a) {
    constexpr int UN = 4;
    const int lane = threadIdx.x & 31, sub = lane & 15, half = lane >> 4;
    const unsigned hmask = 0xffffu << (lane - sub);
    const uint32_t warps = gridDim.x * (blockDim.x >> 5);
    for (uint32_t slot = (blockIdx.x * blockDim.x + threadIdx.x) >> 5; slot < (uint32_t)a.count; slot += warps) {
        const int v = a.nodes ? a.nodes[slot] : (int)slot;
        if ((uint32_t)v >= (uint32_t)a.n) continue;
        const int beg = a.nbr_ptr[v];
        const int cnt = a.nbr_ptr[v + 1] - beg;
        float q[kEl], acc[kEl], m = -INFINITY, z = 0.f;
        load8<BF16>((const char*)a.Q + (int64_t)v * a.ldq, sub, q);
#pragma unroll
        for (int i = 0; i < kEl; ++i) acc[i] = 0.f;
        for (int base = 0; base < cnt; base += 32) {
            const int my_u = base + lane < cnt ? a.nbr_idx[beg + base + lane] : -1;
            const int chunk = cnt - base < 32 ? cnt - base : 32;
            for (int t = 0; t < chunk; t += 2 * UN) {
                Piece kv[UN];
                uint32_t pair[UN];
                float s[UN], m_new = m;
                int u[UN];
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    const int j = t + 2 * i + half;
                    u[i] = __shfl_sync(0xffffffffu, my_u, j & 31);
                    if (j >= chunk) u[i] = -1;
                }
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    if (u[i] >= 0) {
                        const uint8_t* row = a.T + (int64_t)u[i] * a.ldt;
                        kv[i] = ld_piece_nc(row + sub * 16);
                        pair[i] = ld_pair(row + kCodeBytes + 2 * (sub / LPH));
                    }
                }
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    float dot = u[i] >= 0 ? dot8(q, kv[i]) : 0.f;
#pragma unroll
                    for (int o = LPH / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(hmask, dot, o);
                    s[i] = u[i] >= 0 ? dot * scale_of(pair[i] & 255u) * a.c : -INFINITY;
                    m_new = fmaxf(m_new, s[i]);
                }
                if (u[0] >= 0) {                                    // a batch's first slot is its lowest position
                    // scores of -inf alone: measured against 0 they weigh nothing, instead of inf - inf
                    const float ref = m_new == -INFINITY ? 0.f : m_new;
                    const float keep = fast_exp2(m - ref);          // 0 for the first batch
                    z *= keep;
#pragma unroll
                    for (int e = 0; e < kEl; ++e) acc[e] *= keep;
#pragma unroll
                    for (int i = 0; i < UN; ++i) {
                        if (u[i] >= 0) {
                            const float p = fast_exp2(s[i] - ref);
                            z += p;
                            add8(p * scale_of(pair[i] >> 8), kv[i], acc);
                        }
                    }
                    m = m_new;
                }
            }
        }
        const float m2 = __shfl_xor_sync(0xffffffffu, m, 16), z2 = __shfl_xor_sync(0xffffffffu, z, 16);
        const float mm = fmaxf(m, m2);
        const float w1 = m == -INFINITY ? 0.f : fast_exp2(m - mm), w2 = m2 == -INFINITY ? 0.f : fast_exp2(m2 - mm);
        const float inv = cnt == 1 ? 1.f : fast_rcp(z * w1 + z2 * w2);
#pragma unroll
        for (int e = 0; e < kEl; ++e) acc[e] = (acc[e] * w1 + __shfl_xor_sync(0xffffffffu, acc[e], 16) * w2) * inv;
        if (half == 0) store8<BF16>((char*)a.O + (int64_t)v * a.ldo, sub, acc);
    }
}

// ---------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------
#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

// grid: as many blocks as the work needs, at most what the device holds at once
template <typename Kernel, typename Args>
dg4_status launch(Kernel kernel, const Args& args, int64_t per_block, cudaStream_t st) {
    int dev = 0, sms = 0, per_sm = 0;
    DG4_CUDA_TRY(cudaGetDevice(&dev));
    DG4_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    DG4_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, 256, 0));
    const int64_t needed = ((int64_t)args.count + per_block - 1) / per_block;
    const int64_t resident = (int64_t)sms * (per_sm > 0 ? per_sm : 1);
    kernel<<<(unsigned)(needed < resident ? needed : resident), 256, 0, st>>>(args);
    dg4i_count_launch();
    DG4_CUDA_TRY(cudaGetLastError());
    return DG4_OK;
}

dg4_status check_table(const dg4_desc* d, const void* T, int64_t ldt) {
    if (d->heads > 16) DG4_FAIL(DG4_ERR_UNSUPPORTED, "heads = %d: the 8-bit table has at most 16", d->heads);
    return dg4i_check_tensor("T", T, ldt, 1, DG4_KV8_ROW_BYTES);
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

#define WRITE(BF16, LPH) launch(kv8_write_kernel<BF16, LPH>, a, 256 / kLanes, st)
#define READ(BF16, LPH) launch(kv8_read_kernel<BF16, LPH>, a, 256 / kLanes, st)
#define ATTN(BF16, LPH, MAXN) launch(sparse_attn_kv8_kernel<BF16, LPH, MAXN>, a, 256 / kLanes, st)
#define ATTN_WIDE(BF16, LPH) launch(sparse_attn_kv8_wide_kernel<BF16, LPH>, a, 256 / 32, st)

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
    a.nodes = nodes; a.count = nodes ? count : g->n; a.n = g->n; a.heads = desc->heads;
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
    a.Q = Q; a.ldq = ldq * es; a.T = (const uint8_t*)T; a.ldt = ldt; a.O = O; a.ldo = ldo * es;
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
