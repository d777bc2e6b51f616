// Shared projection with a low-rank adapter per request, on the 5th-generation tensor cores:
//     Y = X W^T + U B_a^T (+ residual),    U = bf16(scale_a * X A_a^T),
// K = 128, bf16 operands, fp32 accumulation in tensor memory.  U's rounding is that of any tensor-core operand: it
// perturbs the adapter's contribution by at most 2^-8 of itself, as the rounding of y does to y.
//
// The work is cut into items: up to 128 consecutive rows of ONE request.  An item multiplies with its own adapter only,
// and only its own rows are stored, so nothing is masked and no request's infinities or NaNs can meet another's rows
// (0 * inf in a masked product would).  Each CTA takes a contiguous run of items, so neighbouring items mostly share
// their adapter, which is fetched into shared memory only when it changes.
//
// One persistent CTA per SM, fourteen warps:
//   warp 0       producer: W once, the item's rows of X by TMA, the adapter when it changes, the residual's rows (on a
//                barrier of their own: their buffer comes back from the epilogue, later than X's from the products); it
//                alone walks the requests and passes each item on in a small ring of descriptors;
//   warp 1       owns tensor memory, issues tcgen05.mma: U and the first 128-column block as one product; once U stands
//                in tensor memory as bf16, U B^T on top of the block (A operand from tensor memory); with three blocks
//                the other two as one 256-column product, in the same two steps;
//   warps 2-9    epilogue: each owns 32 rows x 64 columns of a block; tensor memory -> bf16 -> its own 4 KB of
//                staging -> TMA store, or 16-byte stores where the item ends inside the 32 rows;
//   warps 10-13  U: tensor memory -> * scale -> bf16 -> tensor memory, while other products run.
// One block per CTA (the output projection): the next item's first product goes before this item's second one, which
// waits for U.  Few items (decoding: one row per request): an item's three column blocks go to different CTAs, two to an
// SM, so that each fetches a third of W and has one block's epilogue.
//
// Bound by HBM, and under sustained load by power: a QKV row is 256 bytes in, 768 out, and 98 + r kflop.  1.01M rows,
// rank 16, 200 requests: 190 us = 5.5 TB/s (84 % of the measured copy rate; the plain projection takes 185) in short runs,
// sustained 195 us, the SM clock falling from 1.97 to 1.5 GHz at 1 kW.  That is why the waits are suspended ones and the products
// few and wide: a product of N columns reads the same 128 rows of X from shared memory whatever N is, so U apart and
// three blocks apart (36 instructions of N <= 128 per item instead of 19) took 219 us.  Rank 64: 237 us (sustained 248), one X stage
// beside W_qkv (rows stored from registers, without staging, made room for two and took 400).  Output projection with
// residual, rank 64: 129 us = 6.0 TB/s, sustained 131 to 137.  64 requests of one row each: 7.6 us on the device, 9.4 us a
// call through the binding; 512 of them 14, 2 048 of them 37 on the device.
//
// Every mbarrier wait is bounded.  On expiry the kernel records DG4_ERR_TIMEOUT and raises an abort flag; every warp
// leaves at its next item at the latest, without meeting others.  Then the producer waits for the copies it has started,
// the MMA thread for its MMAs, the storing lanes for their stores, and only then is tensor memory freed.

#include "dg4_internal.h"
#include "dg4_sm100.cuh"

#include <atomic>

namespace {

using namespace sm100;

constexpr int kEpiWarps = 8, kUWarps = 4;
constexpr int kThreads = 32 * (2 + kEpiWarps + kUWarps);
constexpr int kTileM = 128;
constexpr int kHalfBytes = 128 * 128;             // a 128-row x 64-column bf16 box
constexpr int kTileBytes = 2 * kHalfBytes;
constexpr int kMaxStages = 2;
constexpr int kSlots = 3;                         // accumulators of 128 columns, at most
constexpr int kRing = 4;                          // item descriptors in flight
constexpr int kUTurns = 2;                        // barriers that announce U's product, in turn
constexpr int kRankMax = 64;

// Where things lie, for ranks up to RANK = 32 or 64 and NB = 3 or 1 column blocks per CTA.
// Shared memory: the rows of A_a stand directly in front of those of W in each half of K (128-byte rows, 128-byte
// swizzle), so ONE product makes U and the first column block: X is read once for both, and its N (128 + the rank) costs
// little more than 128.  B_a per column block 128 rows of RANK columns (128-byte or 64-byte swizzle; the columns past
// the rank are zero).
// Tensor memory: U (fp32) directly in front of the first block's accumulator, accordingly.  With NB = 1 that pair stands
// there two or three times, so that the next item's product need not wait for this one's second product.
template <int RANK, int NB> struct Place {
    static constexpr int kB = 128 * RANK * 2;
    static constexpr int kSets = NB == 3 ? 1 : RANK == 64 ? 2 : 3;      // at most (few requests: one)
    static constexpr int kSetCols = RANK + 128;
    static constexpr int kColUb = NB == 3 ? 448 : kSets * kSetCols;     // U in bf16: RANK / 2 columns
    static_assert(RANK + NB * 128 <= 448 && kColUb + RANK / 2 <= 512, "tensor memory columns");
    static_assert(kSetCols + RANK / 2 <= 256, "tensor memory columns of a CTA with one set");
    __device__ static __forceinline__ uint64_t b_desc(uint32_t addr) { return RANK == 64 ? smem_desc_sw128(addr) : smem_desc_sw64(addr); }
};

struct Item {
    int32_t row0, rows;
    int32_t adapter;          // -1: none
    int32_t last;             // the next item uses another adapter (or there is none)
};

// The walk over the items of a CTA, one request after the other (the producer's state).
struct Walk { int32_t seg, lo, hi, adapter; };

struct Bars {
    uint64_t w_full;
    uint64_t a_full[kMaxStages];
    uint64_t a_empty[kMaxStages];
    uint64_t r_full[kMaxStages], r_empty[kMaxStages];
    uint64_t acc_full[kSlots];
    uint64_t acc_empty[kSlots];
    uint64_t la_full, la_empty;     // A_a in shared memory (read by the first product)
    uint64_t lb_full, lb_empty;     // B_a in shared memory (read by the second one)
    // U's product is done.  With one block per CTA the next item's is committed before this item's U is waited for: on
    // one barrier a U warp that comes late for this item would find it two phases on and, by the parity, not yet done.
    // In turn, the commit after next follows the wait for this item's U, which every U warp has passed its wait for.
    uint64_t u_full[kUTurns];
    uint64_t u_ready, ub_empty;
    uint64_t item_full[kRing], item_empty[kRing];
    uint64_t drain;
    uint32_t tmem_base;
    uint32_t abort_flag;
    int32_t my_items;               // items of this CTA, and where they begin
    Walk first;
    int64_t warp_sum[kThreads / 32];
    Item ring[kRing];
};

struct Params {
    const int32_t* seg_ptr;         // nullable: one request over all rows
    const int32_t* seg_id;
    const float* scale;
    __nv_bfloat16* out[3]; int64_t ldo[3];
    int32_t n, n_seg, n_adapters, rank;
    int32_t n_out;                  // rows of W
    int32_t stages;                 // X (and residual) stages
    int32_t slots;                  // accumulators: 3 (NB = 3), or the number of sets (one: 256 columns of tensor memory)
    int32_t col_ub;
    int32_t off_b, off_x, off_r, off_stage, off_bar;
    int32_t has_res;
    int32_t* status;
    uint32_t poll_limit;
};

struct OutMaps { CUtensorMap m[3]; };

__device__ __forceinline__ void st_shared_v4(uint32_t addr, const uint32_t* r) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void ld_shared_v4(uint32_t addr, uint32_t* r) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void st_global_v4(void* p, const uint32_t* r) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ void raise_timeout(Bars* bars, int32_t* status) {
    atomicExch(&bars->abort_flag, 1u);
    if (status) atomicCAS(status, 0, (int)DG4_ERR_TIMEOUT);
}

// rows of request s, cut to the tensor: whatever the offsets hold, 0 <= lo <= hi <= n
__device__ __forceinline__ void seg_rows(const Params& p, int s, int& lo, int& hi) {
    lo = 0; hi = p.n;
    if (p.seg_ptr) {
        lo = min(max(p.seg_ptr[s], 0), p.n);
        hi = max(lo, min(p.seg_ptr[s + 1], p.n));
    }
}
__device__ __forceinline__ int seg_adapter(const Params& p, int s) {
    const int id = p.seg_id ? p.seg_id[s] : 0;
    return (uint32_t)id < (uint32_t)p.n_adapters ? id : -1;
}

// A place in a ring of n and the parity of its present round (counted on: a division by a runtime n costs the waiting
// thread some 200 clocks, 2600 per QKV item when all roles had them).
struct Turn {
    int at = 0;
    uint32_t odd = 0;
    __device__ __forceinline__ void next(int n) {
        if (++at == n) { at = 0; odd ^= 1u; }
    }
};

// The last request from s on that ends at or before row `pos`, the last of all left out (s itself ends there): steps
// twice as long each time, then halves.  Offsets that decrease give some request in that range.
__device__ __forceinline__ int last_empty(const Params& p, int s, int pos) {
    auto ends = [&](int64_t i) { return min(max(p.seg_ptr[i + 1], 0), p.n) <= pos; };
    int64_t lo = s, hi = (int64_t)p.n_seg - 1;
    for (int64_t step = 16; lo + step < hi; step *= 2) {
        if (!ends(lo + step)) {
            hi = lo + step;
            break;
        }
        lo += step;
    }
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        (ends(mid) ? lo : hi) = mid;
    }
    return (int)lo;
}

// To the next item, which exists.  Runs of empty requests are searched through (one by one they cost 90 ns each, and the
// other warps' waits run out over some ten million of them).
__device__ __forceinline__ void walk_on(const Params& p, Walk& w) {
    w.lo += kTileM;
    for (int empty = 0; w.lo >= w.hi && w.seg + 1 < p.n_seg; ++empty) {
        if (empty == 16) {
            w.seg = last_empty(p, w.seg, w.hi);
            empty = 0;
        }
        ++w.seg;
        seg_rows(p, w.seg, w.lo, w.hi);
        w.adapter = seg_adapter(p, w.seg);
    }
    w.lo = min(w.lo, w.hi);           // offsets that decrease: an item without rows, inside the tensor
}

// Cuts all items into one contiguous run per CTA: every thread counts the tiles of its share of the requests, the
// CTA adds the counts up, and the thread in whose share this CTA's first item falls leaves it in shared memory.
__device__ __forceinline__ void find_items(const Params& p, Bars* bars) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int share = (int)(((int64_t)p.n_seg + kThreads - 1) / kThreads);
    // warp 0, which sets up the barriers and starts W on its way, takes the last share
    const int place = (warp == 0 ? kThreads : (int)threadIdx.x) - 32 + (warp == 0 ? lane : 0);
    const int64_t s0 = (int64_t)place * share;
    const int64_t s1 = min(s0 + share, (int64_t)p.n_seg);
    auto tiles_of = [&](int64_t s, int& lo, int& hi) {
        seg_rows(p, (int)s, lo, hi);
        return (int64_t)((uint32_t)(hi - lo) + kTileM - 1) / kTileM;
    };
    int lo = 0, hi = 0, id = -1;
    int64_t sum = 0;
    for (int64_t s = s0; s < s1; ++s) sum += tiles_of(s, lo, hi);
    if (share == 1 && s0 < s1) id = seg_adapter(p, (int)s0);   // on its way with the offsets
    int64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t below = __shfl_up_sync(0xffffffffu, (long long)incl, o);
        if (lane >= o) incl += below;
    }
    if (lane == 31) bars->warp_sum[warp] = incl;
    if (threadIdx.x == 0) bars->my_items = 0;
    __syncthreads();
    int64_t total = 0, before = incl - sum;
    for (int w = 0; w < kThreads / 32; ++w) {
        const int64_t x = bars->warp_sum[w];
        if (warp == 0 ? w > 0 : (w > 0 && w < warp)) before += x;
        total += x;
    }
    // the first total % gridDim.x CTAs take one item more (32-bit division where it suffices: 64 bits take 300 clocks)
    const int64_t each = total <= 0xffffffffll ? (int64_t)((uint32_t)total / gridDim.x) : total / gridDim.x;
    const int64_t rest = total - each * gridDim.x, b = blockIdx.x;
    const int64_t begin = b * each + min(b, rest), mine = each + (b < rest ? 1 : 0);
    if (mine > 0 && begin >= before && begin < before + sum) {
        int64_t s = s0, at = before;
        if (share > 1) {
            for (;; ++s) {
                const int64_t tiles = tiles_of(s, lo, hi);
                if (begin < at + tiles || s + 1 >= s1) break;
                at += tiles;
            }
            id = seg_adapter(p, (int)s);
        }
        bars->my_items = (int32_t)mine;
        bars->first.seg = (int32_t)s;
        bars->first.lo = lo + (int32_t)(begin - at) * kTileM;
        bars->first.hi = hi;
        bars->first.adapter = id;
    }
}

template <int RANK, int NB>
__global__ void __launch_bounds__(kThreads, NB == 3 ? 1 : 2)
adapter_proj_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                    const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_a,
                    const __grid_constant__ CUtensorMap map_b, const __grid_constant__ OutMaps map_o, Params p) {
    using P = Place<RANK, NB>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    Bars* bars = reinterpret_cast<Bars*>(smem_raw + (base - smem_u32(smem_raw)) + p.off_bar);
    const uint32_t sW = base, sB = base + p.off_b, sX = base + p.off_x, sR = base + p.off_r;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int block0 = blockIdx.y * NB, stages = p.stages;
    const int rank16 = (p.rank + 15) & ~15;
    const int a_half = rank16 * 128;                       // bytes of one half of A_a (a multiple of 1024)
    const int w_half = a_half + NB * kHalfBytes;           // and of A_a and W together
    volatile uint32_t* abort_flag = &bars->abort_flag;

    if (warp == 0) {
        auto init = [&](uint64_t* first, int n, int arrivals) {
            if (lane < n) mbar_init(smem_u32(first + lane), arrivals);
        };
        init(&bars->w_full, 1, 1);
        init(bars->a_full, kMaxStages, 1);
        init(bars->a_empty, kMaxStages, 1);
        init(bars->r_full, kMaxStages, 1);
        init(bars->r_empty, kMaxStages, kEpiWarps);
        init(bars->acc_full, kSlots, 1);
        init(bars->acc_empty, kSlots, kEpiWarps);
        init(&bars->la_full, 1, 1);
        init(&bars->la_empty, 1, 1);
        init(&bars->lb_full, 1, 1);
        init(&bars->lb_empty, 1, 1);
        init(bars->u_full, kUTurns, 1);
        init(&bars->u_ready, 1, kUWarps);
        init(&bars->ub_empty, 1, 1);
        init(bars->item_full, kRing, 1);
        init(bars->item_empty, kRing, 1 + kEpiWarps + kUWarps);
        init(&bars->drain, 1, 1);
        mbar_fence_init();
        __syncwarp();
    }
    if (threadIdx.x == 0) {
        bars->abort_flag = 0;
        // W travels while the items are counted
        mbar_expect_tx(smem_u32(&bars->w_full), (uint32_t)(NB * kTileBytes));
        for (int j = 0; j < NB; ++j)
            for (int h = 0; h < 2; ++h)
                tma_load_2d(sW + h * w_half + a_half + j * kHalfBytes, &map_w, h * 64, (block0 + j) * 128, smem_u32(&bars->w_full));
        tma_prefetch_desc(&map_x);
        tma_prefetch_desc(&map_a);
        tma_prefetch_desc(&map_b);
        for (int j = 0; j < NB; ++j) tma_prefetch_desc(&map_o.m[block0 + j]);
    }
    const uint32_t tmem_cols = p.slots == 1 ? 256u : 512u;
    if (warp == 1) tmem_alloc(smem_u32(&bars->tmem_base), tmem_cols);
    __syncwarp();
    find_items(p, bars);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    const int items = bars->my_items;

    if (warp == 0) {
        // ------------------------------------------------------------------ producer
        if (lane == 0) {
            int armed = 0, armed_r = 0, armed_la = 0, loads = 0;
            Turn q, s;                                         // of the descriptors, of the stages
            Walk w = bars->first;
            int held = -1;                                     // the adapter in shared memory, -1 = released
            for (int i = 0; i < items && !*abort_flag; ++i, q.next(kRing), s.next(stages)) {
                Item it;
                it.row0 = w.lo;
                it.rows = min(w.hi - w.lo, kTileM);
                it.adapter = w.adapter;
                if (i + 1 < items) walk_on(p, w);
                it.last = i + 1 == items || w.adapter != it.adapter;
                if (i >= kRing && !mbar_wait_relaxed(smem_u32(&bars->item_empty[q.at]), q.odd ^ 1u, p.poll_limit)) { raise_timeout(bars, p.status); break; }
                bars->ring[q.at] = it;
                mbar_arrive(smem_u32(&bars->item_full[q.at]));
                if (i >= stages && !mbar_wait_relaxed(smem_u32(&bars->a_empty[s.at]), s.odd ^ 1u, p.poll_limit)) { raise_timeout(bars, p.status); break; }
                mbar_expect_tx(smem_u32(&bars->a_full[s.at]), (uint32_t)kTileBytes);
                for (int h = 0; h < 2; ++h)
                    tma_load_2d(sX + s.at * kTileBytes + h * kHalfBytes, &map_x, h * 64, it.row0, smem_u32(&bars->a_full[s.at]));
                armed = i + 1;
                if (it.adapter >= 0 && it.adapter != held) {
                    // A_a's place is free once the previous adapter's last first product has read it, B_a's after its
                    // last second product: A_a travels while the item before is still being finished
                    const uint32_t free = ((uint32_t)loads & 1u) ^ 1u;
                    if (loads > 0 && !mbar_wait_relaxed(smem_u32(&bars->la_empty), free, p.poll_limit)) { raise_timeout(bars, p.status); break; }
                    mbar_expect_tx(smem_u32(&bars->la_full), (uint32_t)(p.rank * 256));
                    for (int h = 0; h < 2; ++h) tma_load_2d(sW + h * w_half, &map_a, h * 64, it.adapter * p.rank, smem_u32(&bars->la_full));
                    armed_la = loads + 1;
                    if (loads > 0 && !mbar_wait_relaxed(smem_u32(&bars->lb_empty), free, p.poll_limit)) { raise_timeout(bars, p.status); break; }
                    mbar_expect_tx(smem_u32(&bars->lb_full), (uint32_t)(NB * P::kB));
                    for (int j = 0; j < NB; ++j)
                        tma_load_2d(sB + j * P::kB, &map_b, 0, it.adapter * p.n_out + (block0 + j) * 128, smem_u32(&bars->lb_full));
                    ++loads;
                    held = it.adapter;
                }
                if (it.last) held = -1;
                if (p.has_res) {                               // last: its buffer is given back by the epilogue, later than X's
                    if (i >= stages && !mbar_wait_relaxed(smem_u32(&bars->r_empty[s.at]), s.odd ^ 1u, p.poll_limit)) { raise_timeout(bars, p.status); break; }
                    mbar_expect_tx(smem_u32(&bars->r_full[s.at]), (uint32_t)kTileBytes);
                    for (int h = 0; h < 2; ++h)
                        tma_load_2d(sR + s.at * kTileBytes + h * kHalfBytes, &map_r, h * 64, it.row0, smem_u32(&bars->r_full[s.at]));
                    armed_r = i + 1;
                }
            }
            // leave with no copy still landing in shared memory (these waits keep the default limit)
            mbar_wait(smem_u32(&bars->w_full), 0);
            for (int i = (armed > stages ? armed - stages : 0); i < armed; ++i)
                mbar_wait(smem_u32(&bars->a_full[i % stages]), (uint32_t)(i / stages) & 1u);
            for (int i = (armed_r > stages ? armed_r - stages : 0); i < armed_r; ++i)
                mbar_wait(smem_u32(&bars->r_full[i % stages]), (uint32_t)(i / stages) & 1u);
            if (armed_la > 0) mbar_wait(smem_u32(&bars->la_full), (uint32_t)(armed_la - 1) & 1u);
            if (loads > 0) mbar_wait(smem_u32(&bars->lb_full), (uint32_t)(loads - 1) & 1u);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (lane == 0) {
            const uint32_t idesc = idesc_bf16_f32(128, 128), idesc_first = idesc_bf16_f32(128, rank16 + 128),
                           idesc_two = idesc_bf16_f32(128, 256);
            bool ok = mbar_wait_relaxed(smem_u32(&bars->w_full), 0, p.poll_limit);
            int loads = 0, u_items = 0;
            Turn q, s, acc, u;                                 // of the descriptors, the stages, the accumulators, u_full
            bool fresh = true;                                 // the next adapter item brings a new adapter
            bool owed = false, owed_last = false, owed_new = false;   // NB = 1: the second product of the item before
            int owed_slot = 0, b_loads = 0;
            // d = X * (rows of A_a and W from row0 on)^T over K = 128, as many as `id` says
            auto product = [&](uint32_t d, uint32_t x_base, int row0, uint32_t id) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    mma_bf16(d, smem_desc_sw128(x_base + (uint32_t)((ks >> 2) * kHalfBytes + (ks & 3) * 32)),
                             smem_desc_sw128(sW + (uint32_t)((ks >> 2) * w_half + row0 * 128 + (ks & 3) * 32)), id, ks > 0 ? 1u : 0u);
            };
            // d += U * B_a^T for the column blocks from j on
            auto second = [&](uint32_t d, int j, uint32_t id) {
                for (int ks = 0; ks < rank16 / 16; ++ks)
                    mma_bf16_ta(d, tmem + (uint32_t)(p.col_ub + ks * 8), P::b_desc(sB + (uint32_t)(j * P::kB + ks * 32)), id, 1u);
            };
            auto u_wait = [&](bool new_adapter) {              // what the second product needs: U, and B_a
                bool r = mbar_wait_relaxed(smem_u32(&bars->u_ready), (uint32_t)(u_items++) & 1u, p.poll_limit);
                if (new_adapter) r = r && mbar_wait_relaxed(smem_u32(&bars->lb_full), (uint32_t)(b_loads++) & 1u, p.poll_limit);
                tc_fence_after();
                return r;
            };
            auto u_done = [&](bool last) {
                mma_commit(smem_u32(&bars->ub_empty));
                if (last) mma_commit(smem_u32(&bars->lb_empty));
            };
            auto settle = [&]() {                              // NB = 1: what is owed
                if (!owed) return true;
                owed = false;
                if (!u_wait(owed_new)) return false;
                second(tmem + (uint32_t)(owed_slot * P::kSetCols + rank16), 0, idesc);
                mma_commit(smem_u32(&bars->acc_full[owed_slot]));
                u_done(owed_last);
                return true;
            };
            for (int i = 0; i < items && ok && !*abort_flag; ++i, q.next(kRing), s.next(stages)) {
                ok = mbar_wait_relaxed(smem_u32(&bars->item_full[q.at]), q.odd, p.poll_limit);
                if (!ok) break;
                const Item it = bars->ring[q.at];
                mbar_arrive(smem_u32(&bars->item_empty[q.at]));
                const bool ad = it.adapter >= 0;
                const bool new_adapter = ad && fresh;
                // what is owed comes first if this item cannot begin yet
                if (owed && (!mbar_test(smem_u32(&bars->a_full[s.at]), s.odd) || !mbar_test(smem_u32(&bars->acc_empty[acc.at]), acc.odd ^ 1u) ||
                             (new_adapter && !mbar_test(smem_u32(&bars->la_full), (uint32_t)loads & 1u)))) ok = settle();
                ok = ok && mbar_wait_relaxed(smem_u32(&bars->a_full[s.at]), s.odd, p.poll_limit);
                if (new_adapter) ok = ok && mbar_wait_relaxed(smem_u32(&bars->la_full), (uint32_t)(loads++) & 1u, p.poll_limit);
                if (ad) fresh = it.last != 0;
                ok = ok && mbar_wait_relaxed(smem_u32(&bars->acc_empty[acc.at]), acc.odd ^ 1u, p.poll_limit);
                if (!ok) break;
                tc_fence_after();
                const uint32_t x_base = sX + s.at * kTileBytes;
                const uint32_t d = tmem + (uint32_t)(NB == 3 ? 0 : acc.at * P::kSetCols);
                product(ad ? d : d + rank16, x_base, ad ? 0 : rank16, ad ? idesc_first : idesc);
                if (ad) {
                    mma_commit(smem_u32(&bars->u_full[u.at]));
                    u.next(kUTurns);
                }
                if (ad && it.last) mma_commit(smem_u32(&bars->la_empty));
                if (NB == 1) {
                    mma_commit(smem_u32(&bars->a_empty[s.at]));
                    ok = settle();                             // while this item's U is on its way
                    if (ad) {
                        owed = true; owed_last = it.last != 0; owed_new = new_adapter; owed_slot = acc.at;
                    } else {
                        mma_commit(smem_u32(&bars->acc_full[acc.at]));
                    }
                    acc.next(p.slots);
                } else {
                    // the first block is finished at once, for the epilogue to go on with; the other two wait until it
                    // has left both of their accumulators
                    if (ad) {
                        ok = u_wait(new_adapter);
                        if (!ok) break;
                        second(d + rank16, 0, idesc);
                    }
                    mma_commit(smem_u32(&bars->acc_full[0]));
                    for (int j = 1; j < 3; ++j) ok = ok && mbar_wait_relaxed(smem_u32(&bars->acc_empty[j]), acc.odd ^ 1u, p.poll_limit);
                    if (!ok) break;
                    tc_fence_after();
                    product(d + rank16 + 128, x_base, rank16 + 128, idesc_two);
                    mma_commit(smem_u32(&bars->a_empty[s.at]));
                    if (ad) {
                        second(d + rank16 + 128, 1, idesc_two);
                        u_done(it.last != 0);
                    }
                    mma_commit(smem_u32(&bars->acc_full[1]));
                    mma_commit(smem_u32(&bars->acc_full[2]));
                    acc.odd ^= 1u;
                }
            }
            if (ok && !*abort_flag) ok = settle();
            if (!ok) raise_timeout(bars, p.status);
            mma_commit(smem_u32(&bars->drain));                // tensor memory is freed below: every MMA must be done
            mbar_wait(smem_u32(&bars->drain), 0);
        }
    } else if (warp < 2 + kEpiWarps) {
        // ------------------------------------------------------------------ epilogue (warps 2..9)
        const int ew = warp - 2, quad = warp & 3, half = ew >> 2;
        const uint32_t stage = base + p.off_stage + (uint32_t)(ew * 4096);
        Turn q, s, acc_turn;
        bool ok = true;
        for (int i = 0; i < items && ok; ++i, q.next(kRing), s.next(stages)) {
            if (__any_sync(0xffffffffu, *abort_flag != 0)) break;
            if (!mbar_wait_relaxed_warp(smem_u32(&bars->item_full[q.at]), q.odd, p.poll_limit)) { raise_timeout(bars, p.status); break; }
            const Item it = bars->ring[q.at];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->item_empty[q.at]));
            const int valid = it.rows - quad * 32;             // rows of the item among this warp's 32
            for (int j = 0; j < NB; ++j, acc_turn.next(p.slots)) {
                const int slot = acc_turn.at;
                ok = mbar_wait_relaxed_warp(smem_u32(&bars->acc_full[slot]), acc_turn.odd, p.poll_limit);
                if (ok && p.has_res) ok = mbar_wait_relaxed_warp(smem_u32(&bars->r_full[s.at]), s.odd, p.poll_limit);
                if (!ok) { raise_timeout(bars, p.status); break; }
                tc_fence_after();
                const uint32_t t_addr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(rank16 + slot * (NB == 3 ? 128 : P::kSetCols) + half * 64);
                const int row0 = it.row0 + quad * 32;
                if (NB == 3) {
                    // both halves at once (one CTA per SM has the registers), and the accumulator handed back before
                    // the conversions.  A residual does not come with three blocks.
                    uint32_t acc[64];
                    if (valid > 0) {
                        tmem_ld_32x32(t_addr, acc);
                        tmem_ld_32x32(t_addr + 32, acc + 32);
                        tmem_ld_wait();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&bars->acc_empty[slot]));
                        bulk_wait_read0();                     // the previous store has read the staging rows
                    }
                    __syncwarp();
                    __nv_bfloat16* outp = p.out[block0 + j] + (int64_t)(row0 + lane) * p.ldo[block0 + j] + half * 64;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint32_t out[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[e] = pack_bf16(__uint_as_float(acc[c * 8 + 2 * e]), __uint_as_float(acc[c * 8 + 2 * e + 1]));
                        if (valid >= 32) st_shared_v4(stage + sw128_offset(lane, c), out);
                        else if (lane < valid) st_global_v4(outp + c * 8, out);       // the item ends inside these rows
                    }
                    if (valid >= 32) {
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(&map_o.m[block0 + j], half * 64, row0, stage);
                            bulk_commit();
                        }
                    }
                    continue;
                }
                if (lane == 0) bulk_wait_read0();              // the previous store has read the staging rows
                __syncwarp();
#pragma unroll 1
                for (int c2 = 0; c2 < (valid > 0 ? 2 : 0); ++c2) {
                    uint32_t acc[32], res[16];
                    tmem_ld_32x32(t_addr + (uint32_t)(c2 * 32), acc);
                    if (p.has_res) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            ld_shared_v4(sR + (uint32_t)(s.at * kTileBytes + half * kHalfBytes) + sw128_offset(quad * 32 + lane, c2 * 4 + c), res + 4 * c);
                    }
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t out[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float lo = __uint_as_float(acc[c * 8 + 2 * e]), hi = __uint_as_float(acc[c * 8 + 2 * e + 1]);
                            if (p.has_res) {
                                lo += __uint_as_float(res[4 * c + e] << 16);
                                hi += __uint_as_float(res[4 * c + e] & 0xffff0000u);
                            }
                            out[e] = pack_bf16(lo, hi);
                        }
                        st_shared_v4(stage + sw128_offset(lane, c2 * 4 + c), out);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&bars->acc_empty[slot]));
                    if (p.has_res) mbar_arrive(smem_u32(&bars->r_empty[s.at]));
                }
                if (valid >= 32) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&map_o.m[block0 + j], half * 64, row0, stage);
                        bulk_commit();
                    }
                } else if (valid > 0) {
                    // the item ends inside these rows: 8 lanes per row, four rows per instruction
                    __nv_bfloat16* outp = p.out[block0 + j];
                    const int64_t ldo = p.ldo[block0 + j];
                    for (int r = lane >> 3; r < valid; r += 4) {
                        uint32_t v[4];
                        ld_shared_v4(stage + sw128_offset(r, lane & 7), v);
                        st_global_v4(outp + (int64_t)(row0 + r) * ldo + half * 64 + (lane & 7) * 8, v);
                    }
                    __syncwarp();
                }
            }
        }
        if (lane == 0) bulk_wait_all();
    } else {
        // ------------------------------------------------------------------ U (warps 10..13)
        const int quad = warp & 3;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        int u_items = 0;
        Turn q, set, full;
        for (int i = 0; i < items; ++i, q.next(kRing), set.next(NB == 3 ? 1 : p.slots)) {
            if (__any_sync(0xffffffffu, *abort_flag != 0)) break;
            if (!mbar_wait_relaxed_warp(smem_u32(&bars->item_full[q.at]), q.odd, p.poll_limit)) { raise_timeout(bars, p.status); break; }
            const Item it = bars->ring[q.at];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->item_empty[q.at]));
            if (it.adapter < 0) continue;
            const float scale = __ldg(p.scale + it.adapter);
            if (!mbar_wait_relaxed_warp(smem_u32(&bars->u_full[full.at]), full.odd, p.poll_limit) ||
                !mbar_wait_relaxed_warp(smem_u32(&bars->ub_empty), ((uint32_t)u_items & 1u) ^ 1u, p.poll_limit)) {
                raise_timeout(bars, p.status);
                break;
            }
            ++u_items;
            full.next(kUTurns);
            tc_fence_after();
            const uint32_t u = tmem + lanes + (uint32_t)(NB == 3 ? 0 : set.at * P::kSetCols);
            for (int c = 0; c < rank16 / 16; ++c) {            // 16 columns of U: one K step of the second product
                uint32_t f[16], b[8];
                tmem_ld_32x8(u + (uint32_t)(c * 16), f);
                tmem_ld_32x8(u + (uint32_t)(c * 16 + 8), f + 8);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // columns beyond the rank (a rank of 8, 24, ... inside a step of 16) are zero, whatever the unused
                    // rows of A's buffer held
                    const bool in = c * 16 + 2 * e < p.rank;
                    b[e] = in ? pack_bf16(__uint_as_float(f[2 * e]) * scale, __uint_as_float(f[2 * e + 1]) * scale) : 0u;
                }
                tmem_st_32x8(tmem + lanes + (uint32_t)(p.col_ub + c * 8), b);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->u_ready));
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, tmem_cols);
    }
}

// ---------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------
#define CHECK(expr) do { dg4_status _s = (expr); if (_s != DG4_OK) return _s; } while (0)

constexpr int kSmemLimit = 232448;                // what one CTA may hold

struct Call {
    const void* X; int64_t ldx;
    const void* W;
    const dg4_adapters* ad;
    const dg4_segments* seg;
    const void* R; int64_t ldr;
    void* out[3]; int64_t ldo[3];
    int n_out;
};

// bytes of shared memory in front of the X stages: W and A_a, B_a, the staging rows
int fixed_bytes(int nb, int rank, int place_rank) {
    return nb * kTileBytes + ((rank + 15) & ~15) * 256 + nb * 128 * place_rank * 2 + kEpiWarps * 4096;
}
constexpr int kTail = (int)sizeof(Bars) + 1024;         // 1024: the base is aligned by hand

template <int RANK, int NB>
dg4_status launch_place(const dg4_graph* g, const Call& c, int sms, int64_t most, bool split, cudaStream_t st) {
    using P = Place<RANK, NB>;
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    DG4_CUDA_TRY(cudaGetDevice(&dev));
    if (!attr_set[dev].load(std::memory_order_relaxed)) {
        DG4_CUDA_TRY(cudaFuncSetAttribute(adapter_proj_kernel<RANK, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
        attr_set[dev].store(true, std::memory_order_relaxed);
    }
    Params p;
    p.seg_ptr = c.seg ? c.seg->seg_ptr : nullptr;
    p.seg_id = c.seg ? c.seg->seg_id : nullptr;
    p.n_seg = c.seg ? c.seg->n_seg : 1;
    p.n = g->n; p.n_adapters = c.ad->n_adapters; p.rank = c.ad->rank; p.scale = c.ad->scale;
    p.n_out = c.n_out; p.has_res = c.R != nullptr;
    p.status = g->dev_status; p.poll_limit = dg4i_poll_limit();
    p.slots = NB == 3 ? 3 : split ? 1 : P::kSets;
    p.col_ub = NB == 1 && split ? P::kSetCols : P::kColUb;
    const int per_stage = kTileBytes * (p.has_res ? 2 : 1);
    int off = fixed_bytes(NB, p.rank, RANK);
    p.off_stage = off - kEpiWarps * 4096;
    p.off_b = p.off_stage - NB * P::kB;
    p.stages = !split && off + kMaxStages * per_stage + kTail <= kSmemLimit ? kMaxStages : 1;
    p.off_x = off; off += p.stages * kTileBytes;
    p.off_r = off; off += p.has_res ? p.stages * kTileBytes : 0;
    p.off_bar = off; off += kTail;
    CUtensorMap map_x, map_w, map_r, map_a, map_b;
    OutMaps map_o;
    CHECK(dg4i_make_row_map(&map_w, c.W, c.n_out, 128, 128));
    CHECK(dg4i_make_row_map(&map_x, c.X, g->n, c.ldx, 128));
    map_r = map_x;
    if (c.R) CHECK(dg4i_make_row_map(&map_r, c.R, g->n, c.ldr, 128));
    CHECK(dg4i_make_row_map(&map_a, c.ad->A, (int64_t)p.n_adapters * p.rank, 128, p.rank));
    CHECK(dg4i_make_map(&map_b, c.ad->B, p.rank, (int64_t)p.n_adapters * c.n_out, p.rank, 128, RANK));
    for (int j = 0; j < 3; ++j) {
        map_o.m[j] = map_x;
        p.out[j] = nullptr; p.ldo[j] = 0;
        if (j < c.n_out / 128) {
            CHECK(dg4i_make_row_map(&map_o.m[j], c.out[j], g->n, c.ldo[j], 32));
            p.out[j] = (__nv_bfloat16*)c.out[j]; p.ldo[j] = c.ldo[j];
        }
    }
    const dim3 grid((unsigned)(most < sms ? most : sms), (unsigned)(c.n_out / 128 / NB));
    adapter_proj_kernel<RANK, NB><<<grid, kThreads, off, st>>>(map_x, map_w, map_r, map_a, map_b, map_o, p);
    dg4i_count_launch();
    DG4_CUDA_TRY(cudaGetLastError());
    return DG4_OK;
}

template <int RANK>
dg4_status launch_rank(const dg4_graph* g, const Call& c, cudaStream_t st) {
    static std::atomic<int> sm_count[64];
    int dev = 0;
    DG4_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) DG4_FAIL(DG4_ERR_UNSUPPORTED, "device ordinal %d is out of range", dev);
    int sms = sm_count[dev].load(std::memory_order_relaxed);
    if (sms == 0) {
        DG4_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        sm_count[dev].store(sms, std::memory_order_relaxed);
    }
    // items: at most one per full tile and one ragged one per request
    const int64_t most = (int64_t)g->n / kTileM + (c.seg ? c.seg->n_seg : 1);
    if (c.n_out == 128) return launch_place<RANK, 1>(g, c, sms, most, false, st);
    // Column blocks to different CTAs (of one item at most) where the device holds them all at once, two to an SM if two
    // fit: each then fetches a third of W and ends with one block's epilogue instead of three.
    const int one = fixed_bytes(1, c.ad->rank, RANK) + kTileBytes + kTail;
    const bool split = most * 3 <= sms * (2 * (one + 1024) <= 233472 ? 2 : 1);
    return split ? launch_place<RANK, 1>(g, c, sms, most, true, st) : launch_place<RANK, 3>(g, c, sms, most, false, st);
}

dg4_status check_adapters(const dg4_adapters* ad, int n_out) {
    if (!ad) DG4_FAIL(DG4_ERR_INVALID_ARG, "null adapters");
    if (ad->n_adapters < 1) DG4_FAIL(DG4_ERR_INVALID_ARG, "the number of adapters (%d) is below one", ad->n_adapters);
    if (ad->rank < 8 || ad->rank > kRankMax || ad->rank % 8 != 0)
        DG4_FAIL(DG4_ERR_UNSUPPORTED, "rank = %d: must be a multiple of 8 up to %d", ad->rank, kRankMax);
    if ((int64_t)ad->n_adapters * n_out > 0x7fffffff)
        DG4_FAIL(DG4_ERR_UNSUPPORTED, "%d adapters are too many", ad->n_adapters);
    CHECK(dg4i_check_tensor("A", ad->A, 128, 2, 128));
    CHECK(dg4i_check_tensor("B", ad->B, ad->rank, 2, ad->rank));
    if (!ad->scale || ((uintptr_t)ad->scale & 3u)) DG4_FAIL(DG4_ERR_INVALID_ARG, "the adapters' scale is null or not 4-byte aligned");
    return DG4_OK;
}

}  // namespace

extern "C" dg4_status dg4_qkv_project_adapters(const dg4_graph* g, const dg4_desc* desc, const void* X, int64_t ldx,
                                               const void* W_qkv, const dg4_adapters* adapters,
                                               const dg4_segments* segments, void* Q, int64_t ldq, void* K, int64_t ldk,
                                               void* V, int64_t ldv, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, true));
    CHECK(dg4i_check_tensor("X", X, ldx, 2, 128));
    CHECK(dg4i_check_tensor("W_qkv", W_qkv, 128, 2, 128));
    CHECK(check_adapters(adapters, 384));
    if (segments) CHECK(dg4i_check_segments(segments));
    CHECK(dg4i_check_tensor("Q", Q, ldq, 2, 128));
    CHECK(dg4i_check_tensor("K", K, ldk, 2, 128));
    CHECK(dg4i_check_tensor("V", V, ldv, 2, 128));
    Call c = {X, ldx, W_qkv, adapters, segments, nullptr, 0, {Q, K, V}, {ldq, ldk, ldv}, 384};
    return adapters->rank <= 32 ? launch_rank<32>(g, c, (cudaStream_t)stream) : launch_rank<64>(g, c, (cudaStream_t)stream);
}

extern "C" dg4_status dg4_out_project_adapters(const dg4_graph* g, const dg4_desc* desc, const void* O, int64_t ldo,
                                               const void* W_o, const dg4_adapters* adapters,
                                               const dg4_segments* segments, const void* H_res, int64_t ldh, void* H_out,
                                               int64_t ldho, void* stream) {
    CHECK(dg4i_check_device(g));
    CHECK(dg4i_check_desc(desc, true));
    CHECK(dg4i_check_tensor("O", O, ldo, 2, 128));
    CHECK(dg4i_check_tensor("W_o", W_o, 128, 2, 128));
    CHECK(check_adapters(adapters, 128));
    if (segments) CHECK(dg4i_check_segments(segments));
    const bool res = (desc->flags & DG4_FLAG_RESIDUAL) && H_res;
    if (res) CHECK(dg4i_check_tensor("H_res", H_res, ldh, 2, 128));
    CHECK(dg4i_check_tensor("H_out", H_out, ldho, 2, 128));
    Call c = {O, ldo, W_o, adapters, segments, res ? H_res : nullptr, ldh, {H_out, nullptr, nullptr}, {ldho, 0, 0}, 128};
    return adapters->rank <= 32 ? launch_rank<32>(g, c, (cudaStream_t)stream) : launch_rank<64>(g, c, (cudaStream_t)stream);
}
