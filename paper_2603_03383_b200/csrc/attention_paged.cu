// Tree attention over a K/V cache in pages, of a batch whose first keys are the same (Section 3.2 / Fig. 2(b)), on the 5th-generation
// tensor cores.  Two launches: the products and running softmax of all pieces, and their combination.
//
// A row tile is 128 / G whole tree nodes times the G query heads of a KV head: 128 rows of a tensor-core product (fewer where G does not
// divide 128; the others idle).  Behind the shared prefix the nodes of all sequences follow one another, and a tile takes them as they
// come: every shared key is loaded and multiplied once per tile, whoever the rows belong to.  Behind it a tile holds nodes of one
// sequence.  An ITEM is a KV head's keys (the prefix, or one sequence's own) for two row tiles, or for the one that is left over where
// their number is odd; its keys come in tiles of 128.  Items of two row tiles and items of one (the PHASES of the kernel) are each laid
// out on a line on which a key tile counts TILE_COST and the start and end of an item ITEM_COST; the CTAs are divided between the two
// by what they take (not one after the other on all: the prefix of a decoding batch would be cut into 148 pieces of four key tiles, whose partial
// results and cold starts took longer than its products), and each line is cut into equal runs, one per worker.  A worker's PIECE of an item leaves O (fp32, unnormalised) and the running
// (max, sum) of its rows in the workspace, and the second kernel joins the pieces; an item that is one worker's alone and has no prefix
// beside it is written out directly.
//
// One persistent CTA per SM.  Both phases keep two row tiles in flight, each with its own scores S / weights P and accumulator O in tensor
// memory and its own eight softmax warps (two threads per row, 64 columns each): while the tensor core works for one, the other's
// exponentials are taken.  In the phase of pairs the two tiles are those of an item and share K and V; in the other the CTA is two workers,
// whose K and V take turns in one ring.
//   warps 0-7 / 8-15  softmax of row tile 0 / 1
//   warps 16, 17      issue the products of row tile 0 / 1, O += P V and then S = Q K of the next key tile: products of one thread are executed
//                     in order, so S may overwrite the P that the product in front of it reads, and "S is complete" implies that O is
//                     complete up to the tile before.  (A wait costs an issuing warp a hundred cycles even where there is nothing to wait for,
//                     and the tensor core has only some two products queued: one warp for both row tiles left it idle a third of the time.)
//   warp 18           derives the pieces from the lengths, hands them to the other warps, and requests their Q, K and V (a box per page)
//   warp 19           clears V rows behind the last key (their weight is 0, but 0 * NaN is not) and takes non-finite values of the tree's
//                     V rows out (they are given to the rows that see them at the end)
//
// The reference of a row's exponentials is the maximum of the piece's first tile.  It moves only where a later tile's weights reach 2^64:
// P, O and the sum are floating-point numbers, to which the reference's size is all the same as long as nothing overflows.  So an ordinary
// tile forms no maximum; a vote of the two threads of a row says that neither needs the reference moved, and only otherwise they take
// the scores again, exchange their maxima (through tensor memory) and rescale O.
//
// Measured, whole calls: trees of 64 nodes of 8 sequences, 32 / 8 heads of 128, 16384 shared keys and up to 2048 of their own (147 GFLOP):
// 178 us (one card of several took 153), the tensor pipe at 50 %: a pair of key tiles takes some 3.9 k cycles of the 2.05 k that its
// products need; the rest is the chain scores -> exponentials -> weights -> product of each row tile, which its one other row tile does not hide.
// 7 sequences of up to 5001 keys, 29 nodes, 28 / 4 heads: 33 to 37 us for 6.4 us of bytes; start, first tile and joining are two thirds of it.
// All 20 warps have 96 registers; the softmax warps spill (160 bytes stored, 204 loaded a thread at D = 128, 144 and 244 at D = 64).
#include "attn_common.cuh"
#include "paged_common.cuh"
#include "paged_plan.cuh"

namespace mtv {

constexpr int PA_THREADS = 640;
constexpr int PA_MMA_WARP = 16, PA_TMA_WARP = 18, PA_CLEAN_WARP = 19;
constexpr int PA_QUEUE = 4;               // pieces that are handed out and may not have been taken by all
constexpr int PA_KEYS = 128;              // keys of a tile
constexpr int PA_MAX_B = 1024;
constexpr float PA_LIMIT = 64.f;          // weights stay below 2^64
// P goes to the second product as bf16, whose rounding is the largest error beside the output's own (relative 2-norm against 64 bits, N(0, 1) inputs:
// .0023 with it, .00166 without).  As in tree_verify_attention, head size 64 has a second bf16 term, what the rounding of the first left, in every tile
// (three trees of 128 nodes, 16 / 2 heads of 64, 4096 shared keys: 31.2 us without, 35.3 with), and so have thin items, whose products cost nothing beside
// their bytes.  At head size 128 a row tile has one term (its products are a third of the time there: 16384 shared keys 179 us, 238 with two in every tile,
// 192 in four of a piece; one-layer calls of tree_verify_attention are at .0027, short ones at .0017).
template <int D> constexpr bool TWO_TERMS = D == 64;
constexpr int TILE_COST = 4;              // a key tile on a line
__host__ __device__ constexpr int ITEM_COST(int single) { return single ? 8 : 16; }   // what the start and end of an item take, in the same quarters of a key tile, for pairs and for single row tiles
__host__ __device__ constexpr int PHASE_COST(int single) { return single ? 4 : 7; }   // and what a quarter of a key tile takes a CTA, one against the other: pairs are bound by the tensor core and
                                          // its waits (3.9 k cycles a key tile at D = 128), single row tiles by their K and V (2.2 k, two at a time); measured at D = 128, taken at D = 64 too

template <int D> struct PaSmem {
    static constexpr int HALVES = D / 64;
    static constexpr uint32_t HALF = 128 * 128;          // 128 rows of 64 columns, 128-byte swizzle
    static constexpr uint32_t TILE = HALVES * HALF;
    static constexpr int STAGES = D == 128 ? 5 : 10;
    static constexpr uint32_t OFF_RING = 2 * TILE, OFF_BAR = OFF_RING + STAGES * TILE, TOTAL = 1024 + OFF_BAR + 1024;
    static_assert(TOTAL <= 227 * 1024, "shared memory budget");
    static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (128u >> 4) << 24;     // bf16 x bf16 -> fp32, M = 128
    static constexpr uint32_t IDESC_QK = IDESC | (128u >> 3) << 17;                               // N = 128 keys
    static constexpr uint32_t IDESC_PV = IDESC | (uint32_t)(D >> 3) << 17 | 1u << 16;             // N = D columns, B (= V) N-major
};

enum {
    PB_FULL = 0, PB_FREE = 10, PB_CLEAN = 20, PB_QFULL = 30, PB_QFREE = 32, PB_SREADY = 34, PB_PREADY = 36, PB_ODONE = 38, PB_FINAL = 40,
    PB_PIECE = 41,                         // [3 queues][PA_QUEUE]: pairs; single tiles of either half of the CTA
    PB_TAKEN = PB_PIECE + 3 * PA_QUEUE,
    PB_TURN = PB_TAKEN + 3 * PA_QUEUE,     // [2] an issuing warp's turn at the tensor core
    PB_COUNT = PB_TURN + 2
};
constexpr uint32_t PA_OFF_MISC = PB_COUNT * 8, PA_OFF_QUEUE = (PA_OFF_MISC + 40 + 15) / 16 * 16;
static_assert(PA_OFF_QUEUE + 3 * PA_QUEUE * 32 <= 1024, "barrier region");

struct PaParams {
    PagedRef pages;
    PaPhase phase[3];                  // pairs of row tiles, single row tiles, thin ones
    const int32_t *seq_lens;
    const uint64_t *anc;               // [T][2]
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16 *out;
    int32_t *status, *dev_error;
    float scale_log2;
    int B, T, G, Hq, Hkv, shared, npc, page_rows;
};

// ---------------------------------------------------------------------------------------- the division of the work
__device__ __forceinline__ int key_tiles(int keys) { return (keys + PA_KEYS - 1) / PA_KEYS; }
__device__ __forceinline__ int item_cost(int tiles, int ends) { return tiles ? tiles * TILE_COST + ends : 0; }
// own key tiles of a sequence; 0: it is left out
__device__ __forceinline__ int seq_tiles(const PaParams &p, int L) {
    return p.pages.fits(L, p.T) && L >= p.shared ? key_tiles(L - p.shared + p.T) : 0;
}
// tiles of an item in front of position y of its stretch of the line
__device__ __forceinline__ int cut_at(int y, int tiles, int ends) { return y <= ends ? 0 : min((y - ends + TILE_COST / 2) / TILE_COST, tiles); }

struct __align__(16) PaPiece {
    int b;              // -1: the prefix
    int g, tile0;       // KV head, first row tile
    int t0, t1;         // key tiles; t1 = 0: no more pieces
    int L;              // keys in front of the tree, without the shared ones (prefix: the shared ones)
    int slot;
    int whole;          // the item's only piece
};
static_assert(sizeof(PaPiece) == 32, "two 16-byte words");
// The tile needs more than its copy: it holds rows of the tree, or rows behind them.
__device__ __forceinline__ bool is_last(const PaPiece &s, int t) { return s.b >= 0 && (t + 1) * PA_KEYS > s.L; }

// A worker's run of a phase's line (lines are shorter than 2^31: checked by the host).
struct PaWalk {
    int x0, x1, S;      // the run, and the position of the next item
    int b, idx, tiles, L, worker, ends;
    __device__ __forceinline__ void load(const PaParams &p) {
        if (b < 0) {
            L = p.shared;
            tiles = key_tiles(L);
        } else {
            const int len = p.seq_lens[b];
            tiles = seq_tiles(p, len);
            L = len - p.shared;
        }
    }
    __device__ __forceinline__ bool next(const PaParams &p, const PaPhase &f, PaPiece &s) {
        while (S < x1) {
            if (idx >= (b < 0 ? f.prefix_items : f.seq_items) || tiles == 0) {
                if (++b >= p.B) return false;
                idx = 0;
                load(p);
                continue;
            }
            s.t0 = cut_at(x0 - S, tiles, ends);
            s.t1 = cut_at(x1 - S, tiles, ends);
            S += item_cost(tiles, ends);
            const int i = idx++;
            if (s.t0 >= s.t1) continue;
            const int per = b < 0 ? f.prefix_per_head : f.seq_per_head, item = b < 0 ? i : f.prefix_items + b * f.seq_items + i;
            s.b = b; s.L = L;
            s.g = i / per;
            s.tile0 = (b < 0 ? f.prefix_tile0 : f.seq_tile0) + 2 * (i - s.g * per);
            s.slot = item + worker;
            s.whole = s.t0 == 0 && s.t1 == tiles;
            if (threadIdx.x % 32 == 0) {
                if (s.t0 == 0) f.span[item].x = worker;
                if (s.t1 == tiles) f.span[item].y = worker;
            }
            return true;
        }
        return false;
    }
};
// The runs of the workers of a CTA (pairs; single tiles of its halves) and the items they begin in.  One warp.
__device__ __forceinline__ void begin_walks(const PaParams &p, PaWalk (&w)[3], int cta, int n_cta, int lane) {
    auto tiles_of = [&](int b) { return b < p.B ? seq_tiles(p, p.seq_lens[b]) : 0; };
    const int own0 = tiles_of(lane);
    int tiles = own0, seqs = own0 > 0;   // key tiles of an item of every sequence that is not left out, and their number
    for (int b0 = 32; b0 < p.B; b0 += 32) {
        const int t = tiles_of(b0 + lane);
        tiles += t;
        seqs += t > 0;
    }
    tiles = __reduce_add_sync(0xffffffffu, tiles);
    seqs = __reduce_add_sync(0xffffffffu, seqs);
    int prefix[2], length[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        prefix[f] = item_cost(key_tiles(p.shared), ITEM_COST(f)) * p.phase[f].prefix_items;
        length[f] = prefix[f] + (tiles * TILE_COST + seqs * ITEM_COST(f)) * p.phase[f].seq_items;
    }
    // the first CTAs take the pairs, the others the single row tiles
    int n_pairs = n_cta;
    if (length[1]) {
        const float a = (float)length[0] * PHASE_COST(0), b = (float)length[1] * PHASE_COST(1);
        n_pairs = length[0] ? max(1, min(n_cta - 1, __float2int_rn(n_cta * (a / (a + b))))) : 0;
    }
    int y[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int f = k > 0, cost = item_cost(key_tiles(p.shared), ITEM_COST(f));
        const int workers = f ? 2 * (n_cta - n_pairs) : n_pairs, worker = k == 0 ? cta : k == 1 ? cta - n_pairs : cta + n_cta - 2 * n_pairs;
        const bool on = f ? cta >= n_pairs : cta < n_pairs;
        w[k].worker = worker;
        w[k].ends = ITEM_COST(f);
        // none shorter than a key tile, so that no worker in the middle of an item is left without a tile
        const int run = on ? max((length[f] + workers - 1) / workers, TILE_COST) : 0;
        w[k].x0 = on ? (int)min((int64_t)length[f], (int64_t)run * worker) : 0;
        w[k].x1 = (int)min((int64_t)length[f], (int64_t)w[k].x0 + run);
        w[k].b = -1;
        w[k].idx = 0;
        w[k].S = w[k].x0 == w[k].x1 ? w[k].x1 : 0;
        y[k] = -1;
        if (w[k].x0 < w[k].x1) {
            if (w[k].x0 < prefix[f]) {
                w[k].idx = w[k].x0 / cost;
                w[k].S = w[k].idx * cost;
            } else {
                y[k] = w[k].x0 - prefix[f];
            }
        }
    }
    int before_tiles = 0, before_seqs = 0;
    for (int b0 = 0; b0 < p.B && (y[0] >= 0 || y[1] >= 0 || y[2] >= 0); b0 += 32) {
        const int own = b0 ? tiles_of(b0 + lane) : own0;
        const uint32_t some = __ballot_sync(0xffffffffu, own > 0);
        const int n = __popc(some & (0xffffffffu >> (31 - lane)));
        int c = own;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int x = __shfl_up_sync(0xffffffffu, c, o);
            if (lane >= o) c += x;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const PaPhase &f = p.phase[k > 0];
            const int ends = ITEM_COST(k > 0), up_to = ((before_tiles + c) * TILE_COST + (before_seqs + n) * ends) * f.seq_items;
            const uint32_t behind = __ballot_sync(0xffffffffu, up_to > y[k]);
            if (y[k] < 0 || !behind) continue;
            const int at = __ffs((int)behind) - 1;
            const int each = item_cost(__shfl_sync(0xffffffffu, own, at), ends), first = __shfl_sync(0xffffffffu, up_to, at) - each * f.seq_items;
            w[k].b = b0 + at;
            w[k].idx = (y[k] - first) / each;
            w[k].S = w[k].x0 - y[k] + first + w[k].idx * each;
            y[k] = -1;
        }
        before_tiles += __shfl_sync(0xffffffffu, c, 31);
        before_seqs += __popc(some);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (w[k].x0 < w[k].x1) w[k].load(p);
}

// All of a phase's key tiles in the order in which the ring holds them: a round takes, list after list, V of the tile before and K of the
// tile after.  next(list, piece) -> whether there is one; f(list, piece and tile of V or none, piece and tile of K or none) -> whether to go on.
template <int NL, typename N, typename F>
__device__ __forceinline__ bool for_rounds(N &&next, F &&f) {
    PaPiece cur[NL], old[NL];
    int t[NL], old_t[NL];
    bool live[NL], pend[NL];
#pragma unroll
    for (int l = 0; l < NL; ++l) {
        live[l] = next(l, cur[l]);
        t[l] = cur[l].t0;
        pend[l] = false;
        old[l] = cur[l];
        old_t[l] = 0;
    }
    for (;;) {
        bool any = false;
#pragma unroll
        for (int l = 0; l < NL; ++l) {
            if (!live[l] && !pend[l]) continue;
            any = true;
            if (!f(l, pend[l], old[l], old_t[l], live[l], cur[l], t[l])) return false;
            pend[l] = live[l];
            if (live[l]) {
                old[l] = cur[l];
                old_t[l] = t[l];
                if (++t[l] == cur[l].t1) {
                    live[l] = next(l, cur[l]);
                    t[l] = cur[l].t0;
                }
            }
        }
        if (!any) return true;
    }
}

// maximum that a NaN wins
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// What the rounding of two values to bf16 pairs left, as bf16 pairs.
__device__ __forceinline__ uint32_t rounded_off(float2 p, uint32_t w) {
    const float2 r = __fadd2_rn(p, make_float2(-__uint_as_float(w << 16), -__uint_as_float(w & 0xffff0000u)));
    return pack2_bf16(r.x, r.y);
}
__device__ __forceinline__ bool nonfinite16(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }

// The two warps that hold the same rows: whether any of their threads says so.
__device__ __forceinline__ bool any_of_rows(int barrier, bool mine) {
    uint32_t r;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "barrier.cta.red.or.pred q, %2, 64, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(r) : "r"((uint32_t)mine), "r"(barrier) : "memory");
    return r != 0;
}
__device__ __forceinline__ void tmem_put(uint32_t taddr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "f"(v) : "memory");
}
__device__ __forceinline__ float tmem_get(uint32_t taddr) {
    float v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n"
                 "tcgen05.wait::ld.sync.aligned;" : "=f"(v) : "r"(taddr) : "memory");
    return v;
}
__device__ __forceinline__ void pa_cta_sync() { asm volatile("bar.sync 1, %0;" ::"n"(PA_THREADS) : "memory"); }

// ---------------------------------------------------------------------------------------- pieces
template <int D>
__global__ void __launch_bounds__(PA_THREADS, 1)
paged_attn_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                  const __grid_constant__ PaParams p) {
    using SM = PaSmem<D>;
    constexpr bool TWO = TWO_TERMS<D>;
    // tensor-memory columns of a half of the keys (64 scores): P, keys 0-31 at 0-15 and 32-63 at 32-47 with their second terms behind them, or all at 0-31;
    // and what the threads of a row exchange, where second terms go, or behind P
    constexpr int X_COL = TWO ? 16 : 40;
    extern __shared__ unsigned char smem_raw[];
    let_next_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t raw = ptx::smem_u32(smem_raw), pad = (1024u - (raw & 1023u)) & 1023u, sbase = raw + pad;
    unsigned char *gbase = smem_raw + pad;
    const uint32_t bars = sbase + SM::OFF_BAR;
    auto bar = [&](int i) { return bars + (uint32_t)i * 8u; };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(gbase + SM::OFF_BAR + PA_OFF_MISC);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + PA_OFF_MISC + 4);
    volatile int *bad = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + PA_OFF_MISC + 8);   // [2][4]: 1 + the last piece with non-finite V
    int4 *queue = reinterpret_cast<int4 *>(gbase + SM::OFF_BAR + PA_OFF_QUEUE);                    // [3][PA_QUEUE] pieces

    if (warp == PA_TMA_WARP && lane == 0) {
        ptx::prefetch_tensormap(&q_map);
        ptx::prefetch_tensormap(&k_map);
        ptx::prefetch_tensormap(&v_map);
        for (int s = 0; s < SM::STAGES; ++s) {
            ptx::mbar_init(bar(PB_FULL + s), 1);
            ptx::mbar_init(bar(PB_FREE + s), 3);      // the issuing warps, and the one that looks at every entry
            ptx::mbar_init(bar(PB_CLEAN + s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(bar(PB_QFULL + s), 1);
            ptx::mbar_init(bar(PB_QFREE + s), 1);
            ptx::mbar_init(bar(PB_SREADY + s), 1);
            ptx::mbar_init(bar(PB_PREADY + s), 8);
            ptx::mbar_init(bar(PB_ODONE + s), 1);
            ptx::mbar_init(bar(PB_TURN + s), 1);
        }
        ptx::mbar_init(bar(PB_FINAL), 2);
        for (int q = 0; q < 3; ++q)
            for (int i = 0; i < PA_QUEUE; ++i) {
                ptx::mbar_init(bar(PB_PIECE + q * PA_QUEUE + i), 1);
                ptx::mbar_init(bar(PB_TAKEN + q * PA_QUEUE + i), q ? 3 + 8 : 3 + 16);
            }
        ptx::fence_mbar_init();
        *abort_flag = 0;
        for (int k = 0; k < 8; ++k) bad[k] = 0;
    }
    if (warp == PA_MMA_WARP) {
        ptx::tmem_alloc(ptx::smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    previous_done();
    const int n_cta = gridDim.x, cta = blockIdx.x;
    const uint32_t tmem = *tmem_slot;
    auto give_up = [&]() {
        *abort_flag = 1;
        atomicExch(p.dev_error, MTV_ERR_TIMEOUT);
    };
    // a whole warp waits; the same answer for all lanes
    auto wait = [&](int b, uint32_t parity) {
        const bool ok = ptx::mbar_wait(bar(b), parity);
        if (__all_sync(0xffffffffu, ok)) return true;
        if (lane == 0) give_up();
        return false;
    };
    // the n-th piece of a queue; none (or nothing to be had): false
    auto take = [&](int q, int n, PaPiece &s) {
        const int at = q * PA_QUEUE + n % PA_QUEUE;
        if (__any_sync(0xffffffffu, *abort_flag) || !wait(PB_PIECE + at, (n / PA_QUEUE) & 1)) { s.t0 = s.t1 = 0; return false; }
        const int4 a = queue[at * 2], c = queue[at * 2 + 1];
        s.b = a.x; s.g = a.y; s.tile0 = a.z; s.t0 = a.w; s.t1 = c.x; s.L = c.y; s.slot = c.z; s.whole = c.w;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(PB_TAKEN + at));
        __syncwarp();
        return s.t1 > 0;
    };

    if (warp == PA_TMA_WARP) {
        // ------------------------------------------------------------ pieces; Q, K and V
        PaWalk w[3];
        begin_walks(p, w, cta, n_cta, lane);
        // One piece more for a queue, or its end: a piece without tiles.  (There is room, or will be without this warp's doing: the queries
        // of a piece are only requested when the scores of the one before are complete, so this warp is never three pieces ahead.)
        auto hand_out = [&](int q, int n, PaPiece &s) {
            const int at = q * PA_QUEUE + n % PA_QUEUE;
            const bool any = w[q].next(p, p.phase[q > 0], s);
            if (!any) s = PaPiece{};
            if (n >= PA_QUEUE && !wait(PB_TAKEN + at, (n / PA_QUEUE - 1) & 1)) { s.t0 = s.t1 = 0; return false; }
            if (lane == 0) {
                queue[at * 2] = make_int4(s.b, s.g, s.tile0, s.t0);
                queue[at * 2 + 1] = make_int4(s.t1, s.L, s.slot, s.whole);
                ptx::mbar_arrive(bar(PB_PIECE + at));
            }
            __syncwarp();
            return any;
        };
        int entry = 0, stage = 0, turns = 0;
        int n_q[2] = {0, 0};
        const int boxes = PA_KEYS / p.page_rows, box = lane % boxes, half = lane / boxes;
        const uint32_t q_bytes = (uint32_t)(p.npc * p.G) * 128u * SM::HALVES;
        // This lane's entry of the table for a key tile, requested here and looked at where the tile is: nothing waits for it meanwhile.
        // (Where there is no page, or the table names none, zeros are copied.)
        auto find = [&](const PaPiece &s, int t) {
            const int key = t * PA_KEYS + box * p.page_rows;
            int id = -1;
            if (half < SM::HALVES && key < s.L + (s.b < 0 ? 0 : p.T))
                asm volatile("ld.global.s32 %0, [%1];" : "=r"(id)
                             : "l"(p.pages.table + (int64_t)max(s.b, 0) * p.pages.max_pages + ((key + (s.b < 0 ? 0 : p.shared)) >> p.pages.page_shift)));
            return id;
        };
        auto row_in_page = [&](const PaPiece &s, int t) {
            return (t * PA_KEYS + box * p.page_rows + (s.b < 0 ? 0 : p.shared)) & ((1 << p.pages.page_shift) - 1);
        };
        auto load = [&](const CUtensorMap *map, int id, int row, int g) {
            if (entry >= SM::STAGES && !wait(PB_FREE + stage, (turns - 1) & 1)) return false;
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar(PB_FULL + stage), SM::TILE);
            __syncwarp();
            if (half < SM::HALVES)
                ptx::tma_load_4d(sbase + SM::OFF_RING + stage * SM::TILE + half * SM::HALF + box * p.page_rows * 128, map, bar(PB_FULL + stage),
                                 half * 64, row, g, id >= 0 && id < p.pages.n_pages ? id : p.pages.n_pages);
            ++entry;
            if (++stage == SM::STAGES) { stage = 0; ++turns; }
            return true;
        };
        auto phase = [&](auto lists) {
            constexpr int NL = decltype(lists)::value;
            int v_id[NL] = {}, k_id[NL] = {}, n[NL] = {};
            auto next = [&](int l, PaPiece &s) {
                if (!hand_out(NL == 1 ? 0 : 1 + l, n[l]++, s)) return false;
                k_id[l] = find(s, s.t0);
                return true;
            };
            return for_rounds<NL>(next, [&](int l, bool v, const PaPiece &vs, int vt, bool k, const PaPiece &ks, int kt) {
                if (v && !load(&v_map, v_id[l], row_in_page(vs, vt), vs.g)) return false;
                if (!k) return true;
                if (!load(&k_map, k_id[l], row_in_page(ks, kt), ks.g)) return false;
                v_id[l] = k_id[l];
                if (kt + 1 < ks.t1) k_id[l] = find(ks, kt + 1);
                if (kt == ks.t0)
                    for (int s = l; s < (NL == 1 ? 2 : l + 1); ++s) {
                        if (n_q[s] && !wait(PB_QFREE + s, (n_q[s] - 1) & 1)) return false;
                        ++n_q[s];
                        if (lane == 0) {
                            ptx::mbar_arrive_expect_tx(bar(PB_QFULL + s), q_bytes);
                            for (int h = 0; h < SM::HALVES; ++h)
                                ptx::tma_load_4d(sbase + s * SM::TILE + h * SM::HALF, &q_map, bar(PB_QFULL + s), h * 64, ks.g * p.G,
                                                 max(ks.b, 0) * p.T + (ks.tile0 + (NL == 1 ? s : 0)) * p.npc, 0);
                        }
                        __syncwarp();
                    }
                return true;
            });
        };
        if (!phase(std::integral_constant<int, 1>()) || !phase(std::integral_constant<int, 2>()) || *abort_flag) {
            // copies in flight get a bounded chance to land before the CTA can exit
            for (int e = max(0, entry - SM::STAGES); e < entry; ++e) ptx::mbar_wait(bar(PB_FULL + e % SM::STAGES), (e / SM::STAGES) & 1);
            for (int s = 0; s < 2; ++s)
                if (n_q[s]) ptx::mbar_wait(bar(PB_QFULL + s), (n_q[s] - 1) & 1);
        }
    } else if (warp == PA_MMA_WARP || warp == PA_MMA_WARP + 1) {
        // ------------------------------------------------------------ products of row tile s
        const int s = warp - PA_MMA_WARP;
        const bool leader = ptx::elect_one();
        const uint32_t dq = ptx::desc_lo(sbase + s * SM::TILE, 16), dk0 = ptx::desc_lo(sbase + SM::OFF_RING, 16), dv0 = ptx::desc_lo(sbase + SM::OFF_RING, SM::HALF);
        const uint32_t t_s = tmem + s * 128, t_o = tmem + 256 + s * D;
        int entry = 0, n_p = 0, n_q = 0, n_turn = 0;
        uint32_t cleaned = 0;            // parity of each stage's next cleaning
        auto phase = [&](auto lists) {
            constexpr int NL = decltype(lists)::value;
            int n[NL] = {};
            return for_rounds<NL>([&](int l, PaPiece &x) { return take(NL == 1 ? 0 : 1 + l, n[l]++, x); }, [&](int l, bool v, const PaPiece &vs, int vt, bool k, const PaPiece &ks, int kt) {
                const int ve = entry, ke = entry + (v ? 1 : 0);
                entry = ke + (k ? 1 : 0);
                const int v_stage = ve % SM::STAGES, k_stage = ke % SM::STAGES;
                const bool last_v = v && is_last(vs, vt);
                const uint32_t clean_parity = cleaned >> v_stage & 1;
                if (last_v) cleaned ^= 1u << v_stage;
                if (NL == 2 && l != s) {
                    // the other tile's: waited for and handed back all the same, so that this warp is never a turn of the ring ahead or
                    // late (a parity wait cannot tell a phase from the one two before or behind)
                    auto pass = [&](int e, int stage) {
                        if (!wait(PB_FULL + stage, (e / SM::STAGES) & 1)) return false;
                        if (lane == 0) ptx::mbar_arrive(bar(PB_FREE + stage));
                        __syncwarp();
                        return true;
                    };
                    return (!v || pass(ve, v_stage)) && (!k || pass(ke, k_stage));
                }
                auto k_there = [&]() { return wait(PB_FULL + k_stage, (ke / SM::STAGES) & 1) && (kt != ks.t0 || wait(PB_QFULL + s, n_q++ & 1)); };
                // Pairs take turns: the products of a row tile go to the tensor core in one run.  Mixed with the other tile's, both tiles' scores
                // would come when all are done, both softmaxes would then run at once, and the tensor core wait for both.
                auto begin_run = [&]() {
                    if (NL == 2) return true;
                    const int turn = n_turn++;
                    return s == 0 && turn == 0 ? true : wait(PB_TURN + s, (turn + s - 1) & 1);
                };
                auto end_run = [&]() {
                    if (NL == 1 && lane == 0) ptx::mbar_arrive(bar(PB_TURN + (s ^ 1)));
                    __syncwarp();
                };
                // the weights are waited for last: what else there is to wait for is there by then (a new piece's queries may not be)
                const bool ahead = v && k && kt != ks.t0;
                if (ahead && !k_there()) return false;
                if (v) {
                    // (first that it has landed: only then is the stage's cleaning before this one known to be over)
                    if (!wait(PB_FULL + v_stage, (ve / SM::STAGES) & 1) || (last_v && !wait(PB_CLEAN + v_stage, clean_parity))) return false;
                    if (!wait(PB_PREADY + s, n_p++ & 1)) return false;
                    if (!begin_run()) return false;
                    ptx::tc_fence_after();
                    const uint32_t dv = dv0 + (uint32_t)v_stage * (SM::TILE >> 4);
#pragma unroll
                    for (int kk = 0; kk < PA_KEYS / 16; ++kk)
                        ptx::mma_ts_elect(t_o, t_s + (TWO ? kk / 2 * 32 + kk % 2 * 8 : kk / 4 * 64 + kk % 4 * 8), dv + kk * 128, ptx::DESC_HI, SM::IDESC_PV, vt > vs.t0 || kk > 0, leader);
                    if (TWO) {
#pragma unroll
                        for (int kk = 0; kk < PA_KEYS / 16; ++kk)
                            ptx::mma_ts_elect(t_o, t_s + kk / 2 * 32 + 16 + kk % 2 * 8, dv + kk * 128, ptx::DESC_HI, SM::IDESC_PV, true, leader);
                    }
                    if (vt == vs.t1 - 1) ptx::tc_commit_elect(bar(PB_ODONE + s), leader);
                    if (!ahead) end_run();
                }
                if (k) {
                    if (!ahead) {
                        if (!k_there() || !begin_run()) return false;
                        ptx::tc_fence_after();
                    }
                    const uint32_t dk = dk0 + (uint32_t)k_stage * (SM::TILE >> 4);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t o = ((kk / 4) * SM::HALF + (kk % 4) * 32) >> 4;
                        ptx::mma_ss_elect(t_s, dq + o, dk + o, ptx::DESC_HI, SM::IDESC_QK, kk > 0, leader);
                    }
                    ptx::tc_commit_elect(bar(PB_SREADY + s), leader);
                    if (kt == ks.t1 - 1) ptx::tc_commit_elect(bar(PB_QFREE + s), leader);
                    end_run();
                }
                if (v) ptx::tc_commit_elect(bar(PB_FREE + v_stage), leader);
                if (k) ptx::tc_commit_elect(bar(PB_FREE + k_stage), leader);
                return true;
            });
        };
        phase(std::integral_constant<int, 1>()) && phase(std::integral_constant<int, 2>());
        // what was issued is complete, and has signalled, before the CTA can exit
        ptx::tc_commit_elect(bar(PB_FINAL), leader);
        ptx::mbar_wait(bar(PB_FINAL), 0);
    } else if (warp == PA_CLEAN_WARP) {
        // ------------------------------------------------------------ the last V tiles of a sequence
        int stage = 0, turns = 0, n_piece[2] = {0, 0};
        auto phase = [&](auto lists) {
            constexpr int NL = decltype(lists)::value;
            int n[NL] = {};
            return for_rounds<NL>([&](int l, PaPiece &s) { return take(NL == 1 ? 0 : 1 + l, n[l]++, s); }, [&](int l, bool v, const PaPiece &vs, int vt, bool k, const PaPiece &ks, int kt) {
                // Every entry is waited for, and handed back by this warp too (as above).
                auto landed = [&]() { return wait(PB_FULL + stage, turns & 1); };
                auto pass = [&]() {
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(PB_FREE + stage));
                    if (++stage == SM::STAGES) { stage = 0; ++turns; }
                };
                if (v && !landed()) return false;
                if (v && is_last(vs, vt)) {
                    // rows of the tree are looked through, those behind them on their page cleared (the pages behind are copied as zeros)
                    const int first = max(0, vs.L - vt * PA_KEYS), end = min(vs.L + p.T - vt * PA_KEYS, PA_KEYS);
                    const int clear = (end + p.page_rows - 1) / p.page_rows * p.page_rows;
                    bool odd = false;
#pragma unroll
                    for (int h = 0; h < SM::HALVES; ++h) {
                        uint4 *x = reinterpret_cast<uint4 *>(gbase + SM::OFF_RING + stage * SM::TILE + h * SM::HALF);
                        for (int e = end * 8 + lane; e < clear * 8; e += 32) x[e] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 4
                        for (int e = first * 8 + lane; e < end * 8; e += 32) {
                            const uint4 u = x[e];
                            // an exponent of all ones anywhere: the halves of a word side by side
                            auto ones = [](uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
                            if ((ones(u.x) | ones(u.y) | ones(u.z) | ones(u.w)) == 0u) continue;
                            uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (nonfinite16(w[i])) w[i] &= 0xffff0000u;
                                if (nonfinite16(w[i] >> 16)) w[i] &= 0xffffu;
                            }
                            x[e] = make_uint4(w[0], w[1], w[2], w[3]);
                            odd = true;
                        }
                    }
                    if (__any_sync(0xffffffffu, odd) && lane == 0)
                        for (int s = l; s < (NL == 1 ? 2 : l + 1); ++s) bad[s * 4 + (n_piece[s] & 3)] = n_piece[s] + 1;
                    ptx::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(PB_CLEAN + stage));
                }
                if (v) {
                    pass();
                    if (vt == vs.t1 - 1)
                        for (int s = l; s < (NL == 1 ? 2 : l + 1); ++s) ++n_piece[s];
                }
                if (k) {
                    if (!landed()) return false;
                    pass();
                }
                return true;
            });
        };
        phase(std::integral_constant<int, 1>()) && phase(std::integral_constant<int, 2>());
    } else {
        // ------------------------------------------------------------ softmax: thread (row, hf) of row tile s: columns [64 hf, 64 hf + 64)
        const int s = warp >> 3, hf = (warp >> 2) & 1, qd = warp & 3, row = qd * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(qd * 32) << 16);
        const uint32_t t_s = lane_base + s * 128 + hf * 64;      // this half's scores, and P over them
        const uint32_t t_x = lane_base + s * 128 + (hf ^ 1) * 64;
        const uint32_t t_o = lane_base + 256 + s * D + hf * (D / 2);
        const int pair_bar = 2 + s * 4 + qd;
        const int node_in_tile = row / p.G, head = row - node_in_tile * p.G;
        const bool in_tile = node_in_tile < p.npc;
        const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
        // what the other half of the row has: both put theirs where nothing is any more
        auto exchange = [&](int col, float v) {
            tmem_put(t_s + col, v);
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair_bar) : "memory");
            ptx::tc_fence_after();
            return tmem_get(t_x + col);
        };
        int n_s = 0, n_piece = 0;
        bool ok = true;
        for (int f = 0; f < 2 && ok; ++f) {
            const PaPhase &ph = p.phase[f];
            PaPiece pc;
            for (int n = 0; ok && take(f ? 1 + s : 0, n, pc); ++n) {
                const int node = (pc.tile0 + (f ? 0 : s)) * p.npc + node_in_tile;
                const bool mine = in_tile && node < (pc.b < 0 ? p.B * p.T : p.T);
                const bool some = __any_sync(0xffffffffu, mine);
                // visibility of the tree rows as 32-bit words; the rows in front of them are visible to every node, those behind to none
                uint4 anc = make_uint4(0u, 0u, 0u, 0u);
                if (mine && pc.b >= 0) anc = reinterpret_cast<const uint4 *>(p.anc)[node];
                auto anc_word = [&](int w) -> uint32_t { return w < 0 ? 0xffffffffu : w == 0 ? anc.x : w == 1 ? anc.y : w == 2 ? anc.z : w == 3 ? anc.w : 0u; };
                float m_used = -INFINITY, l = 0.f;
                for (int t = pc.t0; t < pc.t1; ++t) {
                    if (!wait(PB_SREADY + s, n_s++ & 1)) { ok = false; break; }
                    ptx::tc_fence_after();
                    if (some) {
                        uint32_t pk[32], rest[TWO ? 32 : 1];     // bf16 pairs; what their rounding left
                        float2 la, lb;
                        bool move = t == pc.t0;
                        for (;;) {
                            uint32_t sr[64];
                            ptx::tmem_ld32(t_s, *reinterpret_cast<uint32_t(*)[32]>(&sr[0]));
                            ptx::tmem_ld32(t_s + 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[32]));
                            ptx::tmem_ld_wait_for(*reinterpret_cast<uint32_t(*)[32]>(&sr[0]));
                            ptx::tmem_ld_wait_for(*reinterpret_cast<uint32_t(*)[32]>(&sr[32]));
                            if ((t + 1) * PA_KEYS > pc.L) {
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const int a0 = t * PA_KEYS + hf * 64 + h * 32 - pc.L;      // tree row of the first column
                                    const uint32_t vis = __funnelshift_r(anc_word(a0 >> 5), anc_word((a0 >> 5) + 1), a0 & 31);
#pragma unroll
                                    for (int e = 0; e < 32; ++e)
                                        if (!((vis >> e) & 1u)) sr[h * 32 + e] = 0xff800000u;   // -inf
                                }
                            }
                            if (move) {
                                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                                for (int e = 0; e < 64; e += 8)
#pragma unroll
                                    for (int k = 0; k < 4; ++k) mx[k] = max3_nan(mx[k], __uint_as_float(sr[e + 2 * k]), __uint_as_float(sr[e + 2 * k + 1]));
                                float mxs = max_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3]) * p.scale_log2;
                                mxs = max_nan(mxs, exchange(X_COL, mxs));
                                if (mxs == INFINITY) mxs = __int_as_float(0x7fffffff);     // inf - inf: the row is NaN, as from the formula
                                const float m_new = mxs <= m_used ? m_used : mxs;            // (a NaN is taken over)
                                const bool need = m_new != m_used && m_used != -INFINITY && mine;
                                if (__any_sync(0xffffffffu, need)) {
                                    const float alpha = need ? ex2(m_used - m_new) : 1.f;
#pragma unroll 1
                                    for (int h = 0; h < D / 32; ++h) {
                                        uint32_t o[16];
                                        ptx::tmem_ld16(t_o + h * 16, o);
                                        ptx::tmem_ld_wait_for16(o);
#pragma unroll
                                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                                        ptx::tmem_st16(t_o + h * 16, o);
                                    }
                                    l *= alpha;
                                }
                                m_used = m_new;
                            }
                            const float m_eff = m_used == -INFINITY ? 0.f : m_used;
                            const float2 nm2 = make_float2(-m_eff, -m_eff);
                            la = lb = make_float2(0.f, 0.f);
                            float px = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                const uint32_t *x = sr + 2 * e;
                                const float2 x01 = __ffma2_rn(make_float2(__uint_as_float(x[0]), __uint_as_float(x[1])), sc2, nm2);
                                const float2 x23 = __ffma2_rn(make_float2(__uint_as_float(x[2]), __uint_as_float(x[3])), sc2, nm2);
                                float2 p01, p23;
                                if (!TWO && e % 8 == 6) {   // every fourth quadruple on the FMA pipes: the special-function unit takes as long as the products
                                    // (with second terms the other pipes have more to do: 35.3 us without polynomials, 36.5 with, in the example above)
                                    px = max3_nan(max3_nan(px, x01.x, x01.y), x23.x, x23.y);   // (neither NaN nor what is above 127 survives there)
                                    p01 = exp2_poly2(x01);
                                    p23 = exp2_poly2(x23);
                                } else {
                                    p01 = make_float2(ex2(x01.x), ex2(x01.y));
                                    p23 = make_float2(ex2(x23.x), ex2(x23.y));
                                }
                                la = __fadd2_rn(la, p01);
                                lb = __fadd2_rn(lb, p23);
                                pk[e] = pack2_bf16(p01.x, p01.y);
                                pk[e + 1] = pack2_bf16(p23.x, p23.y);
                                if constexpr (TWO) {
                                    rest[e] = rounded_off(p01, pk[e]);
                                    rest[e + 1] = rounded_off(p23, pk[e + 1]);
                                }
                            }
                            if (move) break;
                            // a sum that is too large, infinite or NaN, and a row that has met no visible key yet
                            const bool ask = !(max_nan(max_nan(la.x, la.y), max_nan(lb.x, lb.y)) < 1.8446744e19f) || !(px <= PA_LIMIT) || m_used == -INFINITY;
                            if (!any_of_rows(pair_bar, mine && ask)) break;
                            move = true;
                        }
                        l += (la.x + la.y) + (lb.x + lb.y);
                        const bool last = t == pc.t1 - 1;
                        if constexpr (TWO) {
                            if (last) l += exchange(X_COL + 1, l);      // the row's sum
                            // (second terms go over what was exchanged when the other half has read it)
                            if (move || last) asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair_bar) : "memory");
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                ptx::tmem_st16(t_s + h * 32, *reinterpret_cast<uint32_t(*)[16]>(&pk[h * 16]));
                                ptx::tmem_st16(t_s + h * 32 + 16, *reinterpret_cast<uint32_t(*)[16]>(&rest[h * 16]));
                            }
                        } else {
                            ptx::tmem_st32(t_s, pk);
                            if (last) l += exchange(X_COL + 1, l);      // S is another tile's behind this one's P
                        }
                        ptx::tmem_st_wait();
                    }
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(PB_PREADY + s));
                }
                if (!ok || !wait(PB_ODONE + s, n_piece & 1)) { ok = false; break; }
                ptx::tc_fence_after();
                if (some) {
                    const bool odd = bad[s * 4 + (n_piece & 3)] == n_piece + 1;
                    const bool direct = p.shared == 0 && pc.whole;
                    const float inv = direct ? 1.f / l : 1.f;
                    const int slot_row = f ? row : s * 128 + row;
                    float *o_out = ph.o + ((size_t)pc.slot * ph.rows * (D / 8) + (size_t)(hf * (D / 16)) * ph.rows + slot_row) * 8;
                    __nv_bfloat16 *out = p.out + (((size_t)max(pc.b, 0) * p.T + node) * p.Hq + pc.g * p.G + head) * D + hf * (D / 2);
#pragma unroll 1
                    for (int h = 0; h < D / 32; ++h) {
                        uint32_t o[16];
                        ptx::tmem_ld16(t_o + h * 16, o);
                        ptx::tmem_ld_wait_for16(o);
                        if (!mine) continue;
                        if (odd) {
                            // V values that the tensor core did not see: an infinity or NaN with any weight is itself
                            for (int a = max(0, pc.t0 * PA_KEYS - pc.L); a < p.T && pc.L + a < pc.t1 * PA_KEYS; ++a) {
                                if (!(anc_word(a >> 5) >> (a & 31) & 1)) continue;
                                const int64_t at = p.pages.row(pc.b, p.shared + pc.L + a);
                                if (at < 0) continue;
                                const uint16_t *v = reinterpret_cast<const uint16_t *>(p.v) + at + pc.g * p.pages.stride_h + hf * (D / 2) + h * 16;
#pragma unroll
                                for (int e = 0; e < 16; ++e)
                                    if (nonfinite16(v[e])) o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float((uint32_t)v[e] << 16));
                            }
                        }
                        if (direct) {
                            uint32_t w[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) w[e] = pack2_bf16(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
                            *reinterpret_cast<uint4 *>(out + h * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                            *reinterpret_cast<uint4 *>(out + h * 16 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                        } else {
                            ptx::st_global_32(o_out + (size_t)(2 * h) * ph.rows * 8, *reinterpret_cast<const uint32_t(*)[8]>(&o[0]));
                            ptx::st_global_32(o_out + (size_t)(2 * h + 1) * ph.rows * 8, *reinterpret_cast<const uint32_t(*)[8]>(&o[8]));
                        }
                    }
                    if (mine && !direct && hf == 0) ph.ml[(size_t)pc.slot * ph.rows + slot_row] = make_float2(l == 0.f ? -INFINITY : m_used, l);
                }
                ++n_piece;
            }
        }
    }
    // ---- nobody leaves while the tensor core may still work for the CTA
    __syncwarp();
    ptx::tc_fence_before();
    pa_cta_sync();
    ptx::tc_fence_after();
    if (warp == PA_MMA_WARP) ptx::tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------------------------------- thin items
// At most 16 query rows against a KV head's keys (plain decoding; the smallest trees): nothing but the bytes of K and V counts, and a row tile of
// 128 would be nearly empty, its ring full of tiles that wait for each other's scores.  So these items go to warps of their own: mma.sync
// with 16 rows, K and V straight from global memory into the operand registers, no shared memory in between.  A contraction's order
// is free as long as both operands have it, and so is the order of O's columns: a thread takes 16-byte chunks of K as two products' B operands, and 32
// bytes of a V row as its column in 16 products, two keys' values side by side by a byte permutation.
// A CTA of four warps walks a run of the line of all thin items, 16 keys to a warp at a time; while a warp computes on 16 keys, V of them and K
// of its next ones are on the way (8 KB a warp, two CTAs to an SM).  At a piece's end the warps join in shared memory.
// Measured: 64 single tokens, 8 KV heads of 128, 100 to 1000 keys each: 149 MB in 37 us = 4.0 TB/s.  Bound by the bytes in flight, 64 KB an SM
// (V of a block is requested in the iteration that uses it, only K is ahead); 218 registers a thread leave no third CTA (with spills: 89 us instead of 61 in one comparison), and more or shorter pieces change nothing (62, 60).
constexpr int TH_WARPS = 4, TH_KEYS = 16, TH_STEP = TH_WARPS * TH_KEYS;
constexpr int TH_ENDS = 3;                // what an item's start and end take, in steps of 64 keys

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ int thin_steps(int keys) { return (keys + TH_STEP - 1) / TH_STEP; }

template <int D>
__global__ void __launch_bounds__(TH_WARPS * 32, 2)
paged_attn_thin_kernel(const __grid_constant__ PaParams p) {
    constexpr int C = D / 32;              // 32-column parts of a row
    constexpr int J = D / 8;               // products of 8 columns of O
    __shared__ float o_x[TH_WARPS][TH_ROWS][D + 4];
    __shared__ float2 ml_x[TH_WARPS][TH_ROWS];
    __shared__ int start[5];               // x0, x1, S, b, idx
    let_next_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r0 = lane / 4, quad = lane % 4;
    const PaPhase &ph = p.phase[2];
    const int worker = blockIdx.x, workers = gridDim.x;
    previous_done();
    auto cost_of = [&](int b) {
        const int L = b < p.B ? p.seq_lens[b] : -1;
        return L >= 0 && p.pages.fits(L, p.T) && L >= p.shared ? thin_steps(L - p.shared + p.T) + TH_ENDS : 0;
    };
    if (warp == 0) {
        const int own0 = cost_of(lane);
        int total = own0;
        for (int b0 = 32; b0 < p.B; b0 += 32) total += cost_of(b0 + lane);
        total = __reduce_add_sync(0xffffffffu, total);
        const int each = thin_steps(p.shared) + TH_ENDS, prefix = ph.prefix_items * each, length = prefix + total * ph.seq_items;
        const int run = max((length + workers - 1) / workers, 1), x0 = (int)min((int64_t)length, (int64_t)run * worker), x1 = (int)min((int64_t)length, (int64_t)x0 + run);
        int b = -1, idx = 0, S = x1;
        if (x0 < x1 && x0 < prefix) {
            idx = x0 / each;
            S = idx * each;
        } else if (x0 < x1) {
            const int y = x0 - prefix;
            int before = 0;
            for (int b0 = 0; b0 < p.B; b0 += 32) {
                const int own = b0 ? cost_of(b0 + lane) : own0;
                int c = own;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int x = __shfl_up_sync(0xffffffffu, c, o);
                    if (lane >= o) c += x;
                }
                const uint32_t behind = __ballot_sync(0xffffffffu, (before + c) * ph.seq_items > y);
                if (behind) {
                    const int at = __ffs((int)behind) - 1, cost = __shfl_sync(0xffffffffu, own, at);
                    const int first = (before + __shfl_sync(0xffffffffu, c, at) - cost) * ph.seq_items;
                    b = b0 + at;
                    idx = (y - first) / cost;
                    S = prefix + first + idx * cost;
                    break;
                }
                before += __shfl_sync(0xffffffffu, c, 31);
            }
        }
        if (lane == 0) { start[0] = x0; start[1] = x1; start[2] = S; start[3] = b; start[4] = idx; }
    }
    __syncthreads();
    const int x0 = start[0], x1 = start[1];
    int S = start[2], b = start[3], idx = start[4];
    int L = 0, cost = 0;                   // keys of the item (prefix: the shared ones; else its own in front of the tree)
    auto load_item = [&]() {
        if (b < 0) {
            L = p.shared;
            cost = thin_steps(p.shared) + TH_ENDS;
        } else {
            cost = cost_of(b);
            L = p.seq_lens[b] - p.shared;
        }
    };
    if (x0 < x1) load_item();
    while (S < x1) {
        if (idx >= (b < 0 ? ph.prefix_items : ph.seq_items) || cost == 0) {
            if (++b >= p.B) break;
            idx = 0;
            load_item();
            continue;
        }
        const int steps = cost - TH_ENDS;
        const int t0 = max(0, min(x0 - S - TH_ENDS, steps)), t1 = max(0, min(x1 - S - TH_ENDS, steps));
        S += cost;
        const int g = idx++;
        if (t0 >= t1) continue;
        const int item = b < 0 ? g : ph.prefix_items + b * ph.seq_items + g;
        const bool own = b >= 0;
        const int n_keys = L + (own ? p.T : 0), key0 = own ? p.shared : 0, rows = (own ? p.T : p.B * p.T) * p.G;
        if (threadIdx.x == 0) {
            if (t0 == 0) ph.span[item].x = worker;
            if (t1 == steps) ph.span[item].y = worker;
        }
        // ---- the query rows as A operands: columns c * 32 + quad * 8 + [0, 4) and [4, 8) of rows r0 and r0 + 8
        uint32_t qa[C][2][4];
        uint32_t see[2];                   // tree rows that are visible to rows r0 and r0 + 8 (at most 16 nodes)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = r0 + 8 * h, n = r / p.G;
            const bool is = r < rows;
            const __nv_bfloat16 *src = p.q + (((size_t)(own ? b * p.T : 0) + n) * p.Hq + g * p.G + (r - n * p.G)) * D + quad * 8;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 u = is ? *reinterpret_cast<const uint4 *>(src + c * 32) : make_uint4(0u, 0u, 0u, 0u);
                qa[c][0][h] = u.x; qa[c][0][h + 2] = u.y;
                qa[c][1][h] = u.z; qa[c][1][h + 2] = u.w;
            }
            see[h] = is && own ? (uint32_t)p.anc[n * 2] : 0u;
        }
        float o[J][4] = {}, m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        // ---- this warp's blocks of 16 keys: key (t * TH_WARPS + warp) * 16
        const int32_t *table = p.pages.table + (int64_t)max(b, 0) * p.pages.max_pages;
        auto block_key = [&](int t) { return (t * TH_WARPS + warp) * TH_KEYS; };
        auto page_of = [&](int t) { return t < t1 && block_key(t) < n_keys ? table[(block_key(t) + key0) >> p.pages.page_shift] : -1; };
        auto row_at = [&](int t, int id) {     // element offset of the block's first row; < 0: there is none
            return id < 0 || id >= p.pages.n_pages ? -1ll
                   : (long long)id * p.pages.stride_page + (long long)((block_key(t) + key0) & ((1 << p.pages.page_shift) - 1)) * p.pages.stride_t +
                         g * p.pages.stride_h;
        };
        uint4 kx[2][C];                    // keys r0 and r0 + 8 of the block
        auto load_k = [&](long long at) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    kx[h][c] = at >= 0 ? __ldg(reinterpret_cast<const uint4 *>(p.k + at + (r0 + 8 * h) * p.pages.stride_t + c * 32 + quad * 8)) : make_uint4(0u, 0u, 0u, 0u);
        };
        int id = page_of(t0), id_next = page_of(t0 + 1);
        long long at = row_at(t0, id);
        load_k(at);
        for (int t = t0; t < t1; ++t) {
            const int first = block_key(t);
            if (first >= n_keys) break;    // (the item's last step: no keys for this warp)
            // V of keys 2 quad, 2 quad + 1 and the same + 8: columns r0 * (D / 8) + [0, D / 8)
            uint32_t vx[4][J / 2];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int key = 2 * quad + (k & 1) + 8 * (k >> 1);
                const uint4 *src = reinterpret_cast<const uint4 *>(p.v + at + key * p.pages.stride_t + r0 * J);
                const bool is = at >= 0 && first + key < n_keys;     // rows behind the last key may hold anything
#pragma unroll
                for (int c = 0; c < J / 8; ++c) {
                    const uint4 u = is ? __ldg(src + c) : make_uint4(0u, 0u, 0u, 0u);
                    vx[k][c * 4] = u.x; vx[k][c * 4 + 1] = u.y; vx[k][c * 4 + 2] = u.z; vx[k][c * 4 + 3] = u.w;
                }
            }
            // ---- scores of keys [0, 8) and [8, 16): c0, c1 row r0, c2, c3 row r0 + 8, keys 2 quad and 2 quad + 1
            float sc[2][4] = {};
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    mma16816(sc[h], qa[c][0], kx[h][c].x, kx[h][c].y);
                    mma16816(sc[h], qa[c][1], kx[h][c].z, kx[h][c].w);
                }
            const long long at_now = at;
            id = id_next;
            id_next = page_of(t + 2);
            at = row_at(t + 1, id);
            if (t + 1 < t1) load_k(at);    // on its way during the rest
            const bool edge = first + TH_KEYS > L;
            if (edge) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int a = first + 8 * h + 2 * quad + (e & 1) - L;
                        if (a >= 0 && (!own || a >= p.T || !(see[e >> 1] >> a & 1u))) sc[h][e] = -INFINITY;
                    }
            }
            float mx[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                mx[h] = max_nan(max_nan(sc[0][2 * h], sc[0][2 * h + 1]), max_nan(sc[1][2 * h], sc[1][2 * h + 1]));
                mx[h] = max_nan(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
                mx[h] = max_nan(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2)) * p.scale_log2;
                if (mx[h] == INFINITY) mx[h] = __int_as_float(0x7fffffff);     // inf - inf: the row is NaN, as from the formula
            }
            if (__any_sync(0xffffffffu, !(mx[0] <= m[0] + 8.f) || !(mx[1] <= m[1] + 8.f))) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float m_new = mx[h] <= m[h] ? m[h] : mx[h];
                    const float w = m[h] == -INFINITY ? 0.f : ex2(m[h] - m_new);
                    m[h] = m_new;
                    l[h] *= w;
#pragma unroll
                    for (int j = 0; j < J; ++j) { o[j][2 * h] *= w; o[j][2 * h + 1] *= w; }
                }
            }
            const float me[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
            uint32_t pa[4], rest[4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float w0 = ex2(fmaf(sc[h][2 * r], p.scale_log2, -me[r])), w1 = ex2(fmaf(sc[h][2 * r + 1], p.scale_log2, -me[r]));
                    l[r] += w0 + w1;
                    pa[h * 2 + r] = pack2_bf16(w0, w1);
                    rest[h * 2 + r] = rounded_off(make_float2(w0, w1), pa[h * 2 + r]);
                }
            bool odd = false;
            if (edge && own) {
                // values of the tree's rows that are not finite are left out here and given below to the rows that see them
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int e = 0; e < J / 2; ++e) {
                        if (nonfinite16(vx[k][e])) { vx[k][e] &= 0xffff0000u; odd = true; }
                        if (nonfinite16(vx[k][e] >> 16)) { vx[k][e] &= 0xffffu; odd = true; }
                    }
                odd = __any_sync(0xffffffffu, odd);
            }
#pragma unroll
            for (int j = 0; j < J; j += 2) {
                const uint32_t a0 = __byte_perm(vx[0][j / 2], vx[1][j / 2], 0x5410), a1 = __byte_perm(vx[2][j / 2], vx[3][j / 2], 0x5410);
                const uint32_t b0 = __byte_perm(vx[0][j / 2], vx[1][j / 2], 0x7632), b1 = __byte_perm(vx[2][j / 2], vx[3][j / 2], 0x7632);
                mma16816(o[j], pa, a0, a1);
                mma16816(o[j + 1], pa, b0, b1);
                mma16816(o[j], rest, a0, a1);
                mma16816(o[j + 1], rest, b0, b1);
            }
            if (odd && at_now >= 0)
                for (int k = 0; k < TH_KEYS; ++k) {
                    const int a = first + k - L;
                    if (a >= p.T) break;
#pragma unroll
                    for (int j = 0; j < J; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint16_t x = *reinterpret_cast<const uint16_t *>(p.v + at_now + k * p.pages.stride_t + (2 * quad + (e & 1)) * J + j);
                            // (the shared keys and those in front of the tree are seen by all)
                            if (nonfinite16(x) && (a < 0 || (see[e >> 1] >> a & 1u))) o[j][e] += __uint_as_float((uint32_t)x << 16);
                        }
                }
        }
        // ---- the four warps' shares of a row are joined: O[row][column (2 quad + (e & 1)) * J + j]
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (quad == 0) ml_x[warp][r0 + 8 * h] = make_float2(m[h], l[h]);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                o_x[warp][r0 + 8 * h][2 * quad * J + j] = o[j][2 * h];
                o_x[warp][r0 + 8 * h][(2 * quad + 1) * J + j] = o[j][2 * h + 1];
            }
        }
        __syncthreads();
        const bool direct = p.shared == 0 && t1 - t0 == steps;      // the item's only piece
        const size_t slot = (size_t)item + worker;
        for (int e = threadIdx.x; e < rows * (D / 8); e += TH_WARPS * 32) {
            const int row = e % rows, chunk = e / rows;
            float mm = -INFINITY;
#pragma unroll
            for (int w = 0; w < TH_WARPS; ++w) mm = max_nan(mm, ml_x[w][row].x);
            float acc[8] = {}, ll = 0.f;
#pragma unroll
            for (int w = 0; w < TH_WARPS; ++w) {
                const float2 ml = ml_x[w][row];
                const float x = ml.x == -INFINITY ? 0.f : ex2(ml.x - mm);
                ll = fmaf(x, ml.y, ll);
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] = fmaf(x, o_x[w][row][chunk * 8 + k], acc[k]);
            }
            if (direct) {
                const float inv = 1.f / ll;
                const int n = row / p.G;
                *reinterpret_cast<uint4 *>(p.out + (((size_t)b * p.T + n) * p.Hq + g * p.G + row - n * p.G) * D + chunk * 8) =
                    make_uint4(pack2_bf16(acc[0] * inv, acc[1] * inv), pack2_bf16(acc[2] * inv, acc[3] * inv), pack2_bf16(acc[4] * inv, acc[5] * inv),
                               pack2_bf16(acc[6] * inv, acc[7] * inv));
            } else {
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(acc[k]);
                ptx::st_global_32(ph.o + ((slot * (D / 8) + chunk) * TH_ROWS + row) * 8, w);
                if (chunk == 0) ph.ml[slot * TH_ROWS + row] = make_float2(ll == 0.f ? -INFINITY : mm, ll);
            }
        }
        __syncthreads();                   // before the next piece's shares
    }
}

// ---------------------------------------------------------------------------------------- their combination
// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s over the pieces s of a row's two items (the prefix' and the sequence's own).  A thread takes
// 8 columns of a row, neighbouring threads neighbouring rows, as the slots are laid out, and four pieces at a time, their
// (max, sum) and their columns requested together: the kernel is a chain of loads from L2.  SPLIT > 1: that many threads share a row's columns,
// each every SPLIT-th group of four pieces, and meet in shared memory; the order of the additions depends on the pieces alone.
struct PaSource {
    const float *o;       // slot of the first piece, at the row
    const float2 *ml;
    int n, rows;
};
struct PaSum {
    float m, l, acc[8];
    __device__ __forceinline__ void add(float m2, float l2, const float (&a)[8]) {
        const float m_new = max_nan(m, m2);
        const float w = m == -INFINITY ? 0.f : ex2(m - m_new), w2 = m2 == -INFINITY ? 0.f : ex2(m2 - m_new);
        m = m_new;
        l = fmaf(w2, l2, w * l);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w2, a[e], w * acc[e]);
    }
};

template <int D, int SPLIT>
__global__ void __launch_bounds__(256)
paged_attn_combine_kernel(const __grid_constant__ PaParams p) {
    constexpr int CHUNKS = D / 8, ROWS = 256 / (CHUNKS * SPLIT);
    __shared__ PaSource src[2][ROWS];
    __shared__ int64_t out_at[ROWS];
    __shared__ PaSum sums[SPLIT > 1 ? 256 : 1];
    let_next_start();
    const int tid = threadIdx.x, per_seq = p.T * p.G;
    int b = p.B, g = 0, node = 0, head = 0;
    if (tid < ROWS) {
        const int r = (int)blockIdx.x * ROWS + tid, bg = r / per_seq, x = r - bg * per_seq;
        b = bg / p.Hkv; g = bg - b * p.Hkv; node = x / p.G; head = x - node * p.G;
    }
    // row tile and row in it -> phase, item and row of the slot
    auto place = [&](int n, bool prefix, int *item, int *row) -> const PaPhase & {
        const bool thin = prefix ? p.phase[2].prefix_items : p.phase[2].seq_items;
        const int tile = n / p.npc, per = prefix ? p.phase[0].prefix_per_head : p.phase[0].seq_per_head;
        const int k = thin ? 2 : tile / 2 < per ? 0 : 1;
        const PaPhase &f = p.phase[k];
        *row = thin ? n * p.G + head : (k ? 0 : (tile & 1) * 128) + (n - tile * p.npc) * p.G + head;
        const int i = k ? g : g * per + tile / 2;
        *item = prefix ? i : f.prefix_items + b * f.seq_items + i;
        return f;
    };
    previous_done();
    // which sequences can be attended to, a warp each
    if (p.status && (int)blockIdx.x * 8 < p.B) {
        const int b2 = (int)blockIdx.x * 8 + tid / 32, lane = tid % 32;
        if (b2 < p.B) {
            const int len = p.seq_lens[b2];
            int code = seq_tiles(p, len) ? p.pages.check(b2, p.shared, len - p.shared + p.T, lane) : MTV_ERR_CAPACITY;
            if (code == MTV_OK) code = p.pages.check(0, 0, p.shared, lane);
            if (lane == 0) p.status[b2] = code;
        }
    }
    if (tid < ROWS) {
        int64_t at = -1;
        PaSource s0 = {}, s1 = {};
        if (b < p.B) {
            int item0 = 0, row0 = 0, item1, row1;
            const PaPhase &f0 = place(b * p.T + node, true, &item0, &row0), &f1 = place(node, false, &item1, &row1);
            const int len = p.seq_lens[b];
            int2 span0 = make_int2(0, -1);
            if (p.shared) span0 = f0.span[item0];
            const int2 span1 = f1.span[item1];           // (of a sequence that is left out: not looked at)
            auto source = [&](const PaPhase &f, int item, int row, int2 span) {
                const size_t slot = (size_t)item + span.x;
                return PaSource{f.o + (slot * CHUNKS * f.rows + row) * 8, f.ml + slot * f.rows + row, span.y - span.x + 1, f.rows};
            };
            if (seq_tiles(p, len) && (!p.shared || pa_span_ok(f0, span0)) && pa_span_ok(f1, span1)) {
                if (p.shared) s0 = source(f0, item0, row0, span0);
                s1 = source(f1, item1, row1, span1);
                // a single piece was written out by the kernel before
                if (p.shared || s1.n > 1) at = (((int64_t)b * p.T + node) * p.Hq + g * p.G + head) * D;
            }
        }
        src[0][tid] = s0;
        src[1][tid] = s1;
        out_at[tid] = at;
    }
    __syncthreads();
    const int row = tid % ROWS, chunk = tid / ROWS % CHUNKS, part = tid / (ROWS * CHUNKS);
    PaSum sum = {-INFINITY, 0.f, {}};
    if (out_at[row] >= 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const PaSource s = src[k][row];
            for (int i0 = part * 4; i0 < s.n; i0 += SPLIT * 4) {
                float2 ml[4];
                float4 a[4], c[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = min(i0 + u, s.n - 1);
                    const float4 *o = reinterpret_cast<const float4 *>(s.o + ((size_t)i * CHUNKS + chunk) * s.rows * 8);
                    ml[u] = s.ml[(size_t)i * s.rows];
                    a[u] = o[0];
                    c[u] = o[1];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i0 + u < s.n) sum.add(ml[u].x, ml[u].y, {a[u].x, a[u].y, a[u].z, a[u].w, c[u].x, c[u].y, c[u].z, c[u].w});
            }
        }
    }
    if (SPLIT > 1) {
        sums[tid] = sum;
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int k = 1; k < SPLIT; ++k) sum.add(sums[tid + k * ROWS * CHUNKS].m, sums[tid + k * ROWS * CHUNKS].l, sums[tid + k * ROWS * CHUNKS].acc);
    }
    if (out_at[row] < 0) return;
    const float inv = 1.f / sum.l;
    const float *acc = sum.acc;
    *reinterpret_cast<uint4 *>(p.out + out_at[row] + chunk * 8) = make_uint4(pack2_bf16(acc[0] * inv, acc[1] * inv), pack2_bf16(acc[2] * inv, acc[3] * inv),
                                                                            pack2_bf16(acc[4] * inv, acc[5] * inv), pack2_bf16(acc[6] * inv, acc[7] * inv));
}

// ---------------------------------------------------------------------------------------- host
static bool pa_sizes_ok(const mtv_tree *tree, int B, int Hq, int Hkv, int D, int shared) {
    return tree && B >= 1 && B <= PA_MAX_B && Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0 && Hq / Hkv <= 8 && (D == 64 || D == 128) && shared >= 0 &&
           (int64_t)Hq * B * tree->T <= 1 << 28;
}
// All lines stay below 2^31, whatever the lengths.
static bool pa_lines_ok(const PaPhase (&ph)[3], int B, int shared, int64_t slots) {
    for (const PaPhase &f : ph) {
        // (a thin item's steps are of 64 keys and count one)
        const int64_t ends = ITEM_COST(0), prefix = (shared / PA_KEYS + 1) * TILE_COST + ends, own = (slots / PA_KEYS + 2) * TILE_COST + ends;
        if (own * B > 0x7fffffff || prefix > 0x7fffffff) return false;
        if ((double)prefix * f.prefix_items + (double)own * B * f.seq_items > 2147000000.0) return false;
    }
    return true;
}

template <int D>
static int launch_paged(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const PaParams &p, cudaStream_t stream) {
    static PerDeviceOnce once;
    bool *done = once.flag();
    if (!done || !*done) {
        MTV_CUDA_CHECK(cudaFuncSetAttribute(paged_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, PaSmem<D>::TOTAL));
        if (done) *done = true;
    }
    const PaPhase &thin = p.phase[2];
    if (p.phase[0].prefix_items + p.phase[0].seq_items + p.phase[1].prefix_items + p.phase[1].seq_items)
        MTV_CUDA_CHECK(launch_dependent(paged_attn_kernel<D>, dim3(sm_count()), PA_THREADS, PaSmem<D>::TOTAL, stream, q, k, v, p));
    if (thin.prefix_items + thin.seq_items)
        MTV_CUDA_CHECK(launch_dependent(paged_attn_thin_kernel<D>, dim3(2 * sm_count()), TH_WARPS * 32, 0, stream, p));
    const int64_t rows = (int64_t)p.B * p.Hkv * p.T * p.G;
    // Fewer blocks than SMs with a thread per row and chunk (decoding: few rows, each of many pieces): four threads share one.  Whole calls on one card, D = 128
    // (D = 64 goes by the same rule, not measured): 2048 rows (128 blocks) 77 us so and 86 with one thread; 5684 rows (356 blocks) 37.9 and 34.6; 16384 rows 167 and 153.
    constexpr int PER = 256 / (D / 8);
    if (rows < (int64_t)PER * sm_count())
        MTV_CUDA_CHECK(launch_dependent(paged_attn_combine_kernel<D, 4>, dim3((unsigned)((rows + PER / 4 - 1) / (PER / 4))), 256, 0, stream, p));
    else
        MTV_CUDA_CHECK(launch_dependent(paged_attn_combine_kernel<D, 1>, dim3((unsigned)((rows + PER - 1) / PER)), 256, 0, stream, p));
    return MTV_OK;
}

}  // namespace mtv

extern "C" size_t tree_attention_paged_workspace_bytes(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int shared_len) {
    using namespace mtv;
    if (!pa_sizes_ok(tree, B, Hq, Hkv, D, shared_len)) return 0;
    PaPhase ph[3];
    return pa_plan(ph, sm_count(), tree->T, B, Hq / Hkv, Hkv, D, shared_len, nullptr);
}

extern "C" int tree_verify_attention_paged(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, const mtv_bf16 *q, const mtv_bf16 *k_pool,
                                           const mtv_bf16 *v_pool, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                           int shared_len, const int32_t *seq_lens, float scale, mtv_bf16 *out, int32_t *status,
                                           void *ws, size_t ws_bytes, void *stream) {
    using namespace mtv;
    MTV_RANGE("tree_verify_attention_paged");
    if (!tree || !tree->on_device || !q || !k_pool || !v_pool || !seq_lens || !out || !ws) return MTV_ERR_INVALID_ARG;
    if (B < 1 || Hq < 1 || Hkv < 1 || shared_len < 0 || !(scale >= 0.f) || scale > 1e30f) return MTV_ERR_INVALID_ARG;
    if (!pa_sizes_ok(tree, B, Hq, Hkv, D, shared_len)) return MTV_ERR_UNSUPPORTED_SHAPE;
    PaParams p = {};
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D);
    if (rc != MTV_OK) return rc;
    if (shared_len % pool->page_size || shared_len > (int64_t)max_pages * pool->page_size || (((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_pool | (uintptr_t)v_pool) & 15) || ((uintptr_t)ws & 255))
        return MTV_ERR_INVALID_ARG;
    p.T = tree->T; p.B = B; p.G = Hq / Hkv; p.Hq = Hq; p.Hkv = Hkv;
    p.shared = shared_len;
    if (ws_bytes < pa_plan(p.phase, sm_count(), p.T, B, p.G, Hkv, D, shared_len, static_cast<char *>(ws))) return MTV_ERR_WORKSPACE;
    if (!pa_lines_ok(p.phase, B, shared_len, (int64_t)max_pages * pool->page_size)) return MTV_ERR_UNSUPPORTED_SHAPE;
    p.npc = 128 / p.G;
    p.page_rows = pool->page_size < PA_KEYS ? pool->page_size : PA_KEYS;
    p.seq_lens = seq_lens; p.anc = tree->d_anc;
    p.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    p.k = reinterpret_cast<const __nv_bfloat16 *>(k_pool);
    p.v = reinterpret_cast<const __nv_bfloat16 *>(v_pool);
    p.out = reinterpret_cast<__nv_bfloat16 *>(out);
    p.status = status; p.dev_error = tree->d_error;
    p.scale_log2 = (scale == 0.f ? 1.f / sqrtf((float)D) : scale) * 1.4426950408889634f;
    CUtensorMap q_map, k_map, v_map;
    {
        const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)Hq, (cuuint64_t)B * p.T, 1};
        const cuuint64_t str[3] = {(cuuint64_t)D * 2, (cuuint64_t)Hq * D * 2, (cuuint64_t)B * p.T * Hq * D * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)p.G, (cuuint32_t)p.npc, 1};
        if (!encode_map_bf16(&q_map, q, 4, dims, str, box)) return MTV_ERR_CUDA;
    }
    {
        const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)pool->page_size, (cuuint64_t)Hkv, (cuuint64_t)pool->n_pages};
        const cuuint64_t str[3] = {(cuuint64_t)pool->stride_t * 2, (cuuint64_t)pool->stride_h * 2, (cuuint64_t)pool->stride_page * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)p.page_rows, 1, 1};
        if (!encode_map_bf16(&k_map, k_pool, 4, dims, str, box) || !encode_map_bf16(&v_map, v_pool, 4, dims, str, box)) return MTV_ERR_CUDA;
    }
    return D == 128 ? launch_paged<128>(q_map, k_map, v_map, p, (cudaStream_t)stream) : launch_paged<64>(q_map, k_map, v_map, p, (cudaStream_t)stream);
}
