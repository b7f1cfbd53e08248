// Tree attention over pages of e4m3 codes (Section 3.2 / Fig. 2(b); the paper's cache is bf16): the division into items, pieces and phases, the joining
// and the workspace are those of the bf16 cache (attention_paged.cu, paged_attn.cuh); here stands what the codes change.
//   s_ij = (scale k_scale) <q_i, K8_j>,  out_i = v_scale sum_j softmax(s_i)_j V8_j
//
// K needs no conversion: its codes are operands of the 8-bit products.  Queries are brought to 8 bits in two terms, q = q1 + q2, both e4m3, which
// holds the 8 bits of a bf16 exactly: a row is multiplied by the power of two that brings its largest value to [128, 256), q1 is that rounded to a code
// and q2 what is left; values below 2^-9 of the row's largest are held to 2^-17 of it.  Two products of 8 bits take the time of one of 16.
// Weights would want two terms too, at every key tile, on the warps that have the least time; so V is converted instead, to fp16 tiles
// (every code is a number of fp16), by warps of their own, and the second product is fp16 x fp16.  (With K converted as well, those warps were what single
// row tiles waited for: 16 trees of 29 nodes and up to 4000 keys took 106 us so and 60 without, in the form of the kernel that this was measured in; 46 now.)
//   P   weights are fp16, 2^SHIFT at the reference (the maximum of a piece's first tile) and below 2^16: they lose bits below 2^(-14 - SHIFT) of the
//       reference and vanish below 2^(-25 - SHIFT).  11 bits, where bf16 has 8: no second term is needed at any head size.  The reference moves where a
//       later tile's weights do not fit, as for the bf16 cache.
//
// One persistent CTA per SM, two row tiles in flight, each with its scores, weights and accumulator in tensor memory and eight softmax warps:
//   warps 0-7 / 8-15  softmax of row tile 0 / 1; in front of a piece they split its queries
//   warps 16-19       V's codes -> fp16 tiles (128 keys, 128-byte swizzle); rows behind the last key become zeros (their weight is 0, but 0 * NaN is
//                     not), NaN codes of the tree's rows too (they are given to the rows that see them at the end)
//   warps 20, 21      issue the products of row tile 0 / 1.  As for the bf16 cache, a key tile's scores go over the weights of the tile before, which the product
//                     issued in front of them reads, with no wait between: products that one thread issues are carried out in the order in which it issues
//                     them.  Here the two differ in kind (fp16 in front of 8 bits) and in their accumulators; the order is counted on all the same.
//   warp 22           derives the pieces, requests Q and the codes (a box per page)
// K's codes, V's and V's tiles have a ring each.  A CTA works on pairs of row tiles or on single ones, never on both, and every warp's loop stands once for
// either (in_turns): the kernel would else be 193 KB of code, of which an SM's instruction cache holds a part (71 KB; that step took the same 16 trees of 29 from
// 93 to 73 us).  Sixteen scores of a row are in registers at a time, the next on their way: with all 64 the 80 registers of 768 threads spill (that step took the
// long context from 97 to 85 us; 12 bytes stored and 8 loaded a thread are left at D = 128, 20 and 40 at D = 64).
// The two warps that share a row's threads (columns) meet at named barriers, which have no limit: a wait of one of them that runs out is followed as in_step.cuh says.
//
// Measured, whole calls: one tree of 64 nodes, 32 / 8 heads of 128, 60001 keys (63 GFLOP): 77 us; 8 sequences of 64 nodes, 16384 shared keys and up to 2048 of
// their own (147 GFLOP): 153 us, the tensor pipe at 58 % beside the joining (replayed graphs over the same inputs: 64 and 131).  A pair of key tiles takes some
// 3.1 k cycles of the 2.06 k that its products need: the
// chain scores -> weights (1.9 k) -> product (1.3 k from the last weight to the next scores) of a row tile is hidden by the other row tile's alone.
// Looked at and left (us, or the kernel's cycles, of the latter case, each beside the form of the kernel that it was tried in): the warps of both row tiles on each in turn (32 columns a thread: 299 us where 64 took
// 171); halves of key tiles in turn (64 keys a product of scores, 189 us: the queries are read twice as often from shared memory, which is what bounds those
// products); no turns between the issuing warps (192 us); turns passed in the middle of the other tile's softmax (cycles + 15 %); fewer polynomials (+ 4 %),
// more (+ 9 %), other places for them (+ 4 %); waits that poll without suspending (+ 5 %: the issue slots they take are the softmax's); products in loops
// (159 us for 143); weights stored as they come, and the scores computed once more where a weight does not fit, in place of the vote (+ 7 %: the issuing warps
// have more to look at between the weights and the products).
#include <float.h>
#include <limits.h>

#include "fp8.cuh"
#include "in_step.cuh"
#include "paged_attn.cuh"

namespace mtv {

constexpr int P8_THREADS = 768;
constexpr int P8_CONV_WARP = 16, P8_CONV_WARPS = 4, P8_MMA_WARP = 20, P8_TMA_WARP = 22;
constexpr float P8_SHIFT = 8.f, P8_LIMIT = 15.99f;     // weights stay below 2^16, which fp16 ends at

template <int D> struct P8Smem {
    static constexpr int HALVES = D / 64;
    static constexpr uint32_t HALF = 128 * 128;          // 128 rows of 128 bytes (64 columns of 2, or 128 of 1), 128-byte swizzle
    static constexpr uint32_t TILE = HALVES * HALF, CODES = 128 * D;
    static constexpr int K_STAGES = D == 128 ? 4 : 8, V_STAGES = D == 128 ? 2 : 8, TILES = D == 128 ? 2 : 4;
    static constexpr uint32_t OFF_K = 2 * TILE, OFF_V = OFF_K + K_STAGES * CODES, OFF_TILES = OFF_V + V_STAGES * CODES, OFF_ROWS = OFF_TILES + TILES * TILE,
                              OFF_BAR = OFF_ROWS + 2048, TOTAL = OFF_BAR + 960;
    static_assert(TOTAL <= 227 * 1024, "shared memory budget");
    static constexpr uint32_t IDESC = (1u << 4) | (128u >> 4) << 24;                             // e4m3 x e4m3 or fp16 x fp16 -> fp32, M = 128
    static constexpr uint32_t IDESC_QK = IDESC | (128u >> 3) << 17;                               // N = 128 keys
    static constexpr uint32_t IDESC_PV = IDESC | (uint32_t)(D >> 3) << 17 | 1u << 16;             // N = D columns, B (= V) N-major
    // K's codes: rows of D bytes in groups of 8, swizzled over as many bytes
    static constexpr uint32_t K_DESC_HI = D == 128 ? ptx::DESC_HI : (512u >> 4) | 1u << 14 | 4u << 29;
};

enum {
    P8_KFULL = 0, P8_KFREE = 8, P8_VFULL = 16, P8_VFREE = 24, P8_FULL = 32, P8_FREE = 36, P8_QFULL = 40, P8_QREADY = 42, P8_QFREE = 44, P8_SREADY = 46,
    P8_PREADY = 48, P8_ODONE = 50, P8_FINAL = 52,
    P8_PIECE = 53,                         // [2 queues][PA_QUEUE]: pairs, or single tiles of one half of the CTA; those of the other half
    P8_TAKEN = P8_PIECE + 2 * PA_QUEUE,
    P8_TURN = P8_TAKEN + 2 * PA_QUEUE,     // [2] an issuing warp's turn at the tensor core
    P8_ROLE = P8_TURN + 2,                 // whether the CTA has pairs is known
    P8_COUNT = P8_ROLE + 1
};
constexpr uint32_t P8_OFF_MISC = P8_COUNT * 8, P8_OFF_QUEUE = (P8_OFF_MISC + 44 + 15) / 16 * 16;
static_assert(P8_OFF_QUEUE + 2 * PA_QUEUE * 32 <= 960, "barrier region");
static_assert(P8Smem<64>::K_STAGES <= 8 && P8Smem<64>::V_STAGES <= 8 && P8Smem<64>::TILES <= 4, "barriers of the rings");

// What a quarter of a key tile takes a CTA, pairs against single row tiles: the bf16 kernel's numbers.  Pairs gain less from the codes than this says: with 3 : 2 in
// place of 7 : 4 three row tiles over 30001 keys take 65.6 us for 69.0, 12 such trees of up to 3000 keys 55.6 for 59.4, 8 behind 4096 shared keys 85.4 for 91.4 (D = 64:
// 53.6 for 57.3, 44.8 for 48.4), with 1 : 1 69.1, 56.1, 76.2 (53.4, 44.4), with 2 : 1 72.7, 61.9, 98.7 (61.7, 50.5); five row tiles of four trees 38.3 whatever it is.
constexpr int P8_COST_PAIRS = 7, P8_COST_SINGLE = 4;

// What the issuing warps and the converting ones want of a piece (their registers are few).
struct P8Tiles { int t0, t1; };
struct P8Rows {
    int t0, t1;
    int L;              // keys in front of the tree; more than there can be where it is not the piece's (the prefix)
};

// ... and the one that loads: this lane's entry of the page table for the tile.
struct P8Load : PaPiece { int id; };

struct P8Params {
    PaParams a;                            // (its k and v are not used)
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;        // [Hkv]
};

// The power of two that brings a row of bf16 queries whose largest absolute value has these bits (as fp32) to [2^TO, 2^(TO + 1)), and its reciprocal; a row
// that is not finite becomes NaN.
template <int TO> __device__ __forceinline__ float2 row_factor(uint32_t largest) {
    const int e = (int)(largest >> 23);
    if (e == 255) return make_float2(__int_as_float(0x7fffffff), 1.f);
    if (largest == 0u) return make_float2(1.f, 1.f);
    const int k = min(127 + TO - e, 126);
    return make_float2(__int_as_float((127 + k) << 23), __int_as_float((127 - k) << 23));
}
// The factor of a row's scores.  The product of the two scales alone may be beyond fp32 on either side (back, the reciprocal of the row's, spans 2^246); a factor that
// is too small for fp32 is not 0, as a hidden score times it is to stay -inf, nor is one that is too large infinite, as 0 times it is to stay 0.
__device__ __forceinline__ float scores_factor(float scale, float k_scale, float back) {
    const float f = (float)((double)scale * k_scale * back);
    return f == 0.f ? __int_as_float(1) : f == INFINITY && k_scale != INFINITY ? FLT_MAX : f;      // (a k_scale that is not finite shows)
}
__device__ __forceinline__ uint32_t larger_bits(uint32_t m, uint32_t pair) { return max(m, max(pair << 16, pair & 0xffff0000u)); }
__device__ __forceinline__ uint32_t abs2_bf16(uint32_t pair) { return pair & 0x7fff7fffu; }
__device__ __forceinline__ uint32_t to_f16(uint32_t pair, float factor) {
    return pack2_f16(__uint_as_float(pair << 16) * factor, __uint_as_float(pair & 0xffff0000u) * factor);
}

// The run of one worker of a CTA (which = 0: of pairs; 1, 2: of single row tiles) and the item it begins in.  One warp; length, prefix: of the phase's line.
// (The same as begin_walks, one at a time: the kernel is as large as an SM's instruction cache can bear.)
__device__ __forceinline__ void begin_walk(const PaParams &p, PaWalk &w, int which, int cta, int n_cta, int n_pairs, int length, int prefix, int lane) {
    const int single = which > 0, ends = ITEM_COST(single), cost = item_cost(key_tiles(p.shared), ends);
    const int workers = single ? 2 * (n_cta - n_pairs) : n_pairs;
    w.worker = which == 0 ? cta : which == 1 ? cta - n_pairs : cta + n_cta - 2 * n_pairs;
    w.ends = ends;
    // none shorter than a key tile, so that no worker in the middle of an item is left without a tile
    const int run = max((length + workers - 1) / workers, TILE_COST);
    w.x0 = (int)min((int64_t)length, (int64_t)run * w.worker);
    w.x1 = (int)min((int64_t)length, (int64_t)w.x0 + run);
    w.b = -1;
    w.idx = 0;
    w.S = w.x0 == w.x1 ? w.x1 : 0;
    if (w.x0 >= w.x1) return;
    if (w.x0 < prefix) {
        w.idx = w.x0 / cost;
        w.S = w.idx * cost;
    } else {
        const int y = w.x0 - prefix, items = p.phase[single].seq_items;
        int before = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int b = b0 + lane, own = b < p.B ? item_cost(seq_tiles(p, p.seq_lens[b]), ends) * items : 0;
            int c = own;
#pragma unroll 1
            for (int o = 1; o < 32; o *= 2) {
                const int x = __shfl_up_sync(0xffffffffu, c, o);
                if (lane >= o) c += x;
            }
            const uint32_t behind = __ballot_sync(0xffffffffu, before + c > y);
            if (behind) {
                const int at = __ffs((int)behind) - 1, all = __shfl_sync(0xffffffffu, own, at), first = before + __shfl_sync(0xffffffffu, c, at) - all;
                const int each = all / items;
                w.b = b0 + at;
                w.idx = (y - first) / each;
                w.S = prefix + first + w.idx * each;
                break;
            }
            before += __shfl_sync(0xffffffffu, c, 31);
        }
    }
    w.load(p);
}

// All key tiles of a CTA's one or two lists of pieces in the order of for_rounds, the lists taking turns.  P: what a warp wants of a piece.  next(list,
// piece) -> whether there is one; f(list, piece and tile of V or none, piece and tile of K or none) -> whether to go on; ahead(piece, tile): its next tile.
template <typename P, typename N, typename F, typename A>
__device__ __forceinline__ bool in_turns(int lists, N &&next, F &&f, A &&ahead) {
    struct List {
        P cur, old;
        int t, old_t;
        bool live, pend, over;
    } x, y;
    x.live = x.pend = x.over = y.live = y.pend = false;
    y.over = lists < 2;
    int l = 0;
#pragma unroll 1
    while (!x.over || x.pend || !y.over || y.pend) {
        if (!x.over && !x.live) {
            x.live = next(l, x.cur);
            x.over = !x.live;
            x.t = x.cur.t0;
        }
        if (x.live || x.pend) {
            if (!f(l, x.pend, x.old, x.old_t, x.live, x.cur, x.t)) return false;
            x.pend = x.live;
            if (x.live) {
                x.old = x.cur;
                x.old_t = x.t;
                x.live = ++x.t < x.cur.t1;
                if (x.live) ahead(x.cur, x.t);
            }
        }
        if (lists == 2) {
            const List z = x;
            x = y;
            y = z;
            l ^= 1;
        }
    }
    return true;
}

// ptx::mbar_wait in a few instructions (a 32-bit clock, asked between polls, each of which blocks for far less than it takes to wrap).
__device__ __forceinline__ bool short_wait(uint32_t bar, uint32_t parity) {
    static_assert(ptx::WAIT_CYCLE_LIMIT < 1ll << 31, "half a turn of the clock");
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        ".reg .u32 t, u;\n"
        "mov.u32 t, %%clock;\n"
        "AGAIN:\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "@p bra DONE;\n"
        "mov.u32 u, %%clock;\n"
        "sub.u32 u, u, t;\n"
        "setp.lt.u32 q, u, %3;\n"
        "@q bra AGAIN;\n"
        "DONE:\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok) : "r"(bar), "r"(parity), "n"((uint32_t)ptx::WAIT_CYCLE_LIMIT) : "memory");
    return ok != 0;
}

// Four values times the factor, as codes of their first terms and of their second.
__device__ __forceinline__ void to_terms(uint32_t pair0, uint32_t pair1, float factor, uint32_t &first, uint32_t &second) {
    const float x[4] = {__uint_as_float(pair0 << 16) * factor, __uint_as_float(pair0 & 0xffff0000u) * factor,
                        __uint_as_float(pair1 << 16) * factor, __uint_as_float(pair1 & 0xffff0000u) * factor};
    first = e4m3x2(x[0], x[1]) | e4m3x2(x[2], x[3]) << 16;
    const float2 a = f16x2_values(f16x2_lo(first)), b = f16x2_values(f16x2_hi(first));
    second = e4m3x2(x[0] - a.x, x[1] - a.y) | e4m3x2(x[2] - b.x, x[3] - b.y) << 16;
}

// ---------------------------------------------------------------------------------------- pieces
template <int D>
__global__ void __launch_bounds__(P8_THREADS, 1)
paged_attn8_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                   const __grid_constant__ P8Params pp) {
    using SM = P8Smem<D>;
    const PaParams &p = pp.a;
    extern __shared__ __align__(1024) unsigned char gbase[];
    let_next_start();
    // (the shuffle tells the compiler that a warp's number is the same for its lanes: what follows from it needs no divergent branches, and operands of the products
    // no way through vector registers; 16k document 143 -> 135 us, long context 69.1 -> 66.9, single row tiles 52.0 -> 47.7)
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t sbase = ptx::smem_u32(gbase);
    if (sbase & 1023u) {                   // (the swizzles count on it)
        previous_done();
        if (threadIdx.x == 0) atomicExch(p.dev_error, MTV_ERR_TIMEOUT);
        return;
    }
    float *of_rows = reinterpret_cast<float *>(gbase + SM::OFF_ROWS);                              // [2][2][128]: what the two threads of a row exchange
    const uint32_t bars = sbase + SM::OFF_BAR;
    auto bar = [&](int i) { return bars + (uint32_t)i * 8u; };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(gbase + SM::OFF_BAR + P8_OFF_MISC);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + P8_OFF_MISC + 4);
    volatile int *bad = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + P8_OFF_MISC + 8);   // [2][4]: 1 + the last piece with NaN in V
    volatile int *role = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + P8_OFF_MISC + 40);
    int4 *queue = reinterpret_cast<int4 *>(gbase + SM::OFF_BAR + P8_OFF_QUEUE);                    // [2][PA_QUEUE] pieces

    if (warp == P8_TMA_WARP && lane == 0) {
        ptx::prefetch_tensormap(&q_map);
        ptx::prefetch_tensormap(&k_map);
        ptx::prefetch_tensormap(&v_map);
        for (int s = 0; s < SM::K_STAGES; ++s) {
            ptx::mbar_init(bar(P8_KFULL + s), 1);
            ptx::mbar_init(bar(P8_KFREE + s), 2);
            ptx::mbar_init(bar(P8_VFULL + s), 1);
            ptx::mbar_init(bar(P8_VFREE + s), P8_CONV_WARPS);
        }
        for (int s = 0; s < SM::TILES; ++s) {
            ptx::mbar_init(bar(P8_FULL + s), P8_CONV_WARPS);
            ptx::mbar_init(bar(P8_FREE + s), 2);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(bar(P8_QFULL + s), 1);
            ptx::mbar_init(bar(P8_QREADY + s), 8);
            ptx::mbar_init(bar(P8_QFREE + s), 1);
            ptx::mbar_init(bar(P8_SREADY + s), 1);
            ptx::mbar_init(bar(P8_PREADY + s), 8);
            ptx::mbar_init(bar(P8_ODONE + s), 1);
            ptx::mbar_init(bar(P8_TURN + s), 1);
        }
        ptx::mbar_init(bar(P8_FINAL), 2);
        ptx::mbar_init(bar(P8_ROLE), 1);
        for (int q = 0; q < 2; ++q)
            for (int i = 0; i < PA_QUEUE; ++i) {
                ptx::mbar_init(bar(P8_PIECE + q * PA_QUEUE + i), 1);
                ptx::mbar_init(bar(P8_TAKEN + q * PA_QUEUE + i), 2 + P8_CONV_WARPS + 8);
            }
        ptx::fence_mbar_init();
        *abort_flag = 0;
        for (int k = 0; k < 8; ++k) bad[k] = 0;
    }
    if (warp == P8_MMA_WARP) {
        ptx::tmem_alloc(ptx::smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    previous_done();
    const int n_cta = gridDim.x, cta = blockIdx.x;
    const uint32_t tmem = *tmem_slot;
    // a whole warp waits; the same answer for all lanes
    auto wait = [&](int b, uint32_t parity) {
        if (__all_sync(0xffffffffu, short_wait(bar(b), parity))) return true;
        if (lane == 0) {
            *abort_flag = 1;
            atomicExch(p.dev_error, MTV_ERR_TIMEOUT);
        }
        return false;
    };
    // whether the CTA has pairs of row tiles, or single ones
    auto is_pairs = [&]() { return wait(P8_ROLE, 0) && *role; };
    // the n-th piece of a queue (without tiles: there are no more); nothing to be had: false
    auto piece_at = [&](int q, int n) {
        const int at = q * PA_QUEUE + n % PA_QUEUE;
        const int4 a = queue[at * 2], c = queue[at * 2 + 1];
        PaPiece s;
        s.b = a.x; s.g = a.y; s.tile0 = a.z; s.t0 = a.w; s.t1 = c.x; s.L = c.y; s.slot = c.z; s.whole = c.w;
        return s;
    };
    auto look = [&](int q, int n, PaPiece &s) {
        if (__any_sync(0xffffffffu, *abort_flag) || !wait(P8_PIECE + q * PA_QUEUE + n % PA_QUEUE, (n / PA_QUEUE) & 1)) { s.t0 = s.t1 = 0; return false; }
        s = piece_at(q, n);
        return true;
    };
    auto taken = [&](int q, int n) {       // its place may be given to another
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(P8_TAKEN + q * PA_QUEUE + n % PA_QUEUE));
        __syncwarp();
    };
    auto take = [&](int q, int n, PaPiece &s) {
        const bool any = look(q, n, s) && s.t1 > 0;
        taken(q, n);
        return any;
    };

    if (warp == P8_TMA_WARP) {
        // ------------------------------------------------------------ pieces; Q and the codes of K and V
        int tiles = 0, seqs = 0;             // key tiles of an item of every sequence that is not left out, and their number
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int t = b0 + lane < p.B ? seq_tiles(p, p.seq_lens[b0 + lane]) : 0;
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
            const float a = (float)length[0] * P8_COST_PAIRS, b = (float)length[1] * P8_COST_SINGLE;
            n_pairs = length[0] ? max(1, min(n_cta - 1, __float2int_rn(n_cta * (a / (a + b))))) : 0;
        }
        const bool pairs = cta < n_pairs;
        if (lane == 0) {
            *role = pairs;
            ptx::mbar_arrive(bar(P8_ROLE));
        }
        __syncwarp();
        PaWalk walk[2];
#pragma unroll 1
        for (int k = 0; k < (pairs ? 1 : 2); ++k)
            begin_walk(p, walk[k], pairs ? 0 : 1 + k, cta, n_cta, n_pairs, pairs ? length[0] : length[1], pairs ? prefix[0] : prefix[1], lane);
        // One piece more for a queue, or its end: a piece without tiles.  (There is room, or will be without this warp's doing: the queries
        // of a piece are only requested when the scores of the one before are complete, so this warp is never three pieces ahead.)
        auto hand_out = [&](int q, int n, PaPiece &s) {
            const int at = q * PA_QUEUE + n % PA_QUEUE;
            const bool any = walk[q].next(p, p.phase[pairs ? 0 : 1], s);
            if (!any) s = PaPiece{};
            if (n >= PA_QUEUE && !wait(P8_TAKEN + at, (n / PA_QUEUE - 1) & 1)) { s.t0 = s.t1 = 0; return false; }
            if (lane == 0) {
                queue[at * 2] = make_int4(s.b, s.g, s.tile0, s.t0);
                queue[at * 2 + 1] = make_int4(s.t1, s.L, s.slot, s.whole);
                ptx::mbar_arrive(bar(P8_PIECE + at));
            }
            __syncwarp();
            return any;
        };
        int n_q0 = 0, n_q1 = 0;
        const int boxes = PA_KEYS / p.page_rows;
        const uint32_t q_bytes = (uint32_t)(p.npc * p.G) * 128u * SM::HALVES;
        // This lane's entry of the table for a key tile, requested here and looked at where the tile is: nothing waits for it meanwhile.
        // (Where there is no page, or the table names none, zeros are copied.)
        auto find = [&](const PaPiece &s, int t) {
            const int key = t * PA_KEYS + lane * p.page_rows;
            int id = -1;
            if (lane < boxes && key < s.L + (s.b < 0 ? 0 : p.T))
                asm volatile("ld.global.s32 %0, [%1];" : "=r"(id)
                             : "l"(p.pages.table + (int64_t)max(s.b, 0) * p.pages.max_pages + ((key + (s.b < 0 ? 0 : p.shared)) >> p.pages.page_shift)));
            return id;
        };
        auto row_in_page = [&](const PaPiece &s, int t) {
            return (t * PA_KEYS + lane * p.page_rows + (s.b < 0 ? 0 : p.shared)) & ((1 << p.pages.page_shift) - 1);
        };
        struct Ring {
            int entry = 0, stage = 0, turns = 0;
        } rk, rv;
        auto load = [&](Ring &r, int stages, const CUtensorMap *map, uint32_t off, int full, int free, int id, int row, int g) {
            if (r.turns && !wait(free + r.stage, (r.turns - 1) & 1)) return false;
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar(full + r.stage), SM::CODES);
            __syncwarp();
            if (lane < boxes)
                ptx::tma_load_4d(sbase + off + r.stage * SM::CODES + lane * p.page_rows * D, map, bar(full + r.stage), 0, row, g,
                                 id >= 0 && id < p.pages.n_pages ? id : p.pages.n_pages);
            ++r.entry;
            if (++r.stage == stages) { r.stage = 0; ++r.turns; }
            return true;
        };
        int n0 = 0, n1 = 0;
        const int lists = pairs ? 1 : 2;
        const bool ok = in_turns<P8Load>(lists, [&](int l, P8Load &s) {
            int &n = l ? n1 : n0;
            if (!hand_out(l, n++, s)) return false;
            s.id = find(s, s.t0);
            return true;
        }, [&](int l, bool v, const P8Load &vs, int vt, bool k, const P8Load &ks, int kt) {
            if (v && !load(rv, SM::V_STAGES, &v_map, SM::OFF_V, P8_VFULL, P8_VFREE, vs.id, row_in_page(vs, vt), vs.g)) return false;
            if (!k) return true;
            if (!load(rk, SM::K_STAGES, &k_map, SM::OFF_K, P8_KFULL, P8_KFREE, ks.id, row_in_page(ks, kt), ks.g)) return false;
            if (kt == ks.t0)
#pragma unroll 1
                for (int s = l; s < (pairs ? 2 : l + 1); ++s) {
                    int &n = s ? n_q1 : n_q0;
                    if (n && !wait(P8_QFREE + s, (n - 1) & 1)) return false;
                    ++n;
                    if (lane == 0) {
                        ptx::mbar_arrive_expect_tx(bar(P8_QFULL + s), q_bytes);
                        for (int h = 0; h < SM::HALVES; ++h)
                            ptx::tma_load_4d(sbase + s * SM::TILE + h * SM::HALF, &q_map, bar(P8_QFULL + s), h * 64, ks.g * p.G,
                                             max(ks.b, 0) * p.T + (ks.tile0 + (pairs ? s : 0)) * p.npc, 0);
                    }
                    __syncwarp();
                }
            return true;
        }, [&](P8Load &s, int t) { s.id = find(s, t); });
        if (!ok || *abort_flag) {
            // copies in flight get a bounded chance to land before the CTA can exit
            for (int e = max(0, rk.entry - SM::K_STAGES); e < rk.entry; ++e) ptx::mbar_wait(bar(P8_KFULL + e % SM::K_STAGES), (e / SM::K_STAGES) & 1);
            for (int e = max(0, rv.entry - SM::V_STAGES); e < rv.entry; ++e) ptx::mbar_wait(bar(P8_VFULL + e % SM::V_STAGES), (e / SM::V_STAGES) & 1);
            if (n_q0) ptx::mbar_wait(bar(P8_QFULL), (n_q0 - 1) & 1);
            if (n_q1) ptx::mbar_wait(bar(P8_QFULL + 1), (n_q1 - 1) & 1);
        }
    } else if (warp >= P8_CONV_WARP && warp < P8_CONV_WARP + P8_CONV_WARPS) {
        // ------------------------------------------------------------ V's codes -> fp16
        const int tid = (warp - P8_CONV_WARP) * 32 + lane;
        constexpr int PER_ROW = D / 16;                        // 16 codes at a time
        constexpr int TIMES = 128 * PER_ROW / (P8_CONV_WARPS * 32);
        // chunk (row, c) of 16 codes: two chunks of 8 fp16.  Lanes of the second half of a row store them the other way round, so that the eight lanes
        // of a row reach eight different groups of banks.
        const int c = tid % PER_ROW, row0 = tid / PER_ROW, half = c / 4, first_c = 2 * (c % 4) + (D == 128 ? half : 0);
        constexpr int ROWS = P8_CONV_WARPS * 32 / PER_ROW;     // from one of a thread's chunks to its next; a multiple of 8
        static_assert(ROWS % 8 == 0, "the swizzle of a thread's chunks is the same");
        const uint32_t to_a = half * SM::HALF + row0 * 128 + ((first_c ^ (row0 & 7)) << 4), to_b = half * SM::HALF + row0 * 128 + ((first_c ^ 1 ^ (row0 & 7)) << 4);
        const bool swapped = first_c & 1;
        const unsigned char *codes = gbase + SM::OFF_V + tid * 16;
        unsigned char *tiles = gbase + SM::OFF_TILES;
        int n0 = 0, n1 = 0, n_piece0 = 0, n_piece1 = 0, stage = 0, turns = 0, from = 0, from_turns = 0;
        const bool pairs = is_pairs();
        in_turns<P8Rows>(pairs ? 1 : 2, [&](int l, P8Rows &s) {
                PaPiece pc;
                int &n = l ? n1 : n0;
                const bool any = take(l, n++, pc);
                s = {pc.t0, pc.t1, pc.b < 0 ? INT_MAX : pc.L};
                return any;
            }, [&](int l, bool v, const P8Rows &vs, int vt, bool, const P8Rows &, int) {
                if (!v) return true;
                if (!wait(P8_VFULL + from, from_turns & 1)) return false;
                if (turns && !wait(P8_FREE + stage, (turns - 1) & 1)) return false;
                const uint4 *src = reinterpret_cast<const uint4 *>(codes + from * SM::CODES);
                unsigned char *dst = tiles + stage * SM::TILE;
                // rows of the tree are looked through, those behind them become zeros
                const bool last = (vt + 1) * PA_KEYS > vs.L;
                bool odd = false;
#pragma unroll 1
                for (int i0 = 0; i0 < TIMES; i0 += 4) {
                    uint4 u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] = src[(i0 + i) * (P8_CONV_WARPS * 32)];
                    if (last) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int a = vt * PA_KEYS + row0 + (i0 + i) * ROWS - vs.L;        // the row's node
                            const uint32_t nans = nan_codes(u[i].x) | nan_codes(u[i].y) | nan_codes(u[i].z) | nan_codes(u[i].w);
                            if (a >= p.T) u[i] = make_uint4(0u, 0u, 0u, 0u);
                            else if (a >= 0 && nans) {
                                u[i] = make_uint4(without_nans(u[i].x), without_nans(u[i].y), without_nans(u[i].z), without_nans(u[i].w));
                                odd = true;
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint4 lo = make_uint4(f16x2_lo(u[i].x), f16x2_hi(u[i].x), f16x2_lo(u[i].y), f16x2_hi(u[i].y));
                        const uint4 hi = make_uint4(f16x2_lo(u[i].z), f16x2_hi(u[i].z), f16x2_lo(u[i].w), f16x2_hi(u[i].w));
                        *reinterpret_cast<uint4 *>(dst + to_a + (i0 + i) * ROWS * 128) = swapped ? hi : lo;
                        *reinterpret_cast<uint4 *>(dst + to_b + (i0 + i) * ROWS * 128) = swapped ? lo : hi;
                    }
                }
                if (last && __any_sync(0xffffffffu, odd) && lane == 0) {
                    if (pairs || l == 0) bad[n_piece0 & 3] = n_piece0 + 1;
                    if (pairs || l == 1) bad[4 + (n_piece1 & 3)] = n_piece1 + 1;
                }
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(bar(P8_FULL + stage));
                    ptx::mbar_arrive(bar(P8_VFREE + from));
                }
                __syncwarp();
                if (++stage == SM::TILES) { stage = 0; ++turns; }
                if (++from == SM::V_STAGES) { from = 0; ++from_turns; }
                if (vt == vs.t1 - 1) {
                    n_piece0 += pairs || l == 0;
                    n_piece1 += pairs || l == 1;
                }
                return true;
            }, [](P8Rows &, int) {});
    } else if (warp == P8_MMA_WARP || warp == P8_MMA_WARP + 1) {
        // ------------------------------------------------------------ products of row tile s
        const int s = warp - P8_MMA_WARP;
        const bool leader = ptx::elect_one();
        const uint32_t dq = ptx::desc_lo(sbase + s * SM::TILE, 16), dk0 = ptx::desc_lo(sbase + SM::OFF_K, 16), dv0 = ptx::desc_lo(sbase + SM::OFF_TILES, SM::HALF);
        const uint32_t t_s = tmem + s * 128, t_o = tmem + 256 + s * D;
        int n_p = 0, n_q = 0, n_turn = 0;
        int v_stage = 0, v_turns = 0, k_stage = 0, k_turns = 0;
        int n0 = 0, n1 = 0;
        const bool pairs = is_pairs();
        in_turns<P8Tiles>(pairs ? 1 : 2, [&](int l, P8Tiles &x) {
                PaPiece pc;
                int &n = l ? n1 : n0;
                const bool any = take(l, n++, pc);
                x = {pc.t0, pc.t1};
                return any;
            }, [&](int l, bool v, const P8Tiles &vs, int vt, bool k, const P8Tiles &ks, int kt) {
                const int v_at = v_stage, k_at = k_stage, v_parity = v_turns & 1, k_parity = k_turns & 1;
                if (v && ++v_stage == SM::TILES) { v_stage = 0; ++v_turns; }
                if (k && ++k_stage == SM::K_STAGES) { k_stage = 0; ++k_turns; }
                if (!pairs && l != s) {
                    // the other tile's: waited for and handed back all the same, so that this warp is never a turn of a ring ahead or
                    // late (a parity wait cannot tell a phase from the one two before or behind)
                    auto pass = [&](int full, int free, int parity) {
                        if (!wait(full, parity)) return false;
                        if (lane == 0) ptx::mbar_arrive(bar(free));
                        __syncwarp();
                        return true;
                    };
                    return (!v || pass(P8_FULL + v_at, P8_FREE + v_at, v_parity)) && (!k || pass(P8_KFULL + k_at, P8_KFREE + k_at, k_parity));
                }
                auto k_there = [&]() { return wait(P8_KFULL + k_at, k_parity) && (kt != ks.t0 || wait(P8_QREADY + s, n_q++ & 1)); };
                // Pairs take turns: the products of a row tile go to the tensor core in one run.  Mixed with the other tile's, both tiles' scores
                // would come when all are done, both softmaxes would then run at once, and the tensor core wait for both.  (Passed on when the run's products are
                // complete: 1 % fewer cycles than when they are issued.)
                auto begin_run = [&]() {
                    if (!pairs) return true;
                    const int turn = n_turn++;
                    return s == 0 && turn == 0 ? true : wait(P8_TURN + s, (turn + s - 1) & 1);
                };
                auto end_run = [&]() {
                    if (pairs) ptx::tc_commit_elect(bar(P8_TURN + (s ^ 1)), leader);
                };
                // the weights are waited for last: what else there is to wait for is there by then (a new piece's queries may not be), the turn too: a wait
                // for what is there took this warp 400 cycles among the others (16k document 150 us with the turn waited for last, 143 so; long context 73.2, 69.4)
                const bool ahead = v && k && kt != ks.t0;
                if (ahead && !k_there()) return false;
                if (v) {
                    if (!wait(P8_FULL + v_at, v_parity) || !begin_run() || !wait(P8_PREADY + s, n_p++ & 1)) return false;
                    ptx::tc_fence_after();
                    const uint32_t dv = dv0 + (uint32_t)v_at * (SM::TILE >> 4);
#pragma unroll
                    for (int kk = 0; kk < PA_KEYS / 16; ++kk)
                        ptx::mma_ts_elect(t_o, t_s + kk / 4 * 64 + kk % 4 * 8, dv + kk * 128, ptx::DESC_HI, SM::IDESC_PV, vt > vs.t0 || kk > 0, leader);
                    if (vt == vs.t1 - 1) ptx::tc_commit_elect(bar(P8_ODONE + s), leader);
                    if (!ahead) end_run();
                }
                if (k) {
                    if (!ahead) {
                        if (!k_there() || !begin_run()) return false;
                        ptx::tc_fence_after();
                    }
                    const uint32_t dk = dk0 + (uint32_t)k_at * (SM::CODES >> 4);
#pragma unroll
                    for (int term = 0; term < 2; ++term)
#pragma unroll
                        for (int kk = 0; kk < D / 32; ++kk)
                            ptx::mma_ss_f8_elect(t_s, dq + (kk / 2 * SM::HALF + kk % 2 * 64 + term * 32) / 16, ptx::DESC_HI, dk + kk * 2, SM::K_DESC_HI, SM::IDESC_QK, term + kk > 0, leader);
                    ptx::tc_commit_elect(bar(P8_SREADY + s), leader);
                    if (kt == ks.t1 - 1) ptx::tc_commit_elect(bar(P8_QFREE + s), leader);
                    end_run();
                }
                if (v) ptx::tc_commit_elect(bar(P8_FREE + v_at), leader);
                if (k) ptx::tc_commit_elect(bar(P8_KFREE + k_at), leader);
                return true;
            }, [](P8Tiles &, int) {});
        // what was issued is complete, and has signalled, before the CTA can exit
        ptx::tc_commit_elect(bar(P8_FINAL), leader);
        ptx::mbar_wait(bar(P8_FINAL), 0);
    } else if (warp < P8_CONV_WARP) {
        // ------------------------------------------------------------ softmax: thread (row, hf) of row tile s: columns [64 hf, 64 hf + 64)
        const int s = warp >> 3, hf = (warp >> 2) & 1, qd = warp & 3, row = qd * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(qd * 32) << 16);
        const uint32_t t_s = lane_base + s * 128 + hf * 64;      // this half's scores, and P over them
        const uint32_t t_o = lane_base + 256 + s * D + hf * (D / 2);
        const int pair_bar = 2 + s * 4 + qd;
        const int node_in_tile = row / p.G, head = row - node_in_tile * p.G;
        const bool there = wait(P8_ROLE, 0), pairs = there && *role;
        const PaPhase &ph = p.phase[pairs ? 0 : 1];
        const int q = pairs ? 0 : s;
        // what the other thread of the row has (two barriers: what was exchanged before has been read)
        auto pair_sync = [&]() { asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair_bar) : "memory"); };
        auto exchange = [&](float v) {
            pair_sync();
            of_rows[(s * 2 + hf) * 128 + row] = v;
            pair_sync();
            return of_rows[(s * 2 + (hf ^ 1)) * 128 + row];
        };
        auto node_of = [&](const PaPiece &pc) { return (pc.tile0 + (pairs ? s : 0)) * p.npc + node_in_tile; };
        // (what is needed of a piece at its start and end alone stays in the queue until then)
        int n_s = 0;                       // key tiles so far
        float m = 0.f, l = 0.f, vs = 0.f;  // the piece's: reference, sum, scale of V
        bool mine = false;
        int node = -1;                     // the row's, if it sees some of the tree's rows; -1: none, or no row
        PaPiece pc = {};
        int left_at = 0;                   // the key tile in which a wait ran out; -1: in front of the exchange of the queries' maxima
        auto is_mine = [&]() { return node_in_tile < p.npc && node_of(pc) < (pc.b < 0 ? p.B * p.T : p.T); };
        if (!there) all_of_rows(pair_bar, false);
        else pieces_in_step([&](int n) { return look(q, n, pc); }, [&](bool x) { return all_of_rows(pair_bar, x); }, [&](int n) {
            const bool more = pc.t1 > 0;
            float sc = 0.f, vs_next = 0.f;
            if (more) {
                // ---- the piece's queries in two terms, where they are: each thread of a row takes half of its columns.  Their first product then runs beside
                // the end of the piece before.
                const float ks = pp.k_scale[pc.g];
                vs_next = pp.v_scale[pc.g];
                if (!wait(P8_QFULL + s, n & 1)) { left_at = -1; return Way::LEFT; }
                constexpr int CHUNKS = D / 16;
                unsigned char *at = gbase + s * SM::TILE + (D == 128 ? hf * SM::HALF : 0) + row * 128;
                auto chunk = [&](int c) { return reinterpret_cast<uint4 *>(at + (((D == 128 ? 0 : hf * CHUNKS) + c ^ (row & 7)) << 4)); };
                uint32_t most = 0u;
#pragma unroll 4
                for (int c = 0; c < CHUNKS; ++c) {
                    const uint4 u = *chunk(c);
                    most = larger_bits(larger_bits(larger_bits(larger_bits(most, abs2_bf16(u.x)), abs2_bf16(u.y)), abs2_bf16(u.z)), abs2_bf16(u.w));
                }
                most = max(most, __float_as_uint(exchange(__uint_as_float(most))));
                const float2 factor = row_factor<7>(most);
                // 32 columns at a time, where they are: the first terms' 32 bytes, then the second terms'
#pragma unroll 1
                for (int c = 0; c < CHUNKS; c += 4) {
                    uint32_t first[8], second[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint4 u = *chunk(c + e);
                        to_terms(u.x, u.y, factor.x, first[2 * e], second[2 * e]);
                        to_terms(u.z, u.w, factor.x, first[2 * e + 1], second[2 * e + 1]);
                    }
                    *chunk(c) = make_uint4(first[0], first[1], first[2], first[3]);
                    *chunk(c + 1) = make_uint4(first[4], first[5], first[6], first[7]);
                    *chunk(c + 2) = make_uint4(second[0], second[1], second[2], second[3]);
                    *chunk(c + 3) = make_uint4(second[4], second[5], second[6], second[7]);
                }
                sc = scores_factor(p.scale_log2, ks, factor.y);
                ptx::fence_proxy_async();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar(P8_QREADY + s));
            }
            if (n) {
                // ---- the piece before
                if (!wait(P8_ODONE + s, (n - 1) & 1)) { left_at = pc.t0; return more ? Way::LEFT : Way::END; }
                ptx::tc_fence_after();
                const PaPiece old = piece_at(q, n - 1);
                if (__any_sync(0xffffffffu, mine)) {
                    const bool odd = bad[s * 4 + ((n - 1) & 3)] == n;
                    const bool direct = p.shared == 0 && old.whole;
                    const float factor = direct ? vs / l : vs;
                    const int slot_row = pairs ? s * 128 + row : row;
                    float *o_out = ph.o + ((size_t)old.slot * ph.rows * (D / 8) + (size_t)(hf * (D / 16)) * ph.rows + slot_row) * 8;
                    __nv_bfloat16 *out = p.out + (((size_t)max(old.b, 0) * p.T + node_of(old)) * p.Hq + old.g * p.G + head) * D + hf * (D / 2);
#pragma unroll 1
                    for (int h = 0; h < D / 32; ++h) {
                        uint32_t o[16];
                        ptx::tmem_ld16(t_o + h * 16, o);
                        ptx::tmem_ld_wait_for16(o);
                        if (!mine) continue;
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                        if (odd) {
                            // V codes that the tensor core did not see: NaN with any weight is NaN
#pragma unroll 1
                            for (int a = max(0, old.t0 * PA_KEYS - old.L); a < p.T && old.L + a < old.t1 * PA_KEYS; ++a) {
                                if (node < 0 || !(p.anc[node * 2 + (a >> 6)] >> (a & 63) & 1)) continue;
                                const int64_t at = p.pages.row(old.b, p.shared + old.L + a);
                                if (at < 0) continue;
                                const uint8_t *v = pp.v + at + old.g * p.pages.stride_h + hf * (D / 2) + h * 16;
#pragma unroll
                                for (int e = 0; e < 16; ++e)
                                    if ((v[e] & 0x7fu) == 0x7fu) o[e] = 0x7fffffffu;
                            }
                        }
                        if (direct) {
                            uint32_t w[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) w[e] = pack2_bf16(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
                            *reinterpret_cast<uint4 *>(out + h * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                            *reinterpret_cast<uint4 *>(out + h * 16 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                        } else {
                            ptx::st_global_32(o_out + (size_t)(2 * h) * ph.rows * 8, *reinterpret_cast<const uint32_t(*)[8]>(&o[0]));
                            ptx::st_global_32(o_out + (size_t)(2 * h + 1) * ph.rows * 8, *reinterpret_cast<const uint32_t(*)[8]>(&o[8]));
                        }
                    }
                    if (mine && !direct && hf == 0)                // (what weighs 1)
                        ph.ml[(size_t)old.slot * ph.rows + slot_row] = make_float2(l == 0.f ? -INFINITY : m - P8_SHIFT, l);
                }
                if (!pairs || s) taken(q, n - 1);                  // (in a pair the second row tile's warps: its place is not used again before the next but two's scores, both tiles')
            }
            if (!more) return Way::END;
            mine = is_mine();
            node = mine && pc.b >= 0 ? node_of(pc) : -1;
            m = -INFINITY;
            l = 0.f;
            vs = vs_next;
            const bool some = __any_sync(0xffffffffu, mine);
            const float2 sc2 = make_float2(sc, sc);
#pragma unroll 1
            for (int t = pc.t0; t < pc.t1; ++t) {
                if (!wait(P8_SREADY + s, n_s++ & 1)) { left_at = t; return Way::LEFT; }
                ptx::tc_fence_after();
                if (some) {
                    uint32_t a[16], b[16], pk[32];                 // (pk: fp16 pairs)
                    ptx::tmem_ld16(t_s, a);                        // on their way meanwhile
                    if ((t + 1) * PA_KEYS > pc.L) {
                        // Hidden scores become -inf where they are.  Visibility of the tree's rows as 32-bit words; the rows in front of them are visible to every
                        // node, those behind to none.
                        auto anc_word = [&](int w) -> uint32_t { return w < 0 ? 0xffffffffu : w < 4 && node >= 0 ? reinterpret_cast<const uint32_t *>(p.anc)[node * 4 + w] : 0u; };
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            const int a0 = t * PA_KEYS + hf * 64 + c * 16 - pc.L;      // tree row of the first column
                            const uint32_t vis = __funnelshift_r(anc_word(a0 >> 5), anc_word((a0 >> 5) + 1), a0 & 31);
                            uint32_t x[16];
                            ptx::tmem_ld16(t_s + c * 16, x);
                            ptx::tmem_ld_wait_for16(x);
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (!((vis >> e) & 1u)) x[e] = 0xff800000u;
                            ptx::tmem_st16(t_s + c * 16, x);
                        }
                        ptx::tmem_st_wait();
                        ptx::tmem_ld16(t_s, a);
                    }
                    bool move = t == pc.t0;
                    float sum;
                    for (;;) {
                        if (move) {
                            float mxs = -INFINITY;
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {
                                uint32_t x[16];
                                ptx::tmem_ld16(t_s + c * 16, x);
                                ptx::tmem_ld_wait_for16(x);
#pragma unroll
                                for (int e = 0; e < 16; e += 2) mxs = max3_nan(mxs, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                            }
                            mxs *= sc;
                            mxs = max_nan(mxs, exchange(mxs));
                            if (mxs == INFINITY) mxs = __int_as_float(0x7fffffff);     // inf - inf: the row is NaN, as from the formula
                            const float m_new = mxs <= m ? m : mxs;                      // (a NaN is taken over)
                            const bool need = m_new != m && m != -INFINITY && mine;
                            if (__any_sync(0xffffffffu, need)) {
                                const float alpha = need ? ex2(m - m_new) : 1.f;
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
                            m = m_new;
                        }
                        const float shift = m == -INFINITY ? P8_SHIFT : P8_SHIFT - m;
                        const float2 nm2 = make_float2(shift, shift);
                        float2 la = make_float2(0.f, 0.f), lb = la;
                        float px = -INFINITY;
                        // sixteen columns at a time, the next ones on their way meanwhile
                        auto weights = [&](int c, uint32_t (&x)[16]) {
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                const float2 x01 = __ffma2_rn(make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), sc2, nm2);
                                const float2 x23 = __ffma2_rn(make_float2(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])), sc2, nm2);
                                float2 p01, p23;
                                if (e == 12) {      // every fourth quadruple on the FMA pipes: the special-function unit takes as long as the products
                                    px = max3_nan(max3_nan(px, x01.x, x01.y), x23.x, x23.y);   // (neither NaN nor what is above 127 survives there)
                                    p01 = exp2_poly2(x01);
                                    p23 = exp2_poly2(x23);
                                } else {
                                    p01 = make_float2(ex2(x01.x), ex2(x01.y));
                                    p23 = make_float2(ex2(x23.x), ex2(x23.y));
                                }
                                la = __fadd2_rn(la, p01);
                                lb = __fadd2_rn(lb, p23);
                                pk[c * 8 + e / 2] = pack2_f16(p01.x, p01.y);
                                pk[c * 8 + e / 2 + 1] = pack2_f16(p23.x, p23.y);
                            }
                        };
                        ptx::tmem_ld_wait_for16(a);
                        ptx::tmem_ld16(t_s + 16, b);
                        weights(0, a);
                        ptx::tmem_ld_wait_for16(b);
                        ptx::tmem_ld16(t_s + 32, a);
                        weights(1, b);
                        ptx::tmem_ld_wait_for16(a);
                        ptx::tmem_ld16(t_s + 48, b);
                        weights(2, a);
                        ptx::tmem_ld_wait_for16(b);
                        weights(3, b);
                        sum = (la.x + la.y) + (lb.x + lb.y);
                        if (move) break;
                        // a sum that is too large, infinite or NaN: a weight then may be beyond fp16; and a row that has met no visible key so far
                        if (!any_of_rows(pair_bar, mine && (!(sum < 65504.f) || !(px <= P8_LIMIT) || m == -INFINITY))) break;
                        move = true;
                        ptx::tmem_ld16(t_s, a);
                    }
                    l += sum;
                    ptx::tmem_st32(t_s, pk);
                    if (t == pc.t1 - 1) l += exchange(l);          // the row's sum
                    ptx::tmem_st_wait();
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar(P8_PREADY + s));
            }
            return Way::ON;
        }, [&]() {
            if (left_at < 0) {
                exchange(0.f);
                left_at = pc.t0;
            }
            if (__any_sync(0xffffffffu, is_mine()))
                follow_tiles(left_at, pc.t0, pc.t1, [&]() { return any_of_rows(pair_bar, false); }, [&](bool) { exchange(0.f); }, [&]() { exchange(0.f); });
        });
    }
    // ---- nobody leaves while the tensor core may still work for the CTA
    __syncwarp();
    ptx::tc_fence_before();
    asm volatile("bar.sync 1, %0;" ::"n"(P8_THREADS) : "memory");
    ptx::tc_fence_after();
    if (warp == P8_MMA_WARP) ptx::tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------------------------------- thin items
// At most 16 query rows against a KV head's keys (plain decoding; the smallest trees): nothing but the bytes counts.  As for the bf16 cache, warps of
// their own with mma.sync, but with the operands the other way round: S^T = K Q^T and O^T = V^T P^T.  Keys and columns of V then fill the products' 16
// rows, and up to 8 query rows their 8 columns (up to 16 take two products, NR = 2), where query rows as the 16 left three quarters of the products and of O's
// registers to nothing for groups of four.
// A contraction's order is free as long as both operands have it, and so is the order of O's columns: 16 bytes of two K rows are four products' A operands of
// a thread, converted as they stand; 16 bytes of four V rows (8 at D = 64) are two columns in each of 8 products (4), two keys' codes side by side by a byte
// permutation in front of the conversion.  P^T is P transposed, 8 x 8 at a time, by movmatrix.
// A CTA walks a run of the line of all thin items, KEYS keys to a warp at a time.  Asynchronous copies bring them to the warp's own part of shared memory,
// STAGES - 1 blocks ahead: no warp waits for another, and no register holds what is on its way.  At a piece's end the warps join.
// An instruction of copies covers whole rows: where it took half a row of each of 8 keys (as the operands have them), the other half crossed from L2 with it, twice
// in all (that step took 64 single tokens from 88 us to 71).
// Measured: 64 single tokens, 8 KV heads of 128, 500 to 4000 keys each: 277 MB in 52 us = 5.3 TB/s, 81 % of the copy rate (58 us with the joining, 53 in replayed
// graphs); one token of 60001 keys 30 us (18.8 at the memory's rate).  8 warps and 16 keys, 6 and 32, 4 and 32 are within a percent: what is left is the pieces'
// starts and ends.
// Two products for up to 8 rows too (NR = 2 for all): 32 sequences, 8 rows a KV head 36 us for 33.5 (D = 64: 28.9 for 21.4), 64 of 4 or of 1 row 56.5 for 53.  9 and 16 rows, which
// need them, 37.5 and 36.7 (floor 22.8; D = 64, 16 rows: 29.8, floor 11.4).
// Weights are 2^SHIFT at the reference, as in row tiles (so that as small ones count); it may be SLACK too small: they stay below 2^16, which fp16 ends at.
constexpr float T8_SHIFT = 8.f, T8_SLACK = 7.9f;

// NR: products of 8 query rows.
template <int D, int NR> struct T8 {
    static constexpr int WARPS = NR == 1 ? 8 : 4, KEYS = NR == 1 ? 16 : 32, STAGES = 3;
    static constexpr int STEP = WARPS * KEYS;
    static constexpr int ENDS = 2;                 // what an item's start and end take, in steps
    static constexpr uint32_t K_BYTES = KEYS * D, STAGE = 2 * K_BYTES, RING = WARPS * STAGES * STAGE;     // a warp's stages side by side
    static constexpr uint32_t JOIN = WARPS * 8 * NR * (D + 4) * 4;
    static constexpr uint32_t TOTAL = RING > JOIN ? RING : JOIN;                                          // (the warps join where the ring was)
    static_assert(2 * (TOTAL + 2048 + 1024) <= 227 * 1024, "two CTAs on an SM");
};

__device__ __forceinline__ void mma16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// 16 bytes from global to shared memory, or zeros
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool is) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(is ? 16 : 0) : "memory");
}
// Where 16-byte chunk c of a row lies in it, so that the eight lanes that read two neighbouring rows of K, or four rows of V of one parity, together meet
// different banks.
template <int D> __device__ __forceinline__ int chunk_at(int row, int c) {
    return D == 128 ? c ^ (row >> 1 & 3) << 1 ^ (row & 1) << 2 : c ^ (row >> 1 & 3);
}

template <int D, int NR>
__global__ void __launch_bounds__(T8<D, NR>::WARPS * 32, 2)
paged_attn8_thin_kernel(const __grid_constant__ P8Params pp) {
    using SM = T8<D, NR>;
    using Line = ThinLine<SM::STEP, SM::ENDS>;
    constexpr int WARPS = SM::WARPS, STAGES = SM::STAGES;
    constexpr int C = D / 64;              // 64-column parts of a row: 16 bytes of each are a thread's
    constexpr int J = D / 8, JW = J / 4;   // columns of V that are a thread's, and their words
    constexpr int MT = SM::KEYS / 16;      // products of 16 keys
    const PaParams &p = pp.a;
    extern __shared__ __align__(16) unsigned char ring[];
    float (*o_x)[8 * NR][D + 4] = reinterpret_cast<float (*)[8 * NR][D + 4]>(ring);      // [WARPS]
    __shared__ float2 ml_x[WARPS][8 * NR];
    __shared__ int start[5];               // x0, x1, S, b, idx
    let_next_start();
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32, r0 = lane / 4, quad = lane % 4;
    const PaPhase &ph = p.phase[2];
    const int worker = blockIdx.x, workers = gridDim.x;
    // this warp's stages: rows of K, then of V
    const unsigned char *mine = ring + warp * STAGES * SM::STAGE;
    const uint32_t mine_at = ptx::smem_u32(mine);
    constexpr int PER_ROW = D / 16, ROWS = 32 / PER_ROW;         // lanes of a row, rows of an instruction of copies
    const int my_row = lane / PER_ROW, my_chunk = lane % PER_ROW;
    previous_done();
    if (warp == 0) Line::begin(p, worker, workers, lane, start);
    __syncthreads();
    const int x0 = start[0], x1 = start[1];
    int S = start[2], b = start[3], idx = start[4];
    int L = 0, cost = 0;                   // keys of the item (prefix: the shared ones; else its own in front of the tree)
    auto load_item = [&]() {
        if (b < 0) {
            L = p.shared;
            cost = Line::steps(p.shared) + SM::ENDS;
        } else {
            cost = Line::cost_of(p, b);
            L = p.seq_lens[b] - p.shared;
        }
    };
    if (x0 < x1) load_item();
#pragma unroll 1
    while (S < x1) {
        if (idx >= (b < 0 ? ph.prefix_items : ph.seq_items) || cost == 0) {
            if (++b >= p.B) break;
            idx = 0;
            load_item();
            continue;
        }
        const int steps = cost - SM::ENDS;
        const int t0 = max(0, min(x0 - S - SM::ENDS, steps)), t1 = max(0, min(x1 - S - SM::ENDS, steps));
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
        // ---- this warp's blocks of keys, sixteen by sixteen: they may lie on two pages
        const int32_t *table = p.pages.table + (int64_t)max(b, 0) * p.pages.max_pages;
        auto key_of = [&](int t, int mt) { return (t * WARPS + warp) * SM::KEYS + mt * 16; };
        auto page_of = [&](int t, int mt) { return t < t1 && key_of(t, mt) < n_keys ? table[(key_of(t, mt) + key0) >> p.pages.page_shift] : -1; };
        auto row_at = [&](int t, int mt, int id) {       // byte offset of the first row; < 0: there is none
            return id < 0 || id >= p.pages.n_pages ? -1ll
                   : (long long)id * p.pages.stride_page + (long long)((key_of(t, mt) + key0) & ((1 << p.pages.page_shift) - 1)) * p.pages.stride_t +
                         g * p.pages.stride_h;
        };
        // The blocks up to the one STAGES - 1 ahead are requested; the pages of the one behind them are looked up.
        int id_next[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) id_next[mt] = page_of(t0, mt);
        auto request = [&](int t) {
            const uint32_t to = mine_at + (uint32_t)((t - t0) % STAGES) * SM::STAGE;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const long long at = row_at(t, mt, id_next[mt]);
                id_next[mt] = page_of(t + 1, mt);
                if (t >= t1) continue;
                const long long from = (at >= 0 ? at : 0) + my_row * p.pages.stride_t + my_chunk * 16;
                const int left = at >= 0 ? n_keys - key_of(t, mt) - my_row : 0;      // rows behind the last key may hold anything
#pragma unroll
                for (int i = 0; i < 16; i += ROWS) {
                    const uint32_t to_row = to + (mt * 16 + i + my_row) * D + chunk_at<D>(i + my_row, my_chunk) * 16;
                    copy_async(to_row, pp.k + from + i * p.pages.stride_t, i < left);
                    copy_async(to_row + SM::K_BYTES, pp.v + from + i * p.pages.stride_t, i < left);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll 1
        for (int t = t0; t < t0 + STAGES - 1; ++t) request(t);       // (the barrier at a piece's end is between these and the last reads)
        // ---- the query rows as B operands: product (c, i) has columns c * 64 + quad * 16 + 4 i + [0, 2) and [2, 4) of row r0 + 8 nr
        uint32_t qb[NR][C][4][2];
        uint32_t see[NR][2];               // tree rows that are visible to rows 8 nr + 2 quad and the next (at most 16 nodes)
        float sc[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int r = r0 + 8 * nr, n = r / p.G;
            const bool is = r < rows;
            const __nv_bfloat16 *src = p.q + (((size_t)(own ? b * p.T : 0) + n) * p.Hq + g * p.G + (r - n * p.G)) * D + quad * 16;
            uint32_t most = 0u;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 u = is ? *reinterpret_cast<const uint4 *>(src + c * 64) : make_uint4(0u, 0u, 0u, 0u);
                const uint4 v = is ? *reinterpret_cast<const uint4 *>(src + c * 64 + 8) : make_uint4(0u, 0u, 0u, 0u);
                qb[nr][c][0][0] = u.x; qb[nr][c][0][1] = u.y; qb[nr][c][1][0] = u.z; qb[nr][c][1][1] = u.w;
                qb[nr][c][2][0] = v.x; qb[nr][c][2][1] = v.y; qb[nr][c][3][0] = v.z; qb[nr][c][3][1] = v.w;
#pragma unroll
                for (int i = 0; i < 4; ++i) most = larger_bits(larger_bits(most, abs2_bf16(qb[nr][c][i][0])), abs2_bf16(qb[nr][c][i][1]));
            }
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const float2 factor = row_factor<8>(most);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    qb[nr][c][i][0] = to_f16(qb[nr][c][i][0], factor.x);
                    qb[nr][c][i][1] = to_f16(qb[nr][c][i][1], factor.x);
                }
            const float of_row = scores_factor(p.scale_log2, pp.k_scale[g], factor.y);
            const uint32_t seen = is && own ? (uint32_t)p.anc[n * 2] : 0u;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                sc[nr][e] = __shfl_sync(0xffffffffu, of_row, (2 * quad + e) * 4);
                see[nr][e] = __shfl_sync(0xffffffffu, seen, (2 * quad + e) * 4);
            }
        }
        float o[NR][D / 16][4] = {}, m[NR][2], l[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            m[nr][0] = m[nr][1] = -INFINITY;
            l[nr][0] = l[nr][1] = 0.f;
        }
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            const int first = key_of(t, 0);
            if (first >= n_keys) break;    // (the item's last step: no keys for this warp)
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();                  // all lanes' copies of this block are there, and all are done with the block before
            request(t + STAGES - 1);
            const unsigned char *block = mine + (uint32_t)((t - t0) % STAGES) * SM::STAGE;
            // ---- scores: x[mt][nr]: key mt * 16 + r0 (+ 8: elements 2 and 3), rows 8 nr + 2 quad and the next
            float x[MT][NR][4] = {};
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const unsigned char *src = block + (mt * 16 + r0) * D + chunk_at<D>(r0, c * 4 + quad) * 16;      // (of row r0 + 8 too)
                    const uint4 k0 = *reinterpret_cast<const uint4 *>(src), k8 = *reinterpret_cast<const uint4 *>(src + 8 * D);
                    const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w8[4] = {k8.x, k8.y, k8.z, k8.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr)
                            mma16816_f16(x[mt][nr], f16x2_lo(w0[i]), f16x2_lo(w8[i]), f16x2_hi(w0[i]), f16x2_hi(w8[i]), qb[nr][c][i][0], qb[nr][c][i][1]);
                }
            const bool edge = first + SM::KEYS > L;
            if (edge) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int a = first + mt * 16 + r0 + 8 * (e >> 1) - L;
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr)
                            if (a >= 0 && (!own || a >= p.T || !(see[nr][e & 1] >> a & 1u))) x[mt][nr][e] = -INFINITY;
                    }
            }
            // The reference moves where a score of the row is too far above it, and where there is none yet.  (Asked of the exponent that the weight is taken of: far from
            // zero, m + SLACK would be rounded up to a step of fp32, and a weight beyond fp16 could pass.)
            bool ask = false;
#pragma unroll
            for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = max_nan(x[0][nr][e], x[0][nr][e + 2]);
#pragma unroll
                    for (int mt = 1; mt < MT; ++mt) mx = max3_nan(mx, x[mt][nr][e], x[mt][nr][e + 2]);
                    ask = ask || !(fmaf(mx, sc[nr][e], T8_SHIFT - m[nr][e]) <= T8_SHIFT + T8_SLACK);
                }
            if (__any_sync(0xffffffffu, ask)) {
#pragma unroll
                for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = max_nan(x[0][nr][e], x[0][nr][e + 2]);
#pragma unroll
                        for (int mt = 1; mt < MT; ++mt) mx = max3_nan(mx, x[mt][nr][e], x[mt][nr][e + 2]);
#pragma unroll
                        for (int k = 4; k < 32; k *= 2) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, k));
                        mx *= sc[nr][e];
                        if (mx == INFINITY) mx = __int_as_float(0x7fffffff);     // inf - inf: the row is NaN, as from the formula
                        const float m_new = mx <= m[nr][e] ? m[nr][e] : mx;
                        const float w = m[nr][e] == -INFINITY ? 0.f : ex2(m[nr][e] - m_new);
                        m[nr][e] = m_new;
                        l[nr][e] *= w;
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) { o[nr][j][e] *= w; o[nr][j][e + 2] *= w; }
                    }
            }
            uint32_t pb[MT][NR][2];        // P^T: keys mt * 16 + 2 quad and the next (+ 8: [1]), row 8 nr + r0
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                const float me[2] = {m[nr][0] == -INFINITY ? T8_SHIFT : T8_SHIFT - m[nr][0], m[nr][1] == -INFINITY ? T8_SHIFT : T8_SHIFT - m[nr][1]};
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float w0 = ex2(fmaf(x[mt][nr][2 * h], sc[nr][0], me[0])), w1 = ex2(fmaf(x[mt][nr][2 * h + 1], sc[nr][1], me[1]));
                        l[nr][0] += w0;
                        l[nr][1] += w1;
                        pb[mt][nr][h] = transposed(pack2_f16(w0, w1));
                    }
            }
            bool odd = false;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                uint32_t vx[4][JW];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int key = 2 * quad + (k & 1) + 8 * (k >> 1);
                    const unsigned char *src = block + SM::K_BYTES + (mt * 16 + key) * D + chunk_at<D>(key, r0 * J / 16) * 16 + r0 * J % 16;
                    if constexpr (JW == 4) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(src);
                        vx[k][0] = u.x; vx[k][1] = u.y; vx[k][2] = u.z; vx[k][3] = u.w;
                    } else {
                        const uint2 u = *reinterpret_cast<const uint2 *>(src);
                        vx[k][0] = u.x; vx[k][1] = u.y;
                    }
                }
                if (edge && own) {
                    // NaN codes of the tree's rows are left out here and given below to the rows that see them
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int e = 0; e < JW; ++e)
                            if (nan_codes(vx[k][e])) { vx[k][e] = without_nans(vx[k][e]); odd = true; }
                }
#pragma unroll
                for (int w = 0; w < JW; ++w) {
                    // keys 2 quad and 2 quad + 1 side by side, columns 4 w + [0, 2) and [2, 4); the same of the keys 8 behind
                    const uint32_t a = __byte_perm(vx[0][w], vx[1][w], 0x5140), a2 = __byte_perm(vx[0][w], vx[1][w], 0x7362);
                    const uint32_t c = __byte_perm(vx[2][w], vx[3][w], 0x5140), c2 = __byte_perm(vx[2][w], vx[3][w], 0x7362);
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) {
                        mma16816_f16(o[nr][2 * w], f16x2_lo(a), f16x2_hi(a), f16x2_lo(c), f16x2_hi(c), pb[mt][nr][0], pb[mt][nr][1]);
                        mma16816_f16(o[nr][2 * w + 1], f16x2_lo(a2), f16x2_hi(a2), f16x2_lo(c2), f16x2_hi(c2), pb[mt][nr][0], pb[mt][nr][1]);
                    }
                }
            }
            if (edge && own && __any_sync(0xffffffffu, odd))
#pragma unroll 1
                for (int k = 0; k < SM::KEYS; ++k) {
                    const int a = first + k - L;
                    if (a >= p.T) break;
                    const long long at = row_at(t, k / 16, page_of(t, k / 16));
                    if (at < 0) continue;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint8_t y = pp.v[at + k % 16 * p.pages.stride_t + r0 * J + 2 * j + (e >> 1)];
                            // (the shared keys and those in front of the tree are seen by all)
#pragma unroll
                            for (int nr = 0; nr < NR; ++nr)
                                if ((y & 0x7fu) == 0x7fu && (a < 0 || (see[nr][e & 1] >> a & 1u))) o[nr][j][e] = __int_as_float(0x7fffffff);
                        }
                }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();                   // the ring is the joining's now
        // ---- the warps' shares of a row are joined: o[nr][j][e] is row 8 nr + 2 quad + (e & 1), column r0 * J + 2 j + (e >> 1)
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = 8 * nr + 2 * quad + e;
                float sum = l[nr][e];
#pragma unroll
                for (int k = 4; k < 32; k *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, k);
                if (r0 == 0) ml_x[warp][row] = make_float2(m[nr][e], sum);
#pragma unroll
                for (int j = 0; j < D / 16; ++j) *reinterpret_cast<float2 *>(&o_x[warp][row][r0 * J + 2 * j]) = make_float2(o[nr][j][e], o[nr][j][e + 2]);
            }
        __syncthreads();
        const bool direct = p.shared == 0 && t1 - t0 == steps;      // the item's only piece
        const size_t slot = (size_t)item + worker;
        const float vs = pp.v_scale[g];
#pragma unroll 1
        for (int e = threadIdx.x; e < rows * (D / 8); e += WARPS * 32) {
            const int row = e % rows, chunk = e / rows;
            float mm = -INFINITY;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) mm = max_nan(mm, ml_x[w][row].x);
            float acc[8] = {}, ll = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float2 ml = ml_x[w][row];
                const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - mm);
                ll = fmaf(f, ml.y, ll);
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] = fmaf(f, o_x[w][row][chunk * 8 + k], acc[k]);
            }
            const float factor = direct ? vs / ll : vs;
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] *= factor;
            if (direct) {
                const int n = row / p.G;
                *reinterpret_cast<uint4 *>(p.out + (((size_t)b * p.T + n) * p.Hq + g * p.G + row - n * p.G) * D + chunk * 8) =
                    make_uint4(pack2_bf16(acc[0], acc[1]), pack2_bf16(acc[2], acc[3]), pack2_bf16(acc[4], acc[5]), pack2_bf16(acc[6], acc[7]));
            } else {
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(acc[k]);
                ptx::st_global_32(ph.o + ((slot * (D / 8) + chunk) * TH_ROWS + row) * 8, w);
                if (chunk == 0) ph.ml[slot * TH_ROWS + row] = make_float2(ll == 0.f ? -INFINITY : mm - T8_SHIFT, ll);
            }
        }
        __syncthreads();                   // before the next piece's codes
    }
}

// ---------------------------------------------------------------------------------------- host
template <int D>
static int launch_paged8(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const P8Params &p, cudaStream_t stream) {
    static PerDeviceOnce once;
    bool *done = once.flag();
    if (!done || !*done) {
        MTV_CUDA_CHECK(cudaFuncSetAttribute(paged_attn8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, P8Smem<D>::TOTAL));
        MTV_CUDA_CHECK(cudaFuncSetAttribute(paged_attn8_thin_kernel<D, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, T8<D, 1>::TOTAL));
        MTV_CUDA_CHECK(cudaFuncSetAttribute(paged_attn8_thin_kernel<D, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, T8<D, 2>::TOTAL));
        if (done) *done = true;
    }
    const PaPhase (&ph)[3] = p.a.phase;
    if (ph[0].prefix_items + ph[0].seq_items + ph[1].prefix_items + ph[1].seq_items)
        MTV_CUDA_CHECK(launch_dependent(paged_attn8_kernel<D>, dim3(sm_count()), P8_THREADS, P8Smem<D>::TOTAL, stream, q, k, v, p));
    if (ph[2].prefix_items + ph[2].seq_items) {
        // at most 8 rows in every item: products of 8
        const int rows = (ph[2].prefix_items ? p.a.B : 1) * p.a.T * p.a.G;
        if (rows <= 8) MTV_CUDA_CHECK(launch_dependent(paged_attn8_thin_kernel<D, 1>, dim3(2 * sm_count()), T8<D, 1>::WARPS * 32, T8<D, 1>::TOTAL, stream, p));
        else MTV_CUDA_CHECK(launch_dependent(paged_attn8_thin_kernel<D, 2>, dim3(2 * sm_count()), T8<D, 2>::WARPS * 32, T8<D, 2>::TOTAL, stream, p));
    }
    return pa_combine(p.a, D, stream);
}

}  // namespace mtv

extern "C" int tree_verify_attention_paged_fp8(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, const mtv_bf16 *q, const uint8_t *k_pool,
                                               const uint8_t *v_pool, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                               int shared_len, const int32_t *seq_lens, const float *k_scale, const float *v_scale, float scale,
                                               mtv_bf16 *out, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
    using namespace mtv;
    MTV_RANGE("tree_verify_attention_paged_fp8");
    if (!tree || !tree->on_device || !q || !k_pool || !v_pool || !seq_lens || !k_scale || !v_scale || !out || !ws) return MTV_ERR_INVALID_ARG;
    if (B < 1 || Hq < 1 || Hkv < 1 || shared_len < 0 || !(scale >= 0.f) || scale > 1e30f) return MTV_ERR_INVALID_ARG;
    if (!pa_sizes_ok(tree, B, Hq, Hkv, D, shared_len)) return MTV_ERR_UNSUPPORTED_SHAPE;
    P8Params pp = {};
    PaParams &p = pp.a;
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D, 16);
    if (rc != MTV_OK) return rc;
    if (shared_len % pool->page_size || shared_len > (int64_t)max_pages * pool->page_size ||
        (((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_pool | (uintptr_t)v_pool) & 15) || ((uintptr_t)ws & 255))
        return MTV_ERR_INVALID_ARG;
    p.T = tree->T; p.B = B; p.G = Hq / Hkv; p.Hq = Hq; p.Hkv = Hkv;
    p.shared = shared_len;
    if (ws_bytes < pa_plan(p.phase, sm_count(), p.T, B, p.G, Hkv, D, shared_len, static_cast<char *>(ws))) return MTV_ERR_WORKSPACE;
    if (!pa_lines_ok(p.phase, B, shared_len, (int64_t)max_pages * pool->page_size)) return MTV_ERR_UNSUPPORTED_SHAPE;
    p.npc = 128 / p.G;
    p.page_rows = pool->page_size < PA_KEYS ? pool->page_size : PA_KEYS;
    p.seq_lens = seq_lens; p.anc = tree->d_anc;
    p.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    p.out = reinterpret_cast<__nv_bfloat16 *>(out);
    p.status = status; p.dev_error = tree->d_error;
    p.scale_log2 = (scale == 0.f ? 1.f / sqrtf((float)D) : scale) * 1.4426950408889634f;
    pp.k = k_pool; pp.v = v_pool; pp.k_scale = k_scale; pp.v_scale = v_scale;
    CUtensorMap q_map = {}, k_map = {}, v_map = {};
    const PaPhase (&ph)[3] = p.phase;
    if (ph[0].prefix_items + ph[0].seq_items + ph[1].prefix_items + ph[1].seq_items) {      // (thin items need no maps)
        const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)Hq, (cuuint64_t)B * p.T, 1};
        const cuuint64_t str[3] = {(cuuint64_t)D * 2, (cuuint64_t)Hq * D * 2, (cuuint64_t)B * p.T * Hq * D * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)p.G, (cuuint32_t)p.npc, 1};
        if (!encode_map_bf16(&q_map, q, 4, dims, str, box)) return MTV_ERR_CUDA;
        const cuuint64_t dims8[4] = {(cuuint64_t)D, (cuuint64_t)pool->page_size, (cuuint64_t)Hkv, (cuuint64_t)pool->n_pages};
        const cuuint64_t str8[3] = {(cuuint64_t)pool->stride_t, (cuuint64_t)pool->stride_h, (cuuint64_t)pool->stride_page};
        const cuuint32_t box8[4] = {(cuuint32_t)D, (cuuint32_t)p.page_rows, 1, 1};
        if (!encode_map_bytes(&k_map, k_pool, 4, dims8, str8, box8, D) || !encode_map_bytes(&v_map, v_pool, 4, dims8, str8, box8, 0)) return MTV_ERR_CUDA;
    }
    return D == 128 ? launch_paged8<128>(q_map, k_map, v_map, pp, (cudaStream_t)stream) : launch_paged8<64>(q_map, k_map, v_map, pp, (cudaStream_t)stream);
}
