// What the kernels of the attention over pages share, whatever its rows are held in: parameters, pieces of work and their order, the joining's entry.
#pragma once
#include "attn_common.cuh"
#include "paged_common.cuh"
#include "paged_plan.cuh"

namespace mtv {

constexpr int PA_QUEUE = 4;               // pieces that are handed out and may not have been taken by all
constexpr int PA_KEYS = 128;              // keys of a tile
constexpr int PA_MAX_B = 1024;
constexpr int TILE_COST = 4;              // a key tile on a line
// What the start and end of an item take, in the same quarters of a key tile, for pairs and for single row tiles.  With codes, replayed graphs: 8 for pairs takes a 16k document of 8
// trees from 131 to 147 us and 16 trees of 64 nodes from 59 to 62, 24 these from 59 to 62.6; at D = 64 the latter 47.3 with 16, 47.9 with 8, 49.7 with 24.  Single row tiles
// (16 trees of 29 nodes) take 46 us with 4, 8, 12 or 16, at D = 64 38.
__host__ __device__ constexpr int ITEM_COST(int single) { return single ? 8 : 16; }

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
// The runs of the workers of a CTA (pairs; single tiles of its halves) and the items they begin in.  One warp.  The costs: what a quarter of a key
// tile takes a CTA in the one phase and in the other.
__device__ __forceinline__ void begin_walks(const PaParams &p, PaWalk (&w)[3], int cta, int n_cta, int lane, int cost_pairs, int cost_single) {
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
        const float a = (float)length[0] * cost_pairs, b = (float)length[1] * cost_single;
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
// ... whether all of them do.
__device__ __forceinline__ bool all_of_rows(int barrier, bool mine) {
    uint32_t r;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "barrier.cta.red.and.pred q, %2, 64, p;\n"
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

// ---------------------------------------------------------------------------------------- thin items
// The line of all thin items, in steps of STEP keys of which an item's start and end take ENDS more, and a worker's run of it.
template <int STEP, int ENDS> struct ThinLine {
    static __device__ __forceinline__ int steps(int keys) { return (keys + STEP - 1) / STEP; }
    // of an item of sequence b; 0: it is left out
    static __device__ __forceinline__ int cost_of(const PaParams &p, int b) {
        const int L = b < p.B ? p.seq_lens[b] : -1;
        return L >= 0 && p.pages.fits(L, p.T) && L >= p.shared ? steps(L - p.shared + p.T) + ENDS : 0;
    }
    // One warp: start = the run x0, x1, the position S, sequence b and index idx of the item that it begins in.
    static __device__ __forceinline__ void begin(const PaParams &p, int worker, int workers, int lane, int (&start)[5]) {
        const PaPhase &ph = p.phase[2];
        const int own0 = cost_of(p, lane);
        int total = own0;
        for (int b0 = 32; b0 < p.B; b0 += 32) total += cost_of(p, b0 + lane);
        total = __reduce_add_sync(0xffffffffu, total);
        const int each = steps(p.shared) + ENDS, prefix = ph.prefix_items * each, length = prefix + total * ph.seq_items;
        const int run = max((length + workers - 1) / workers, 1), x0 = (int)min((int64_t)length, (int64_t)run * worker), x1 = (int)min((int64_t)length, (int64_t)x0 + run);
        int b = -1, idx = 0, S = x1;
        if (x0 < x1 && x0 < prefix) {
            idx = x0 / each;
            S = idx * each;
        } else if (x0 < x1) {
            const int y = x0 - prefix;
            int before = 0;
            for (int b0 = 0; b0 < p.B; b0 += 32) {
                const int own = b0 ? cost_of(p, b0 + lane) : own0;
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
};

// The checks of a call's sizes, and the second launch: joins the pieces (attention_paged.cu).
bool pa_sizes_ok(const mtv_tree *tree, int B, int Hq, int Hkv, int D, int shared);
bool pa_lines_ok(const PaPhase (&ph)[3], int B, int shared, int64_t slots);
int pa_combine(const PaParams &p, int D, cudaStream_t stream);

}  // namespace mtv
