// Tree attention over a K/V cache in pages, of a batch whose first keys are the same (Section 3.2 / Fig. 2(b)), on the 5th-generation
// tensor cores.  Two launches: the products and running softmax of all pieces, and their combination.
//
// A row tile is 128 / G whole tree nodes times the G query heads of a KV head: 128 rows of a tensor-core product (fewer where G does not
// divide 128; the others idle).  Behind the shared prefix the nodes of all sequences follow one another, and a tile takes them as they
// come: every shared key is loaded and multiplied once per tile, whoever the rows belong to.  Behind it a tile holds nodes of one
// sequence.  An ITEM is a KV head's keys (the prefix, or one sequence's own) for two row tiles, or for the one that is left over where
// their number is odd; its keys come in tiles of 128.  Items of two row tiles and items of one are worked off one kind
// after the other (the PHASES of the kernel), each laid out on a line on which a key tile counts TILE_COST and the start and end of an item
// ITEM_COST, and each line is cut into equal runs, one per worker.  A worker's PIECE of an item leaves O (fp32, unnormalised) and the running
// (max, sum) of its rows in the workspace, and the second kernel joins the pieces; an item that is one worker's alone and has no prefix
// beside it is written out directly.
//
// One persistent CTA per SM.  Both phases keep two row tiles in flight, each with its own scores S / weights P and accumulator O in tensor
// memory and its own four softmax warps (a thread per row): while the tensor core works for one, the other's exponentials are
// taken.  In the phase of pairs the two tiles are those of an item and share K and V; in the other the CTA is two workers, whose K and V
// take turns in one ring.  Warp 8 issues all products, in the order  O_0 += P_0 V, S_0 = Q_0 K, O_1 += P_1 V, S_1 = Q_1 K  with S one key
// tile ahead of O: products of one thread are executed in order, so S may overwrite the P that the product in front of it reads, and
// "S is complete" implies that O is complete up to the tile before.  Warp 9 requests Q, K and V (a box per page); warp 10 clears V rows behind
// the last key (their weight is 0, but 0 * NaN is not) and takes non-finite values of the tree's V rows out (they are given to the rows that see
// them at the end); warp 11 reports the sequences' status.
//
// The running maximum moves only when a tile's exceeds it by more than 8 (log2 units): O is rescaled rarely and P stays below 2^8.
#include "attn_common.cuh"
#include "paged_common.cuh"

namespace mtv {

constexpr int PA_THREADS = 384;
constexpr int PA_MMA_WARP = 8, PA_TMA_WARP = 9, PA_CLEAN_WARP = 10, PA_STATUS_WARP = 11;
constexpr int PA_KEYS = 128;              // keys of a tile
constexpr int PA_MAX_B = 1024;
constexpr float PA_RESCALE = 8.f;
constexpr int TILE_COST = 4, ITEM_COST = 4;   // what a piece's start and end take, in quarters of a key tile

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
static_assert(sizeof(uint64_t) * (PA_MAX_B + 1) <= PaSmem<64>::OFF_RING, "the sequences' costs are summed in the query tiles' space");

enum {
    PB_FULL = 0, PB_FREE = 10, PB_CLEAN = 20, PB_QFULL = 30, PB_QFREE = 32, PB_SREADY = 34, PB_PREADY = 36, PB_ODONE = 38, PB_FINAL = 40,
    PB_COUNT = 41
};

struct PaPhase {
    int prefix_items, seq_items;       // items of the prefix, and of each sequence
    int prefix_per_head, seq_per_head;
    int prefix_tile0, seq_tile0;       // row tile of a head's first item (0 where an item is a pair)
    int workers, rows;                 // at most; rows of a slot
    float *o;                          // [slots][D / 8][rows][8]
    float2 *ml;                        // [slots][rows]
};
struct PaParams {
    PagedRef pages;
    PaPhase phase[2];                  // pairs of row tiles, single row tiles
    const int32_t *seq_lens;
    const uint64_t *anc;               // [T][2]
    const __nv_bfloat16 *v;
    __nv_bfloat16 *out;
    int32_t *status, *dev_error;
    float scale_log2;
    int B, T, G, Hq, Hkv, shared, npc, page_rows;
};

// ---------------------------------------------------------------------------------------- the division of the work
__device__ __forceinline__ int key_tiles(int keys) { return (keys + PA_KEYS - 1) / PA_KEYS; }
__device__ __forceinline__ uint32_t item_cost(int tiles) { return tiles ? (uint32_t)tiles * TILE_COST + ITEM_COST : 0u; }
// own key tiles of a sequence; 0: it is left out
__device__ __forceinline__ int seq_tiles(const PaParams &p, int L) {
    return p.pages.fits(L, p.T) && L >= p.shared ? key_tiles(L - p.shared + p.T) : 0;
}
// tiles of an item in front of position y of its stretch of the line
__device__ __forceinline__ int cut_at(int64_t y, int tiles) {
    const int64_t t = (y - ITEM_COST + TILE_COST / 2) / TILE_COST;      // (truncation towards zero: below ITEM_COST the first tile is not reached)
    return y <= ITEM_COST ? 0 : t > tiles ? tiles : (int)t;
}
__device__ __forceinline__ uint64_t line_length(const PaParams &p, const PaPhase &f, uint64_t seq_costs) {
    return (uint64_t)f.prefix_items * item_cost(key_tiles(p.shared)) + seq_costs * f.seq_items;
}
// Workers that have a run: none shorter than a key tile, so that no worker in the middle of an item is left without a tile.
__device__ __forceinline__ uint64_t line_workers(const PaPhase &f, uint64_t length) {
    const uint64_t most = length / TILE_COST;
    return most < (uint64_t)f.workers ? most : (uint64_t)f.workers;
}
// cum[b]: costs of an item of each sequence before b, for b <= B.  One warp.
__device__ __forceinline__ void sum_costs(const PaParams &p, uint64_t *cum, int lane) {
    uint64_t before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        uint64_t c = b0 + lane < p.B ? item_cost(seq_tiles(p, p.seq_lens[b0 + lane])) : 0;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint64_t x = __shfl_up_sync(0xffffffffu, c, o);
            if (lane >= o) c += x;
        }
        if (b0 + lane < p.B) cum[b0 + lane + 1] = before + c;
        before += __shfl_sync(0xffffffffu, c, 31);
    }
    if (lane == 0) cum[0] = 0;
}
// A worker's run, and the item it begins in.
struct PaStart {
    uint64_t x0, x1, S;
    int b, idx;
};
__device__ __forceinline__ PaStart find_start(const PaParams &p, const PaPhase &f, const uint64_t *cum, int worker) {
    PaStart r = {};
    const uint64_t W = line_length(p, f, cum[p.B]), n = line_workers(f, W);
    if ((uint64_t)worker >= n) return r;                 // x0 = x1: nothing
    r.x0 = W * worker / n;
    r.x1 = W * (worker + 1) / n;
    const uint64_t cost = item_cost(key_tiles(p.shared)), prefix = cost * f.prefix_items;
    if (r.x0 < prefix) {
        r.b = -1;
        r.idx = (int)(r.x0 / cost);
        r.S = r.idx * cost;
        return r;
    }
    const uint64_t y = r.x0 - prefix;
    int lo = 0, hi = p.B;                                // the last b with cum[b] * seq_items <= y < the next one's
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (cum[mid] * f.seq_items <= y) lo = mid; else hi = mid;
    }
    const uint64_t own = cum[lo + 1] - cum[lo];
    r.b = lo;
    r.idx = own ? (int)((y - cum[lo] * f.seq_items) / own) : 0;
    r.S = prefix + cum[lo] * f.seq_items + r.idx * own;
    return r;
}
struct PaPiece {
    int b;              // -1: the prefix
    int g, tile0;       // KV head, first row tile
    int t0, t1, tiles;  // key tiles [t0, t1) of the item's
    int L;              // keys in front of the tree, without the shared ones (prefix: the shared ones)
    int slot;
};
struct PaWalk {
    uint64_t x0, x1, S;
    int b, idx, tiles, L, worker;
    __device__ __forceinline__ void begin(const PaParams &p, const PaStart &s, int w) {
        x0 = s.x0; x1 = s.x1; S = s.S; b = s.b; idx = s.idx; worker = w;
        if (x0 < x1) load(p);
    }
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
            s.t0 = cut_at((int64_t)x0 - (int64_t)S, tiles);
            s.t1 = cut_at((int64_t)x1 - (int64_t)S, tiles);
            S += item_cost(tiles);
            const int i = idx++;
            if (s.t0 >= s.t1) continue;
            const int per = b < 0 ? f.prefix_per_head : f.seq_per_head;
            s.b = b; s.L = L; s.tiles = tiles;
            s.g = i / per;
            s.tile0 = (b < 0 ? f.prefix_tile0 : f.seq_tile0) + 2 * (i - s.g * per);
            s.slot = (b < 0 ? i : f.prefix_items + b * f.seq_items + i) + worker;
            return true;
        }
        return false;
    }
};
// The tile needs more than its copy: it holds rows of the tree, or rows behind them.
__device__ __forceinline__ bool is_last(const PaPiece &s, int t) { return s.b >= 0 && (t + 1) * PA_KEYS > s.L; }

// All of a phase's key tiles in the order in which the ring holds them: a round takes, list after list, V of the tile before and K of the
// tile after.  f(list, piece and tile of V or none, piece and tile of K or none) -> whether to go on.
template <int NL, typename F>
__device__ __forceinline__ bool for_rounds(const PaParams &p, const PaPhase &ph, const PaStart *starts, int worker, int worker_step, F &&f) {
    PaWalk w[NL];
    PaPiece cur[NL], old[NL];
    int t[NL], old_t[NL];
    bool live[NL], pend[NL];
#pragma unroll
    for (int l = 0; l < NL; ++l) {
        w[l].begin(p, starts[l], worker + l * worker_step);
        live[l] = w[l].next(p, ph, cur[l]);
        t[l] = live[l] ? cur[l].t0 : 0;
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
                    live[l] = w[l].next(p, ph, cur[l]);
                    t[l] = live[l] ? cur[l].t0 : 0;
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
__device__ __forceinline__ bool nonfinite16(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }

__device__ __forceinline__ void pa_cta_sync() { asm volatile("bar.sync 1, %0;" ::"n"(PA_THREADS) : "memory"); }

// ---------------------------------------------------------------------------------------- pieces
template <int D>
__global__ void __launch_bounds__(PA_THREADS, 1)
paged_attn_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                  const __grid_constant__ PaParams p) {
    using SM = PaSmem<D>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ PaStart starts[3];        // pairs; single tiles of either half of the CTA
    let_next_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t raw = ptx::smem_u32(smem_raw), pad = (1024u - (raw & 1023u)) & 1023u, sbase = raw + pad;
    unsigned char *gbase = smem_raw + pad;
    const uint32_t bars = sbase + SM::OFF_BAR;
    auto bar = [&](int i) { return bars + (uint32_t)i * 8u; };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(gbase + SM::OFF_BAR + PB_COUNT * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + PB_COUNT * 8 + 4);
    volatile int *bad = reinterpret_cast<volatile int *>(gbase + SM::OFF_BAR + PB_COUNT * 8 + 8);   // [2][4]: 1 + the last piece with non-finite V

    if (warp == PA_TMA_WARP && lane == 0) {
        ptx::prefetch_tensormap(&q_map);
        ptx::prefetch_tensormap(&k_map);
        ptx::prefetch_tensormap(&v_map);
        for (int s = 0; s < SM::STAGES; ++s) {
            ptx::mbar_init(bar(PB_FULL + s), 1);
            ptx::mbar_init(bar(PB_FREE + s), 2);      // the products, and the warp that looks at every entry
            ptx::mbar_init(bar(PB_CLEAN + s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(bar(PB_QFULL + s), 1);
            ptx::mbar_init(bar(PB_QFREE + s), 1);
            ptx::mbar_init(bar(PB_SREADY + s), 1);
            ptx::mbar_init(bar(PB_PREADY + s), 4);
            ptx::mbar_init(bar(PB_ODONE + s), 1);
        }
        ptx::mbar_init(bar(PB_FINAL), 1);
        ptx::fence_mbar_init();
        *abort_flag = 0;
        for (int k = 0; k < 8; ++k) bad[k] = 0;
    }
    if (warp == PA_MMA_WARP) {
        ptx::tmem_alloc(ptx::smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        ptx::tmem_relinquish();
    }
    previous_done();
    uint64_t *cum = reinterpret_cast<uint64_t *>(gbase);
    if (warp == 0) sum_costs(p, cum, lane);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const int n_cta = gridDim.x, cta = blockIdx.x;
    if (threadIdx.x < 3) starts[threadIdx.x] = find_start(p, p.phase[threadIdx.x > 0], cum, threadIdx.x == 2 ? cta + n_cta : cta);
    __syncthreads();
    const uint32_t tmem = *tmem_slot;
    auto give_up = [&]() {
        *abort_flag = 1;
        atomicExch(p.dev_error, MTV_ERR_TIMEOUT);
    };
    // a whole warp waits; the same answer for all lanes
    auto wait = [&](int b, uint32_t parity) {
        const bool ok = !*abort_flag && ptx::mbar_wait(bar(b), parity);
        if (__all_sync(0xffffffffu, ok)) return true;
        if (lane == 0) give_up();
        return false;
    };

    if (warp == PA_TMA_WARP) {
        // ------------------------------------------------------------ Q, K and V
        ptx::fence_proxy_async();        // the sums above were written where queries are going to land
        int entry = 0, stage = 0, turns = 0;
        int n_q[2] = {0, 0};
        const int boxes = PA_KEYS / p.page_rows, box = lane % boxes, half = lane / boxes;
        const uint32_t q_bytes = (uint32_t)(p.npc * p.G) * 128u * SM::HALVES;
        // this lane's page of a key tile, and the row in it; no page: copied as zeros
        auto find = [&](const PaPiece &s, int t, int *row) {
            const int off = t * PA_KEYS + box * p.page_rows, key = off + (s.b < 0 ? 0 : p.shared);
            *row = key & ((1 << p.pages.page_shift) - 1);
            int page = p.pages.n_pages;
            if (half < SM::HALVES && off < s.L + (s.b < 0 ? 0 : p.T)) {
                const int id = p.pages.table[(int64_t)max(s.b, 0) * p.pages.max_pages + (key >> p.pages.page_shift)];
                if (id >= 0 && id < p.pages.n_pages) page = id;
            }
            return page;
        };
        auto load = [&](const CUtensorMap *map, int page, int row, int g) {
            if (entry >= SM::STAGES && !wait(PB_FREE + stage, (turns - 1) & 1)) return false;
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar(PB_FULL + stage), SM::TILE);
            __syncwarp();
            if (half < SM::HALVES)
                ptx::tma_load_4d(sbase + SM::OFF_RING + stage * SM::TILE + half * SM::HALF + box * p.page_rows * 128, map, bar(PB_FULL + stage),
                                 half * 64, row, g, page);
            ++entry;
            if (++stage == SM::STAGES) { stage = 0; ++turns; }
            return true;
        };
        auto phase = [&](auto lists, const PaPhase &ph, const PaStart *st) {
            constexpr int NL = decltype(lists)::value;
            int v_page[NL] = {}, v_row[NL] = {};
            return for_rounds<NL>(p, ph, st, cta, n_cta, [&](int l, bool v, const PaPiece &vs, int vt, bool k, const PaPiece &ks, int kt) {
                if (v && !load(&v_map, v_page[l], v_row[l], vs.g)) return false;
                if (!k) return true;
                int row;
                const int page = find(ks, kt, &row);
                if (!load(&k_map, page, row, ks.g)) return false;
                v_page[l] = page;
                v_row[l] = row;
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
        if (!phase(std::integral_constant<int, 1>(), p.phase[0], starts) || !phase(std::integral_constant<int, 2>(), p.phase[1], starts + 1)) {
            // copies in flight get a bounded chance to land before the CTA can exit
            for (int e = max(0, entry - SM::STAGES); e < entry; ++e) ptx::mbar_wait(bar(PB_FULL + e % SM::STAGES), (e / SM::STAGES) & 1);
            for (int s = 0; s < 2; ++s)
                if (n_q[s]) ptx::mbar_wait(bar(PB_QFULL + s), (n_q[s] - 1) & 1);
        }
    } else if (warp == PA_MMA_WARP) {
        // ------------------------------------------------------------ all products
        const bool leader = ptx::elect_one();
        const uint32_t dq0 = ptx::desc_lo(sbase, 16), dk0 = ptx::desc_lo(sbase + SM::OFF_RING, 16), dv0 = ptx::desc_lo(sbase + SM::OFF_RING, SM::HALF);
        int entry = 0;
        uint32_t cleaned = 0;            // parity of each stage's next cleaning
        int n_p[2] = {0, 0}, n_q[2] = {0, 0};
        auto phase = [&](auto lists, const PaPhase &ph, const PaStart *st) {
            constexpr int NL = decltype(lists)::value;
            return for_rounds<NL>(p, ph, st, cta, n_cta, [&](int l, bool v, const PaPiece &vs, int vt, bool k, const PaPiece &ks, int kt) {
                const int ve = entry, ke = entry + (v ? 1 : 0);
                entry = ke + (k ? 1 : 0);
                const int v_stage = ve % SM::STAGES, k_stage = ke % SM::STAGES;
                const int s0 = l, s1 = NL == 1 ? 2 : l + 1;
                for (int s = s0; s < s1; ++s) {
                    if (v) {
                        if (s == s0) {
                            if (is_last(vs, vt)) {
                                if (!wait(PB_CLEAN + v_stage, cleaned >> v_stage & 1)) return false;
                                cleaned ^= 1u << v_stage;
                            } else if (!wait(PB_FULL + v_stage, (ve / SM::STAGES) & 1)) {
                                return false;
                            }
                        }
                        if (!wait(PB_PREADY + s, n_p[s]++ & 1)) return false;
                        ptx::tc_fence_after();
                        const uint32_t dv = dv0 + (uint32_t)v_stage * (SM::TILE >> 4);
#pragma unroll
                        for (int kk = 0; kk < PA_KEYS / 16; ++kk)
                            ptx::mma_ts_elect(tmem + 256 + s * D, tmem + s * 128 + kk * 8, dv + kk * 128, ptx::DESC_HI, SM::IDESC_PV, vt > vs.t0 || kk > 0, leader);
                        if (vt == vs.t1 - 1) ptx::tc_commit_elect(bar(PB_ODONE + s), leader);
                        if (s == s1 - 1) ptx::tc_commit_elect(bar(PB_FREE + v_stage), leader);
                    }
                    if (k) {
                        if (s == s0 && !wait(PB_FULL + k_stage, (ke / SM::STAGES) & 1)) return false;
                        if (kt == ks.t0 && !wait(PB_QFULL + s, n_q[s]++ & 1)) return false;
                        ptx::tc_fence_after();
                        const uint32_t dq = dq0 + (uint32_t)s * (SM::TILE >> 4), dk = dk0 + (uint32_t)k_stage * (SM::TILE >> 4);
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t o = ((kk / 4) * SM::HALF + (kk % 4) * 32) >> 4;
                            ptx::mma_ss_elect(tmem + s * 128, dq + o, dk + o, ptx::DESC_HI, SM::IDESC_QK, kk > 0, leader);
                        }
                        ptx::tc_commit_elect(bar(PB_SREADY + s), leader);
                        if (kt == ks.t1 - 1) ptx::tc_commit_elect(bar(PB_QFREE + s), leader);
                        if (s == s1 - 1) ptx::tc_commit_elect(bar(PB_FREE + k_stage), leader);
                    }
                }
                return true;
            });
        };
        phase(std::integral_constant<int, 1>(), p.phase[0], starts) && phase(std::integral_constant<int, 2>(), p.phase[1], starts + 1);
        // what was issued is complete, and has signalled, before the CTA can exit
        ptx::tc_commit_elect(bar(PB_FINAL), leader);
        ptx::mbar_wait(bar(PB_FINAL), 0);
    } else if (warp == PA_CLEAN_WARP) {
        // ------------------------------------------------------------ the last V tiles of a sequence
        int stage = 0, turns = 0, n_piece[2] = {0, 0};
        auto phase = [&](auto lists, const PaPhase &ph, const PaStart *st) {
            constexpr int NL = decltype(lists)::value;
            return for_rounds<NL>(p, ph, st, cta, n_cta, [&](int l, bool v, const PaPiece &vs, int vt, bool k, const PaPiece &ks, int kt) {
                // Every entry is waited for, and handed back by this warp too: a parity wait cannot tell a phase from the one two
                // before or behind, so nobody may be a turn of the ring ahead or late.
                auto landed = [&]() { return wait(PB_FULL + stage, turns & 1); };
                auto pass = [&]() {
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(PB_FREE + stage));
                    if (++stage == SM::STAGES) { stage = 0; ++turns; }
                };
                if (v && !landed()) return false;
                if (v && is_last(vs, vt)) {
                    const int first = max(0, vs.L - vt * PA_KEYS), end = vs.L + p.T - vt * PA_KEYS;
                    bool odd = false;
#pragma unroll
                    for (int h = 0; h < SM::HALVES; ++h) {
                        uint4 *x = reinterpret_cast<uint4 *>(gbase + SM::OFF_RING + stage * SM::TILE + h * SM::HALF);
                        for (int e = first * 8 + lane; e < PA_KEYS * 8; e += 32) {
                            if (e / 8 >= end) {
                                x[e] = make_uint4(0u, 0u, 0u, 0u);
                                continue;
                            }
                            const uint4 u = x[e];
                            uint32_t w[4] = {u.x, u.y, u.z, u.w};
                            bool here = false;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (nonfinite16(w[i])) { w[i] &= 0xffff0000u; here = true; }
                                if (nonfinite16(w[i] >> 16)) { w[i] &= 0xffffu; here = true; }
                            }
                            if (here) x[e] = make_uint4(w[0], w[1], w[2], w[3]);
                            odd = odd || here;
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
        phase(std::integral_constant<int, 1>(), p.phase[0], starts) && phase(std::integral_constant<int, 2>(), p.phase[1], starts + 1);
    } else if (warp == PA_STATUS_WARP) {
        // ------------------------------------------------------------ which sequences can be attended to
        if (p.status && cta < p.B) {
            const int prefix = p.pages.check(0, 0, p.shared, lane);
            for (int b = cta; b < p.B; b += n_cta) {
                const int L = p.seq_lens[b];
                int code = seq_tiles(p, L) ? p.pages.check(b, p.shared, L - p.shared + p.T, lane) : MTV_ERR_CAPACITY;
                if (code == MTV_OK) code = prefix;
                if (lane == 0) p.status[b] = code;
            }
        }
    } else {
        // ------------------------------------------------------------ softmax: a thread per row of row tile s
        const int s = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lane_base + s * 128, t_o = tmem + lane_base + 256 + s * D;
        const int node_in_tile = row / p.G, head = row % p.G;
        const bool in_tile = node_in_tile < p.npc;
        const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
        int n_s = 0, n_piece = 0;
        bool ok = true;
        for (int f = 0; f < 2 && ok; ++f) {
            const PaPhase &ph = p.phase[f];
            PaWalk walk;
            PaPiece pc;
            walk.begin(p, starts[f ? 1 + s : 0], f ? cta + s * n_cta : cta);
            while (ok && walk.next(p, ph, pc)) {
                const int node = (pc.tile0 + (f ? 0 : s)) * p.npc + node_in_tile;
                const bool mine = in_tile && node < (pc.b < 0 ? p.B * p.T : p.T);
                const bool some = __any_sync(0xffffffffu, mine);
                uint64_t alo = 0, ahi = 0;
                if (mine && pc.b >= 0) { alo = p.anc[node * 2]; ahi = p.anc[node * 2 + 1]; }
                // visibility of the tree rows as 32-bit words; the rows in front of them are visible to every node, those behind to none
                auto anc_word = [&](int w) -> uint32_t {
                    return w < 0 ? 0xffffffffu : w == 0 ? (uint32_t)alo : w == 1 ? (uint32_t)(alo >> 32) : w == 2 ? (uint32_t)ahi : w == 3 ? (uint32_t)(ahi >> 32) : 0u;
                };
                float m_used = -INFINITY, l = 0.f;
                for (int t = pc.t0; t < pc.t1; ++t) {
                    if (!wait(PB_SREADY + s, n_s++ & 1)) { ok = false; break; }
                    ptx::tc_fence_after();
                    if (some) {
                        uint32_t sr[128];
#pragma unroll
                        for (int h = 0; h < 4; ++h) ptx::tmem_ld32(t_s + h * 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[h * 32]));
#pragma unroll
                        for (int h = 0; h < 4; ++h) ptx::tmem_ld_wait_for(*reinterpret_cast<uint32_t(*)[32]>(&sr[h * 32]));
                        if ((t + 1) * PA_KEYS > pc.L) {
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                const int a0 = t * PA_KEYS + h * 32 - pc.L;      // tree row of the first column
                                const uint32_t vis = __funnelshift_r(anc_word(a0 >> 5), anc_word((a0 >> 5) + 1), a0 & 31);
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!((vis >> e) & 1u)) sr[h * 32 + e] = 0xff800000u;   // -inf
                            }
                        }
                        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int e = 0; e < 128; e += 8)
#pragma unroll
                            for (int k = 0; k < 4; ++k) mx[k] = max3_nan(mx[k], __uint_as_float(sr[e + 2 * k]), __uint_as_float(sr[e + 2 * k + 1]));
                        float mxs = max_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3]) * p.scale_log2;
                        if (mxs == INFINITY) mxs = __int_as_float(0x7fffffff);     // inf - inf: the row is NaN, as from the formula
                        const float m_new = mxs <= m_used + PA_RESCALE ? m_used : mxs;   // (a NaN is taken over)
                        const bool need = t > pc.t0 && m_new != m_used && m_used != -INFINITY && mine;
                        if (__any_sync(0xffffffffu, need)) {
                            const float alpha = need ? ex2(m_used - m_new) : 1.f;
#pragma unroll 1
                            for (int h = 0; h < D / 16; ++h) {
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
                        const float m_eff = m_used == -INFINITY ? 0.f : m_used;
                        const float2 nm2 = make_float2(-m_eff, -m_eff);
                        float2 la = make_float2(0.f, 0.f), lb = make_float2(0.f, 0.f);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t pk[32];
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                const uint32_t *x = sr + h * 64 + 2 * e;
                                const float2 x01 = __ffma2_rn(make_float2(__uint_as_float(x[0]), __uint_as_float(x[1])), sc2, nm2);
                                const float2 x23 = __ffma2_rn(make_float2(__uint_as_float(x[2]), __uint_as_float(x[3])), sc2, nm2);
                                const float2 p01 = make_float2(ex2(x01.x), ex2(x01.y)), p23 = make_float2(ex2(x23.x), ex2(x23.y));
                                la = __fadd2_rn(la, p01);
                                lb = __fadd2_rn(lb, p23);
                                pk[e] = pack2_bf16(p01.x, p01.y);
                                pk[e + 1] = pack2_bf16(p23.x, p23.y);
                            }
                            ptx::tmem_st32(t_s + h * 32, pk);
                        }
                        l += (la.x + la.y) + (lb.x + lb.y);
                        ptx::tmem_st_wait();
                    }
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar(PB_PREADY + s));
                }
                if (!ok) break;
                if (!wait(PB_ODONE + s, n_piece & 1)) { ok = false; break; }
                ptx::tc_fence_after();
                if (some) {
                    const bool odd = bad[s * 4 + (n_piece & 3)] == n_piece + 1;
                    const bool direct = p.shared == 0 && pc.t0 == 0 && pc.t1 == pc.tiles;
                    const float inv = direct ? 1.f / l : 1.f;
                    const int slot_row = f ? row : s * 128 + row;
                    float *o_out = ph.o + (size_t)pc.slot * ph.rows * D + (size_t)slot_row * 8;
                    __nv_bfloat16 *out = p.out + (((size_t)max(pc.b, 0) * p.T + node) * p.Hq + pc.g * p.G + head) * D;
#pragma unroll 1
                    for (int h = 0; h < D / 16; ++h) {
                        uint32_t o[16];
                        ptx::tmem_ld16(t_o + h * 16, o);
                        ptx::tmem_ld_wait_for16(o);
                        if (odd && mine) {
                            // V values that the tensor core did not see: an infinity or NaN with any weight is itself
                            for (int a = max(0, pc.t0 * PA_KEYS - pc.L); a < p.T && pc.L + a < pc.t1 * PA_KEYS; ++a) {
                                if (!((a < 64 ? alo >> a : ahi >> (a - 64)) & 1)) continue;
                                const int64_t at = p.pages.row(pc.b, p.shared + pc.L + a);
                                if (at < 0) continue;
                                const uint16_t *v = reinterpret_cast<const uint16_t *>(p.v) + at + pc.g * p.pages.stride_h + h * 16;
#pragma unroll
                                for (int e = 0; e < 16; ++e)
                                    if (nonfinite16(v[e])) o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float((uint32_t)v[e] << 16));
                            }
                        }
                        if (!mine) continue;
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
                    if (mine && !direct) ph.ml[(size_t)pc.slot * ph.rows + slot_row] = make_float2(m_used, l);
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

// ---------------------------------------------------------------------------------------- their combination
// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s over the pieces s of a row's two items (the prefix' and the sequence's own), in the order
// of the keys whoever worked them off.  A thread takes 8 columns of a row: neighbouring threads neighbouring rows, as the slots are laid out.
struct PaSource {
    const float *o;       // slot of the first piece, at the row
    const float2 *ml;
    int n, rows;
};
__device__ __forceinline__ PaSource find_source(const PaParams &p, const PaPhase &f, const uint64_t *cum, uint64_t S, int tiles, int item, int row, int D) {
    const uint64_t W = line_length(p, f, cum[p.B]), n = line_workers(f, W);
    // first: the last worker that begins at or before the item (the next one, if that one's run ends before the first tile); last: the
    // last worker that begins before its end and has a tile of it
    uint64_t w = S * n / W;
    while (w > 0 && W * w / n > S) --w;
    while (w + 1 < n && W * (w + 1) / n <= S) ++w;
    while (w + 1 < n && cut_at((int64_t)(W * (w + 1) / n) - (int64_t)S, tiles) == 0) ++w;
    const uint64_t end = S + item_cost(tiles);
    uint64_t last = (end - 1) * n / W;
    if (last >= n) last = n - 1;
    while (last + 1 < n && W * (last + 1) / n < end) ++last;
    while (last > w && cut_at((int64_t)(W * last / n) - (int64_t)S, tiles) >= tiles) --last;
    PaSource r;
    const size_t slot = (size_t)item + w;
    r.o = f.o + slot * f.rows * D + (size_t)row * 8;
    r.ml = f.ml + slot * f.rows + row;
    r.n = (int)(last - w) + 1;
    r.rows = f.rows;
    return r;
}

template <int D>
__global__ void __launch_bounds__(256)
paged_attn_combine_kernel(const __grid_constant__ PaParams p) {
    constexpr int CHUNKS = D / 8, ROWS = 256 / CHUNKS;
    __shared__ uint64_t cum[PA_MAX_B + 1];
    __shared__ PaSource src[2][ROWS];
    __shared__ int64_t out_at[ROWS];
    let_next_start();
    previous_done();
    const int tid = threadIdx.x;
    if (tid < 32) sum_costs(p, cum, tid);
    __syncthreads();
    const int per_seq = p.T * p.G;
    if (tid < ROWS) {
        const int64_t r = (int64_t)blockIdx.x * ROWS + tid;
        const int64_t bg = r / per_seq;
        const int b = (int)(bg / p.Hkv), g = (int)(bg % p.Hkv), x = (int)(r % per_seq), node = x / p.G, head = x % p.G;
        out_at[tid] = -1;
        src[0][tid].n = src[1][tid].n = 0;
        const int tiles = b < p.B ? seq_tiles(p, p.seq_lens[b]) : 0;
        if (tiles) {
            // row tile and row in it -> phase, item and row of the slot
            auto find = [&](int n, bool prefix) {
                const int tile = n / p.npc, per = prefix ? p.phase[0].prefix_per_head : p.phase[0].seq_per_head;
                const int k = tile / 2 < per ? 0 : 1;
                const PaPhase &f = p.phase[k];
                const int row = (k ? 0 : (tile & 1) * 128) + (n - tile * p.npc) * p.G + head;
                const int i = k ? g : g * per + tile / 2;
                const uint64_t cost = item_cost(key_tiles(p.shared));
                if (prefix) return find_source(p, f, cum, i * cost, key_tiles(p.shared), i, row, D);
                return find_source(p, f, cum, f.prefix_items * cost + cum[b] * f.seq_items + (uint64_t)i * item_cost(tiles), tiles,
                                   f.prefix_items + b * f.seq_items + i, row, D);
            };
            if (p.shared) src[0][tid] = find(b * p.T + node, true);
            src[1][tid] = find(node, false);
            // a single piece was written out by the kernel before
            if (p.shared || src[1][tid].n > 1) out_at[tid] = (((int64_t)b * p.T + node) * p.Hq + g * p.G + head) * D;
        }
    }
    __syncthreads();
    const int row = tid % ROWS, chunk = tid / ROWS;
    if (out_at[row] < 0) return;
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const PaSource s = src[k][row];
        for (int i = 0; i < s.n; ++i) m = max_nan(m, s.ml[(size_t)i * s.rows].x);
    }
    float acc[8] = {}, l = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const PaSource s = src[k][row];
#pragma unroll 4
        for (int i = 0; i < s.n; ++i) {
            const float2 ml = s.ml[(size_t)i * s.rows];
            const float4 *o = reinterpret_cast<const float4 *>(s.o + ((size_t)i * CHUNKS + chunk) * s.rows * 8);
            const float4 a = o[0], c = o[1];
            const float w = ml.x == -INFINITY ? 0.f : ex2(ml.x - m);
            l = fmaf(w, ml.y, l);
            acc[0] = fmaf(w, a.x, acc[0]); acc[1] = fmaf(w, a.y, acc[1]); acc[2] = fmaf(w, a.z, acc[2]); acc[3] = fmaf(w, a.w, acc[3]);
            acc[4] = fmaf(w, c.x, acc[4]); acc[5] = fmaf(w, c.y, acc[5]); acc[6] = fmaf(w, c.z, acc[6]); acc[7] = fmaf(w, c.w, acc[7]);
        }
    }
    const float inv = 1.f / l;
    *reinterpret_cast<uint4 *>(p.out + out_at[row] + chunk * 8) = make_uint4(pack2_bf16(acc[0] * inv, acc[1] * inv), pack2_bf16(acc[2] * inv, acc[3] * inv),
                                                                            pack2_bf16(acc[4] * inv, acc[5] * inv), pack2_bf16(acc[6] * inv, acc[7] * inv));
}

// ---------------------------------------------------------------------------------------- host
// The phases of a call and the layout of its workspace; returns the bytes.
static size_t pa_plan(PaPhase (&ph)[2], int T, int B, int G, int Hkv, int D, int shared, char *ws) {
    const int npc = 128 / G, sms = sm_count();
    const int prefix_tiles = shared ? (B * T + npc - 1) / npc : 0, seq_tiles = (T + npc - 1) / npc;
    size_t at = 0;
    for (int f = 0; f < 2; ++f) {
        PaPhase &x = ph[f];
        x.prefix_per_head = f ? prefix_tiles % 2 : prefix_tiles / 2;
        x.seq_per_head = f ? seq_tiles % 2 : seq_tiles / 2;
        x.prefix_items = Hkv * x.prefix_per_head;
        x.seq_items = Hkv * x.seq_per_head;
        x.prefix_tile0 = f ? prefix_tiles - 1 : 0;
        x.seq_tile0 = f ? seq_tiles - 1 : 0;
        x.workers = f ? 2 * sms : sms;
        x.rows = f ? 128 : 256;
        const size_t items = (size_t)x.prefix_items + (size_t)B * x.seq_items;
        const size_t slots = items ? items + x.workers : 0;     // a piece's slot: its item's number plus its worker's
        x.o = reinterpret_cast<float *>(ws + at);
        at += align_up(slots * x.rows * D * sizeof(float), 256);
        x.ml = reinterpret_cast<float2 *>(ws + at);
        at += align_up(slots * x.rows * sizeof(float2), 256);
    }
    return at;
}

static bool pa_sizes_ok(const mtv_tree *tree, int B, int Hq, int Hkv, int D, int shared) {
    return tree && B >= 1 && B <= PA_MAX_B && Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0 && Hq / Hkv <= 8 && (D == 64 || D == 128) && shared >= 0 &&
           (int64_t)Hkv * B * tree->T <= 1 << 28;
}

template <int D>
static int launch_paged(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const PaParams &p, cudaStream_t stream) {
    static PerDeviceOnce once;
    bool *done = once.flag();
    if (!done || !*done) {
        MTV_CUDA_CHECK(cudaFuncSetAttribute(paged_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, PaSmem<D>::TOTAL));
        if (done) *done = true;
    }
    MTV_CUDA_CHECK(launch_dependent(paged_attn_kernel<D>, dim3(sm_count()), PA_THREADS, PaSmem<D>::TOTAL, stream, q, k, v, p));
    const int64_t rows = (int64_t)p.B * p.Hkv * p.T * p.G;
    const int per_block = 256 / (D / 8);
    MTV_CUDA_CHECK(launch_dependent(paged_attn_combine_kernel<D>, dim3((unsigned)((rows + per_block - 1) / per_block)), 256, 0, stream, p));
    return MTV_OK;
}

}  // namespace mtv

extern "C" size_t tree_attention_paged_workspace_bytes(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int shared_len) {
    using namespace mtv;
    if (!pa_sizes_ok(tree, B, Hq, Hkv, D, shared_len)) return 0;
    PaPhase ph[2];
    return pa_plan(ph, tree->T, B, Hq / Hkv, Hkv, D, shared_len, nullptr);
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
    if (ws_bytes < pa_plan(p.phase, p.T, B, p.G, Hkv, D, shared_len, static_cast<char *>(ws))) return MTV_ERR_WORKSPACE;
    p.npc = 128 / p.G;
    p.page_rows = pool->page_size < PA_KEYS ? pool->page_size : PA_KEYS;
    p.seq_lens = seq_lens; p.anc = tree->d_anc;
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
