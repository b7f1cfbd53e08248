// A K/V cache in pages: rows appended with the rotary embedding, and the accepted rows of a step moved to the front of the tree's
// slots (Section 3.2, "Tensorization of Tree Topology" and "Zero-Copy Retrieval"; the paper's own cache is contiguous).
// Slot s of sequence b is row s % page of page page_table[b][s / page]; page sizes are powers of two.
#include "paged_common.cuh"

namespace mtv {

constexpr int PAGED_THREADS = 256;
constexpr int APPEND_DEEP = 1;       // pairs of 16-byte chunks that a thread asks for at a time
constexpr int PAGED_MAX_HEADS = 4096;
constexpr int APPEND_ROWS = 2;       // rows of a block

// (x[d], x[d + D/2]) -> (x[d] cos - x[d + D/2] sin, x[d + D/2] cos + x[d] sin) for 8 columns, in fp32, rounded once to bf16
__device__ __forceinline__ void rotate8(uint4 &a, uint4 &b, const float *cs, const float *sn) {
    uint32_t *wa = reinterpret_cast<uint32_t *>(&a), *wb = reinterpret_cast<uint32_t *>(&b);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float x0 = __uint_as_float(wa[k] << 16), x1 = __uint_as_float(wa[k] & 0xffff0000u);
        const float y0 = __uint_as_float(wb[k] << 16), y1 = __uint_as_float(wb[k] & 0xffff0000u);
        const float2 c = *reinterpret_cast<const float2 *>(cs + 2 * k), s = *reinterpret_cast<const float2 *>(sn + 2 * k);
        const __nv_bfloat162 o1 = __floats2bfloat162_rn(x0 * c.x - y0 * s.x, x1 * c.y - y1 * s.y);
        const __nv_bfloat162 o2 = __floats2bfloat162_rn(y0 * c.x + x0 * s.x, y1 * c.y + x1 * s.y);
        wa[k] = *reinterpret_cast<const uint32_t *>(&o1);
        wb[k] = *reinterpret_cast<const uint32_t *>(&o2);
    }
}

struct AppendParams {
    int B, T, n_rows, Hq, Hkv, D, n_layers, layers_per_block, row_blocks;
    const __nv_bfloat16 *q, *k_new, *v_new;
    __nv_bfloat16 *q_out;
    __nv_bfloat16 *const *k_pools, *const *v_pools;
    PagedRef pages;
    const int32_t *seq_lens, *starts, *depth;   // starts: ragged rows, position = slot; or null: T tree nodes per sequence
    double log2_theta;
    int32_t *status;
};

// Rows of sequence b in this call.
__device__ __forceinline__ int rows_of(const AppendParams &p, int b, int *first) {
    *first = p.starts ? p.starts[b] : b * p.T;
    return p.starts ? p.starts[b + 1] - *first : p.T;
}

// 16 bytes of a row, whatever its address
template <bool VEC> __device__ __forceinline__ uint4 load8(const __nv_bfloat16 *p) {
    uint4 x;
    if constexpr (VEC) {
        x = *reinterpret_cast<const uint4 *>(p);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) reinterpret_cast<__nv_bfloat16 *>(&x)[k] = p[k];
    }
    return x;
}
template <bool VEC> __device__ __forceinline__ void store8(__nv_bfloat16 *p, const uint4 &x) {
    if constexpr (VEC) {
        *reinterpret_cast<uint4 *>(p) = x;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) p[k] = reinterpret_cast<const __nv_bfloat16 *>(&x)[k];
    }
}

// Bound by memory: per row and layer Hq rows are read and written, 2 Hkv read and 2 Hkv written.  A block takes APPEND_ROWS rows of
// some layers, works their angles out once (in double precision as far as the reduction to one turn goes: positions reach tens of
// thousands of radians; the sine and cosine of what is left in fp32), and moves 16-byte chunks.  The first of them are requested before
// anything else: lengths, pages and angles are worked out meanwhile.  The blocks behind the rows' own report one sequence per warp.
// Measured: trees of 4 x 64 nodes, 32 + 2 x 8 heads of 128, 32 layers: 35.7 us (201 MB, 5.6 TB/s; 31.1 at the memory's rate); five prompts of
// 3005 tokens, 28 + 2 x 4 heads, one layer: 13.5 us (8.6): 1503 blocks are 1.7 waves, and each begins with the chain length, page, angle.  Two rows a block: four
// take 34.9 and 15.4, one 36.5 and 17.4; two pairs in flight per thread 34.8 and 14.9, as fewer blocks fit.
// VEC: the rows begin at multiples of 16 bytes.
template <int D, bool VEC>
__global__ void __launch_bounds__(PAGED_THREADS)
kv_append_rope_paged_kernel(const AppendParams p) {
    constexpr int HALF = D / 2, PER_HEAD = D / 16, SLOTS = PAGED_THREADS / PER_HEAD;    // threads of a head; heads at a time
    __shared__ __align__(16) float cs[APPEND_ROWS][HALF], sn[APPEND_ROWS][HALF];
    __shared__ int64_t dst_of[APPEND_ROWS];    // of the row inside a pool; -1: no K/V row is written
    __shared__ int pos_of[APPEND_ROWS];        // -1: the row is left alone
    const int tid = threadIdx.x;
    previous_done();
    let_next_start();
    if ((int)blockIdx.x >= p.row_blocks) {
        const int b = ((int)blockIdx.x - p.row_blocks) * (PAGED_THREADS / 32) + tid / 32;
        if (!p.status || blockIdx.y || b >= p.B) return;
        int first;
        const int n = rows_of(p, b, &first), L = p.seq_lens[b];
        const int code = p.pages.check(b, L, n, tid % 32);
        if (tid % 32 == 0) p.status[b] = code;
        return;
    }
    const int r0 = (int)blockIdx.x * APPEND_ROWS;
    // A thread takes two chunks of 8 columns of a head, half a row apart; heads of a row in the order queries, keys, values, rows of a layer
    // behind one another.  (row, h) of its next pair, the row counted over the layers: a step is SLOTS heads.
    const int c = tid % PER_HEAD * 8, heads = p.Hq + 2 * p.Hkv;
    const int l0 = (int)blockIdx.y * p.layers_per_block, end = min(p.n_layers - l0, p.layers_per_block) * APPEND_ROWS;
    const int step_rows = SLOTS / heads, step_heads = SLOTS - step_rows * heads;
    int row = tid / PER_HEAD / heads, h = tid / PER_HEAD - row * heads;
    uint4 x[APPEND_DEEP][2];
    int at_row[APPEND_DEEP], at_h[APPEND_DEEP];
    auto request = [&] {
#pragma unroll
        for (int k = 0; k < APPEND_DEEP; ++k) {
            const int j = row % APPEND_ROWS;
            at_row[k] = row < end && r0 + j < p.n_rows ? row : -1;
            at_h[k] = h;
            if (at_row[k] >= 0) {
                const size_t i = (size_t)(l0 + row / APPEND_ROWS) * p.n_rows + r0 + j;
                const int g = h - p.Hq;
                const __nv_bfloat16 *src = g < 0 ? p.q + (i * p.Hq + h) * D : g < p.Hkv ? p.k_new + (i * p.Hkv + g) * D : p.v_new + (i * p.Hkv + g - p.Hkv) * D;
                x[k][0] = load8<VEC>(src + c);
                x[k][1] = load8<VEC>(src + HALF + c);
            }
            row += step_rows;
            h += step_heads;
            if (h >= heads) { h -= heads; ++row; }
        }
    };
    request();
    const double per_position = exp2(-2.0 * (tid % HALF) / D * p.log2_theta) * 0.15915494309189535;   // turns: / 2 pi
    int b0 = 0;
    if (p.starts) {        // the sequence of the block's first row: how many end at or before it
        for (int s = 0; s < p.B; s += PAGED_THREADS) b0 += __syncthreads_count(s + tid < p.B && p.starts[s + tid + 1] <= r0);
    }
    if (tid < APPEND_ROWS) {
        const int r = r0 + tid;
        int pos = -1;
        int64_t dst = -1;
        int b = p.starts ? b0 : r / p.T;
        if (p.starts)
            while (b < p.B && p.starts[b + 1] <= r) ++b;
        if (r < p.n_rows && b < p.B) {
            int first;
            const int n = rows_of(p, b, &first), L = p.seq_lens[b], i = r - first;
            if (i >= 0 && i < n && p.pages.fits(L, n)) {
                pos = L + (p.starts ? i : p.depth[i]);
                dst = p.pages.row(b, L + i);
            }
        }
        pos_of[tid] = pos;
        dst_of[tid] = dst;
    }
    __syncthreads();
    {
        const int j = tid / HALF, d = tid % HALF;
        if (j < APPEND_ROWS && pos_of[j] >= 0) {
            const double turns = (double)pos_of[j] * per_position;
            const float a = (float)((turns - rint(turns)) * 6.283185307179586);
            sincosf(a, &sn[j][d], &cs[j][d]);
        }
    }
    __syncthreads();
    for (;;) {
#pragma unroll
        for (int k = 0; k < APPEND_DEEP; ++k) {
            const int j = at_row[k] % APPEND_ROWS;
            if (at_row[k] < 0 || pos_of[j] < 0) continue;
            const int layer = l0 + at_row[k] / APPEND_ROWS, g = at_h[k] - p.Hq;
            __nv_bfloat16 *dst;
            if (g < 0) {
                dst = p.q_out + (((size_t)layer * p.n_rows + r0 + j) * p.Hq + at_h[k]) * D;
            } else {
                if (dst_of[j] < 0) continue;
                const bool is_v = g >= p.Hkv;
                dst = (is_v ? p.v_pools : p.k_pools)[layer] + dst_of[j] + (g - (is_v ? p.Hkv : 0)) * p.pages.stride_h;
            }
            if (g < p.Hkv) rotate8(x[k][0], x[k][1], &cs[j][c], &sn[j][c]);
            store8<VEC>(dst + c, x[k][0]);
            store8<VEC>(dst + HALF + c, x[k][1]);
        }
        if (row >= end) break;
        request();
    }
}

static int launch_append(AppendParams &p, cudaStream_t stream) {
    p.row_blocks = (p.n_rows + APPEND_ROWS - 1) / APPEND_ROWS;
    // enough blocks to fill the device a few times over, as many layers per block as that leaves
    long per = (long)p.row_blocks * p.n_layers / (12L * sm_count());
    per = per < 1 ? 1 : per > 64 ? 64 : per;
    if (per > p.n_layers) per = p.n_layers;
    p.layers_per_block = (int)per;
    const int report = p.status || !p.row_blocks ? (p.B + PAGED_THREADS / 32 - 1) / (PAGED_THREADS / 32) : 0;
    const bool vec = (((uintptr_t)p.q | (uintptr_t)p.q_out | (uintptr_t)p.k_new | (uintptr_t)p.v_new) & 15) == 0;
    auto kernel = p.D == 128 ? (vec ? kv_append_rope_paged_kernel<128, true> : kv_append_rope_paged_kernel<128, false>)
                             : (vec ? kv_append_rope_paged_kernel<64, true> : kv_append_rope_paged_kernel<64, false>);
    MTV_CUDA_CHECK(launch_dependent(kernel, dim3(p.row_blocks + report, (unsigned)((p.n_layers + per - 1) / per)),
                                    PAGED_THREADS, 0, stream, p));
    return MTV_OK;
}

static int append_args(AppendParams &p, int B, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q, mtv_bf16 *q_out, const mtv_bf16 *k_new,
                       const mtv_bf16 *v_new, mtv_bf16 *const *k_pools, mtv_bf16 *const *v_pools, const mtv_pool_layout *pool,
                       const int32_t *page_table, int max_pages, const int32_t *seq_lens, float rope_theta, int32_t *status, bool no_rows) {
    if (!k_pools || !v_pools || !seq_lens) return MTV_ERR_INVALID_ARG;
    if (!no_rows && (!q || !q_out || !k_new || !v_new)) return MTV_ERR_INVALID_ARG;
    if (B < 1 || Hq < 1 || Hkv < 1 || n_layers < 1 || !(rope_theta >= 0.f && rope_theta < INFINITY)) return MTV_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || n_layers > 65535 || Hq > PAGED_MAX_HEADS || Hkv > PAGED_MAX_HEADS) return MTV_ERR_UNSUPPORTED_SHAPE;
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D);
    if (rc != MTV_OK) return rc;
    p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.D = D; p.n_layers = n_layers;
    p.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    p.q_out = reinterpret_cast<__nv_bfloat16 *>(q_out);
    p.k_new = reinterpret_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = reinterpret_cast<const __nv_bfloat16 *>(v_new);
    p.k_pools = reinterpret_cast<__nv_bfloat16 *const *>(k_pools);
    p.v_pools = reinterpret_cast<__nv_bfloat16 *const *>(v_pools);
    p.seq_lens = seq_lens;
    p.log2_theta = log2(rope_theta == 0.f ? 10000.0 : (double)rope_theta);
    p.status = status;
    return MTV_OK;
}

// ---------------------------------------------------------------------------------------- compaction
struct CompactParams {
    int T, K, Hkv, D;
    __nv_bfloat16 *const *k_pools, *const *v_pools;
    PagedRef pages;
    const int32_t *seq_lens, *accept_len, *acc_nodes;
    int32_t *new_lens, *status;
    bool in_place;   // new_lens is seq_lens: lengths move in a launch of their own, behind all blocks that read them
};

// One warp: whether sequence b's accepted rows can be moved, and how many there are.
__device__ __forceinline__ int compact_check(const CompactParams &p, int b, int lane, int *L_out, int *n_out) {
    const int L = p.seq_lens[b], n = p.accept_len[b];
    *L_out = L;
    *n_out = n;
    if (!p.pages.fits(L, p.T)) return MTV_ERR_CAPACITY;
    if (n < 0 || n > p.K) return MTV_ERR_BOUNDS;
    bool ok = true;
    if (lane >= 1 && lane <= n) {
        const int node = p.acc_nodes[(size_t)b * (p.K + 1) + lane];
        ok = lane < p.T && node >= 0 && node < p.T && p.pages.row(b, L + node) >= 0 && p.pages.row(b, L + lane) >= 0;
    }
    return __all_sync(0xffffffffu, ok) ? MTV_OK : MTV_ERR_BOUNDS;
}

// grid = (n_layers, B).  Latency: length and nodes, pages, rows, stores follow one another; a block takes all heads of a layer so that
// the chain is gone through once.  A source row may be an earlier one's destination (acc_nodes = [0, 2, ..]: j = 1 reads slot 2, j = 2
// writes it), within a head only: the heads go through in groups whose rows the block's registers hold, all read before any is written.
__global__ void __launch_bounds__(PAGED_THREADS)
kv_compact_paged_kernel(const CompactParams p) {
    constexpr int PER = 4;
    __shared__ int64_t src_of[MTV_MAX_K + 1], dst_of[MTV_MAX_K + 1];
    __shared__ int n_rows;
    const int layer = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    let_next_start();
    previous_done();
    if (tid < 32) {
        int L, n;
        const int code = compact_check(p, b, tid, &L, &n);
        if (tid == 0) {
            n_rows = code == MTV_OK ? n : 0;
            if (layer == 0 && p.status) p.status[b] = code;
            if (layer == 0 && !p.in_place && code == MTV_OK) p.new_lens[b] = L + n + 1;
        }
        if (code == MTV_OK && tid >= 1 && tid <= n) {
            src_of[tid] = p.pages.row(b, L + p.acc_nodes[(size_t)b * (p.K + 1) + tid]);
            dst_of[tid] = p.pages.row(b, L + tid);
        }
    }
    __syncthreads();
    const int n = n_rows;
    if (n <= 0) return;
    __nv_bfloat16 *const pool[2] = {p.k_pools[layer], p.v_pools[layer]};
    const int vec = p.D / 8, per_head = 2 * n * vec;                     // 16-byte chunks; at most 256
    const int group = PER * PAGED_THREADS / per_head;                    // heads at a time, at least PER
    for (int g0 = 0; g0 < p.Hkv; g0 += group) {
        const int total = min(group, p.Hkv - g0) * per_head;
        uint4 x[PER];
        __nv_bfloat16 *to[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int e = tid + k * PAGED_THREADS;
            if (e < total) {
                const int c = e % vec, j = e / vec % n + 1, v = e / (vec * n) & 1, g = g0 + e / per_head;
                __nv_bfloat16 *base = (v ? pool[1] : pool[0]) + g * p.pages.stride_h + c * 8;
                x[k] = *reinterpret_cast<const uint4 *>(base + src_of[j]);
                to[k] = base + dst_of[j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (tid + k * PAGED_THREADS < total) *reinterpret_cast<uint4 *>(to[k]) = x[k];
    }
}

// In place: the lengths, one warp per sequence, once every block of the compaction has read them.
__global__ void __launch_bounds__(PAGED_THREADS)
paged_lens_advance_kernel(int B, const CompactParams p) {
    let_next_start();
    previous_done();
    const int b = (int)blockIdx.x * (PAGED_THREADS / 32) + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (b >= B) return;
    int L, n;
    if (compact_check(p, b, lane, &L, &n) == MTV_OK && lane == 0) p.new_lens[b] = L + n + 1;
}

}  // namespace mtv

extern "C" int tree_kv_append_rope_paged(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q_layers,
                                         mtv_bf16 *q_out_layers, const mtv_bf16 *k_new_layers, const mtv_bf16 *v_new_layers,
                                         mtv_bf16 *const *k_pools, mtv_bf16 *const *v_pools, const mtv_pool_layout *pool,
                                         const int32_t *page_table, int max_pages, const int32_t *seq_lens, float rope_theta,
                                         int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("tree_kv_append_rope_paged");
    if (!tree || !tree->on_device) return MTV_ERR_INVALID_ARG;
    AppendParams p = {};
    const int rc = append_args(p, B, Hq, Hkv, D, n_layers, q_layers, q_out_layers, k_new_layers, v_new_layers, k_pools, v_pools, pool, page_table,
                               max_pages, seq_lens, rope_theta, status, false);
    if (rc != MTV_OK) return rc;
    if (B > (1 << 30) / tree->T) return MTV_ERR_UNSUPPORTED_SHAPE;
    p.T = tree->T;
    p.n_rows = B * tree->T;
    p.depth = tree->d_depth;
    return launch_append(p, (cudaStream_t)stream);
}

extern "C" int kv_append_rope_paged(int B, int n_rows, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q_layers, mtv_bf16 *q_out_layers,
                                    const mtv_bf16 *k_new_layers, const mtv_bf16 *v_new_layers, mtv_bf16 *const *k_pools,
                                    mtv_bf16 *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                    const int32_t *seq_lens, const int32_t *row_starts, float rope_theta, int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_append_rope_paged");
    if (!row_starts || n_rows < 0) return MTV_ERR_INVALID_ARG;
    if (n_rows > 1 << 30) return MTV_ERR_UNSUPPORTED_SHAPE;
    AppendParams p = {};
    const int rc = append_args(p, B, Hq, Hkv, D, n_layers, q_layers, q_out_layers, k_new_layers, v_new_layers, k_pools, v_pools, pool, page_table,
                               max_pages, seq_lens, rope_theta, status, n_rows == 0);
    if (rc != MTV_OK) return rc;
    p.n_rows = n_rows;
    p.starts = row_starts;
    return launch_append(p, (cudaStream_t)stream);
}

extern "C" int kv_compact_accepted_paged(const mtv_tree_t *tree, int B, int Hkv, int D, int n_layers, mtv_bf16 *const *k_pools,
                                         mtv_bf16 *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                         const int32_t *seq_lens, int32_t *new_lens, const int32_t *accept_len, const int32_t *acc_nodes,
                                         int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_compact_accepted_paged");
    if (!tree || !k_pools || !v_pools || !seq_lens || !new_lens || !accept_len || !acc_nodes || B < 1 || Hkv < 1 || n_layers < 1)
        return MTV_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || B > 65535 || Hkv > PAGED_MAX_HEADS) return MTV_ERR_UNSUPPORTED_SHAPE;
    CompactParams p = {};
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D);
    if (rc != MTV_OK) return rc;
    p.T = tree->T; p.K = tree->K; p.Hkv = Hkv; p.D = D;
    p.k_pools = reinterpret_cast<__nv_bfloat16 *const *>(k_pools);
    p.v_pools = reinterpret_cast<__nv_bfloat16 *const *>(v_pools);
    p.seq_lens = seq_lens; p.accept_len = accept_len; p.acc_nodes = acc_nodes;
    p.new_lens = new_lens; p.status = status;
    p.in_place = new_lens == seq_lens;
    cudaStream_t st = (cudaStream_t)stream;
    MTV_CUDA_CHECK(launch_dependent(kv_compact_paged_kernel, dim3(n_layers, B), PAGED_THREADS, 0, st, p));
    if (p.in_place)
        MTV_CUDA_CHECK(launch_dependent(paged_lens_advance_kernel, dim3((B + PAGED_THREADS / 32 - 1) / (PAGED_THREADS / 32)), PAGED_THREADS, 0, st, B, p));
    return MTV_OK;
}
