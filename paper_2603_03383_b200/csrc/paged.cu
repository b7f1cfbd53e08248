// A K/V cache in pages: rows appended with the rotary embedding, and the accepted rows of a step moved to the front of the tree's
// slots (Section 3.2, "Tensorization of Tree Topology" and "Zero-Copy Retrieval"; the paper's own cache is contiguous).
// Slot s of sequence b is row s % page of page page_table[b][s / page]; page sizes are powers of two.
// The rows are bf16, or e4m3 codes with one scale per layer and head: then K rows are rotated in fp32 and rounded once, to the code, and rows
// can be read back as bf16.
#include "fp8.cuh"
#include "paged_common.cuh"
#include "sm100_ptx.cuh"

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

// The same over `scale`, rounded once to codes; cs null: nothing is rotated.
__device__ __forceinline__ void quantise8(const uint4 &a, const uint4 &b, const float *cs, const float *sn, float scale, uint2 &ca, uint2 &cb) {
    // (1 / scale is infinite in fp32 up to 2^-128, and 0 times it would be NaN: with a subnormal scale both are taken 2^64 larger)
    const bool tiny = scale < 0x1p-126f;
    const float factor = __frcp_rn(tiny ? scale * 0x1p64f : scale);
    const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
    uint32_t pa[4], pb[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float x0 = __uint_as_float(wa[k] << 16), x1 = __uint_as_float(wa[k] & 0xffff0000u);
        float y0 = __uint_as_float(wb[k] << 16), y1 = __uint_as_float(wb[k] & 0xffff0000u);
        if (cs) {
            const float2 c = *reinterpret_cast<const float2 *>(cs + 2 * k), s = *reinterpret_cast<const float2 *>(sn + 2 * k);
            const float u0 = fmaf(x0, c.x, -__fmul_rn(y0, s.x)), u1 = fmaf(x1, c.y, -__fmul_rn(y1, s.y));
            y0 = fmaf(x0, s.x, __fmul_rn(y0, c.x));
            y1 = fmaf(x1, s.y, __fmul_rn(y1, c.y));
            x0 = u0;
            x1 = u1;
        }
        if (tiny) { x0 *= 0x1p64f; x1 *= 0x1p64f; y0 *= 0x1p64f; y1 *= 0x1p64f; }
        pa[k] = e4m3x2(x0 * factor, x1 * factor);
        pb[k] = e4m3x2(y0 * factor, y1 * factor);
    }
    ca = make_uint2(pa[0] | pa[1] << 16, pa[2] | pa[3] << 16);
    cb = make_uint2(pb[0] | pb[1] << 16, pb[2] | pb[3] << 16);
}

struct AppendParams {
    int B, T, n_rows, Hq, Hkv, D, n_layers, layers_per_block, row_blocks;
    const __nv_bfloat16 *q, *k_new, *v_new;
    __nv_bfloat16 *q_out;
    void *const *k_pools, *const *v_pools;
    const float *k_scale, *v_scale;            // [n_layers][Hkv], or null: the pools are bf16
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
// Codes: the same rows in 34.4 us (185 MB, 5.4 TB/s; 28.2) and 13.9 (8.0; six blocks an SM, with five 15.4).
// VEC: the rows begin at multiples of 16 bytes.  FP8: the pools hold codes.
template <int D, bool VEC, bool FP8>
__global__ void __launch_bounds__(PAGED_THREADS, 6)
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
    float scale[APPEND_DEEP];
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
                if (FP8 && g >= 0) scale[k] = g < p.Hkv ? p.k_scale[(l0 + row / APPEND_ROWS) * p.Hkv + g] : p.v_scale[(l0 + row / APPEND_ROWS) * p.Hkv + g - p.Hkv];
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
                const int64_t at = dst_of[j] + (g - (is_v ? p.Hkv : 0)) * p.pages.stride_h;
                void *pool = (is_v ? p.v_pools : p.k_pools)[layer];
                if constexpr (FP8) {
                    uint2 a, b;
                    if (is_v) quantise8(x[k][0], x[k][1], nullptr, nullptr, scale[k], a, b);
                    else quantise8(x[k][0], x[k][1], &cs[j][c], &sn[j][c], scale[k], a, b);
                    *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(pool) + at + c) = a;
                    *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(pool) + at + HALF + c) = b;
                    continue;
                }
                dst = static_cast<__nv_bfloat16 *>(pool) + at;
            }
            if (g < p.Hkv) rotate8(x[k][0], x[k][1], &cs[j][c], &sn[j][c]);
            store8<VEC>(dst + c, x[k][0]);
            store8<VEC>(dst + HALF + c, x[k][1]);
        }
        if (row >= end) break;
        request();
    }
}

template <bool FP8>
static int launch_append(AppendParams &p, cudaStream_t stream) {
    p.row_blocks = (p.n_rows + APPEND_ROWS - 1) / APPEND_ROWS;
    // enough blocks to fill the device a few times over, as many layers per block as that leaves
    long per = (long)p.row_blocks * p.n_layers / (12L * sm_count());
    per = per < 1 ? 1 : per > 64 ? 64 : per;
    if (per > p.n_layers) per = p.n_layers;
    p.layers_per_block = (int)per;
    const int report = p.status || !p.row_blocks ? (p.B + PAGED_THREADS / 32 - 1) / (PAGED_THREADS / 32) : 0;
    const bool vec = (((uintptr_t)p.q | (uintptr_t)p.q_out | (uintptr_t)p.k_new | (uintptr_t)p.v_new) & 15) == 0;
    auto kernel = p.D == 128 ? (vec ? kv_append_rope_paged_kernel<128, true, FP8> : kv_append_rope_paged_kernel<128, false, FP8>)
                             : (vec ? kv_append_rope_paged_kernel<64, true, FP8> : kv_append_rope_paged_kernel<64, false, FP8>);
    MTV_CUDA_CHECK(launch_dependent(kernel, dim3(p.row_blocks + report, (unsigned)((p.n_layers + per - 1) / per)),
                                    PAGED_THREADS, 0, stream, p));
    return MTV_OK;
}

static int append_args(AppendParams &p, int B, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q, mtv_bf16 *q_out, const mtv_bf16 *k_new,
                       const mtv_bf16 *v_new, void *const *k_pools, void *const *v_pools, int code_bytes, const mtv_pool_layout *pool,
                       const int32_t *page_table, int max_pages, const int32_t *seq_lens, float rope_theta, int32_t *status, bool no_rows) {
    if (!k_pools || !v_pools || !seq_lens) return MTV_ERR_INVALID_ARG;
    if (!no_rows && (!q || !q_out || !k_new || !v_new)) return MTV_ERR_INVALID_ARG;
    if (B < 1 || Hq < 1 || Hkv < 1 || n_layers < 1 || !(rope_theta >= 0.f && rope_theta < INFINITY)) return MTV_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || n_layers > 65535 || Hq > PAGED_MAX_HEADS || Hkv > PAGED_MAX_HEADS) return MTV_ERR_UNSUPPORTED_SHAPE;
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D, 16 / code_bytes);
    if (rc != MTV_OK) return rc;
    p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.D = D; p.n_layers = n_layers;
    p.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    p.q_out = reinterpret_cast<__nv_bfloat16 *>(q_out);
    p.k_new = reinterpret_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = reinterpret_cast<const __nv_bfloat16 *>(v_new);
    p.k_pools = k_pools;
    p.v_pools = v_pools;
    p.seq_lens = seq_lens;
    p.log2_theta = log2(rope_theta == 0.f ? 10000.0 : (double)rope_theta);
    p.status = status;
    return MTV_OK;
}

// ---------------------------------------------------------------------------------------- compaction
struct CompactParams {
    int T, K, Hkv, D;
    char *const *k_pools, *const *v_pools;
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
// SIZE: bytes of an element.
template <int SIZE>
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
    char *const pool[2] = {p.k_pools[layer], p.v_pools[layer]};
    const int vec = p.D * SIZE / 16, per_head = 2 * n * vec;                     // 16-byte chunks; at most 256
    const int group = PER * PAGED_THREADS / per_head;                    // heads at a time, at least PER
    for (int g0 = 0; g0 < p.Hkv; g0 += group) {
        const int total = min(group, p.Hkv - g0) * per_head;
        uint4 x[PER];
        char *to[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int e = tid + k * PAGED_THREADS;
            if (e < total) {
                const int c = e % vec, j = e / vec % n + 1, v = e / (vec * n) & 1, g = g0 + e / per_head;
                char *base = (v ? pool[1] : pool[0]) + g * p.pages.stride_h * SIZE + c * 16;
                x[k] = *reinterpret_cast<const uint4 *>(base + src_of[j] * SIZE);
                to[k] = base + dst_of[j] * SIZE;
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

// ---------------------------------------------------------------------------------------- reading back
struct ReadParams {
    int B, n_rows, Hkv, n_layers, layers_per_block, row_blocks;
    const uint8_t *const *k_pools, *const *v_pools;
    const float *k_scale, *v_scale;            // [n_layers][Hkv]
    PagedRef pages;
    const int32_t *first, *starts;             // first: or null, zeros
    __nv_bfloat16 *k_out, *v_out;              // [n_layers][n_rows][Hkv][D]
    int32_t *status;
};

// Bound by memory: a byte read and two written per value.  A block takes READ_ROWS rows of some layers, finds their pages once, and its threads move
// 16 codes at a time, READ_DEEP requested together; the blocks behind the rows' own report one sequence per warp.  A thread's next chunk is counted on, not divided
// for (with divisions and 8 codes at a time 42 and 64 us).
// Measured: four prefixes of 17002 rows, 8 heads of 128, one layer: 22.2 us (104 MB, 4.7 TB/s; 16.0 at the memory's rate); 2050 rows of 28 layers, 4 heads: 33.4 (176 MB,
// 5.3 TB/s; 27.0).  1063 blocks are 1.4 waves of five an SM; 8 rows a block 21.3 and 33.2, 32 rows 23.0 and 32.0.
// WIDE: the outputs begin at multiples of 32 bytes.
constexpr int READ_ROWS = 16, READ_DEEP = 4;
template <int D, bool WIDE>
__global__ void __launch_bounds__(PAGED_THREADS)
kv_read_paged_kernel(const ReadParams p) {
    constexpr int PER_HEAD = D / 16;
    __shared__ int64_t src_of[READ_ROWS];      // of the row inside a pool; -1: the row is left alone
    const int tid = threadIdx.x;
    let_next_start();
    previous_done();
    if ((int)blockIdx.x >= p.row_blocks) {
        const int b = ((int)blockIdx.x - p.row_blocks) * (PAGED_THREADS / 32) + tid / 32;
        if (!p.status || blockIdx.y || b >= p.B) return;
        const int code = p.pages.check(b, p.first ? p.first[b] : 0, p.starts[b + 1] - p.starts[b], tid % 32);
        if (tid % 32 == 0) p.status[b] = code;
        return;
    }
    const int r0 = (int)blockIdx.x * READ_ROWS;
    int b = 0;                                 // the sequence of the block's first row: how many end at or before it
    for (int s = 0; s < p.B; s += PAGED_THREADS) b += __syncthreads_count(s + tid < p.B && p.starts[s + tid + 1] <= r0);
    if (tid < READ_ROWS) {
        const int r = r0 + tid;
        int64_t src = -1;
        while (b < p.B && p.starts[b + 1] <= r) ++b;
        if (r < p.n_rows && b < p.B) {
            const int start = p.starts[b], n = p.starts[b + 1] - start, L = p.first ? p.first[b] : 0, i = r - start;
            if (i >= 0 && p.pages.fits(L, n)) src = p.pages.row(b, L + i);
        }
        src_of[tid] = src;
    }
    __syncthreads();
    // Chunks of a row, rows of a pool, K and V, layers, one behind the other: (row, in_row) of a thread's next chunk, the row counted over pools and layers.
    const int l0 = (int)blockIdx.y * p.layers_per_block, end = min(p.n_layers - l0, p.layers_per_block) * 2 * READ_ROWS;
    const int per_row = p.Hkv * PER_HEAD, step_rows = PAGED_THREADS / per_row, step_chunks = PAGED_THREADS - step_rows * per_row;
    int row = tid / per_row, in_row = tid - row * per_row;
    while (row < end) {
        uint4 x[READ_DEEP];
        float scale[READ_DEEP];
        __nv_bfloat16 *dst[READ_DEEP];
#pragma unroll
        for (int k = 0; k < READ_DEEP; ++k) {
            const int l = l0 + row / (2 * READ_ROWS), v = row / READ_ROWS & 1, j = row % READ_ROWS, g = in_row / PER_HEAD, c = in_row % PER_HEAD * 16;
            dst[k] = nullptr;
            if (row < end && src_of[j] >= 0) {
                x[k] = *reinterpret_cast<const uint4 *>((v ? p.v_pools : p.k_pools)[l] + src_of[j] + g * p.pages.stride_h + c);
                scale[k] = (v ? p.v_scale : p.k_scale)[l * p.Hkv + g];
                dst[k] = (v ? p.v_out : p.k_out) + (((size_t)l * p.n_rows + r0 + j) * p.Hkv + g) * D + c;
            }
            row += step_rows;
            in_row += step_chunks;
            if (in_row >= per_row) { in_row -= per_row; ++row; }
        }
#pragma unroll
        for (int k = 0; k < READ_DEEP; ++k) {
            if (!dst[k]) continue;
            const uint32_t codes[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 f = f16x2_values(i % 2 ? f16x2_hi(codes[i / 2]) : f16x2_lo(codes[i / 2]));
                const __nv_bfloat162 o = __floats2bfloat162_rn(f.x * scale[k], f.y * scale[k]);
                w[i] = *reinterpret_cast<const uint32_t *>(&o);
            }
            if constexpr (WIDE) {
                ptx::st_global_32(dst[k], w);
            } else {
                *reinterpret_cast<uint4 *>(dst[k]) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(dst[k] + 8) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------- host
template <bool FP8>
static int append_tree(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q, mtv_bf16 *q_out, const mtv_bf16 *k_new,
                       const mtv_bf16 *v_new, void *const *k_pools, void *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table,
                       int max_pages, const int32_t *seq_lens, const float *k_scale, const float *v_scale, float rope_theta, int32_t *status, void *stream) {
    if (!tree || !tree->on_device || (FP8 && (!k_scale || !v_scale))) return MTV_ERR_INVALID_ARG;
    AppendParams p = {};
    const int rc = append_args(p, B, Hq, Hkv, D, n_layers, q, q_out, k_new, v_new, k_pools, v_pools, FP8 ? 1 : 2, pool, page_table, max_pages, seq_lens,
                               rope_theta, status, false);
    if (rc != MTV_OK) return rc;
    if (B > (1 << 30) / tree->T) return MTV_ERR_UNSUPPORTED_SHAPE;
    p.T = tree->T;
    p.n_rows = B * tree->T;
    p.depth = tree->d_depth;
    p.k_scale = k_scale; p.v_scale = v_scale;
    return launch_append<FP8>(p, (cudaStream_t)stream);
}

template <bool FP8>
static int append_rows(int B, int n_rows, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q, mtv_bf16 *q_out, const mtv_bf16 *k_new,
                       const mtv_bf16 *v_new, void *const *k_pools, void *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table,
                       int max_pages, const int32_t *seq_lens, const int32_t *row_starts, const float *k_scale, const float *v_scale, float rope_theta,
                       int32_t *status, void *stream) {
    if (!row_starts || n_rows < 0 || (FP8 && (!k_scale || !v_scale))) return MTV_ERR_INVALID_ARG;
    if (n_rows > 1 << 30) return MTV_ERR_UNSUPPORTED_SHAPE;
    AppendParams p = {};
    const int rc = append_args(p, B, Hq, Hkv, D, n_layers, q, q_out, k_new, v_new, k_pools, v_pools, FP8 ? 1 : 2, pool, page_table, max_pages, seq_lens,
                               rope_theta, status, n_rows == 0);
    if (rc != MTV_OK) return rc;
    p.n_rows = n_rows;
    p.starts = row_starts;
    p.k_scale = k_scale; p.v_scale = v_scale;
    return launch_append<FP8>(p, (cudaStream_t)stream);
}

template <int SIZE>
static int compact(const mtv_tree_t *tree, int B, int Hkv, int D, int n_layers, void *const *k_pools, void *const *v_pools, const mtv_pool_layout *pool,
                   const int32_t *page_table, int max_pages, const int32_t *seq_lens, int32_t *new_lens, const int32_t *accept_len,
                   const int32_t *acc_nodes, int32_t *status, void *stream) {
    if (!tree || !k_pools || !v_pools || !seq_lens || !new_lens || !accept_len || !acc_nodes || B < 1 || Hkv < 1 || n_layers < 1)
        return MTV_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || B > 65535 || Hkv > PAGED_MAX_HEADS) return MTV_ERR_UNSUPPORTED_SHAPE;
    CompactParams p = {};
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D, 16 / SIZE);
    if (rc != MTV_OK) return rc;
    p.T = tree->T; p.K = tree->K; p.Hkv = Hkv; p.D = D;
    p.k_pools = reinterpret_cast<char *const *>(k_pools);
    p.v_pools = reinterpret_cast<char *const *>(v_pools);
    p.seq_lens = seq_lens; p.accept_len = accept_len; p.acc_nodes = acc_nodes;
    p.new_lens = new_lens; p.status = status;
    p.in_place = new_lens == seq_lens;
    cudaStream_t st = (cudaStream_t)stream;
    MTV_CUDA_CHECK(launch_dependent(kv_compact_paged_kernel<SIZE>, dim3(n_layers, B), PAGED_THREADS, 0, st, p));
    if (p.in_place)
        MTV_CUDA_CHECK(launch_dependent(paged_lens_advance_kernel, dim3((B + PAGED_THREADS / 32 - 1) / (PAGED_THREADS / 32)), PAGED_THREADS, 0, st, B, p));
    return MTV_OK;
}
template <typename P> static void *const *untyped(P *const *pools) { return reinterpret_cast<void *const *>(pools); }

}  // namespace mtv

extern "C" int tree_kv_append_rope_paged(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q_layers,
                                         mtv_bf16 *q_out_layers, const mtv_bf16 *k_new_layers, const mtv_bf16 *v_new_layers,
                                         mtv_bf16 *const *k_pools, mtv_bf16 *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table,
                                         int max_pages, const int32_t *seq_lens, float rope_theta, int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("tree_kv_append_rope_paged");
    return append_tree<false>(tree, B, Hq, Hkv, D, n_layers, q_layers, q_out_layers, k_new_layers, v_new_layers, untyped(k_pools), untyped(v_pools), pool,
                         page_table, max_pages, seq_lens, nullptr, nullptr, rope_theta, status, stream);
}

extern "C" int kv_append_rope_paged(int B, int n_rows, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q_layers, mtv_bf16 *q_out_layers,
                                    const mtv_bf16 *k_new_layers, const mtv_bf16 *v_new_layers, mtv_bf16 *const *k_pools, mtv_bf16 *const *v_pools,
                                    const mtv_pool_layout *pool, const int32_t *page_table, int max_pages, const int32_t *seq_lens,
                                    const int32_t *row_starts, float rope_theta, int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_append_rope_paged");
    return append_rows<false>(B, n_rows, Hq, Hkv, D, n_layers, q_layers, q_out_layers, k_new_layers, v_new_layers, untyped(k_pools), untyped(v_pools), pool,
                         page_table, max_pages, seq_lens, row_starts, nullptr, nullptr, rope_theta, status, stream);
}

extern "C" int kv_compact_accepted_paged(const mtv_tree_t *tree, int B, int Hkv, int D, int n_layers, mtv_bf16 *const *k_pools,
                                         mtv_bf16 *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                         const int32_t *seq_lens, int32_t *new_lens, const int32_t *accept_len, const int32_t *acc_nodes,
                                         int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_compact_accepted_paged");
    return compact<2>(tree, B, Hkv, D, n_layers, untyped(k_pools), untyped(v_pools), pool, page_table, max_pages, seq_lens, new_lens, accept_len, acc_nodes,
                      status, stream);
}

extern "C" int tree_kv_append_rope_paged_fp8(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q_layers,
                                             mtv_bf16 *q_out_layers, const mtv_bf16 *k_new_layers, const mtv_bf16 *v_new_layers,
                                             uint8_t *const *k_pools, uint8_t *const *v_pools, const mtv_pool_layout *pool,
                                             const int32_t *page_table, int max_pages, const int32_t *seq_lens, const float *k_scale,
                                             const float *v_scale, float rope_theta, int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("tree_kv_append_rope_paged_fp8");
    return append_tree<true>(tree, B, Hq, Hkv, D, n_layers, q_layers, q_out_layers, k_new_layers, v_new_layers, untyped(k_pools), untyped(v_pools), pool,
                        page_table, max_pages, seq_lens, k_scale, v_scale, rope_theta, status, stream);
}

extern "C" int kv_append_rope_paged_fp8(int B, int n_rows, int Hq, int Hkv, int D, int n_layers, const mtv_bf16 *q_layers, mtv_bf16 *q_out_layers,
                                        const mtv_bf16 *k_new_layers, const mtv_bf16 *v_new_layers, uint8_t *const *k_pools, uint8_t *const *v_pools,
                                        const mtv_pool_layout *pool, const int32_t *page_table, int max_pages, const int32_t *seq_lens,
                                        const int32_t *row_starts, const float *k_scale, const float *v_scale, float rope_theta, int32_t *status,
                                        void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_append_rope_paged_fp8");
    return append_rows<true>(B, n_rows, Hq, Hkv, D, n_layers, q_layers, q_out_layers, k_new_layers, v_new_layers, untyped(k_pools), untyped(v_pools), pool,
                        page_table, max_pages, seq_lens, row_starts, k_scale, v_scale, rope_theta, status, stream);
}

extern "C" int kv_compact_accepted_paged_fp8(const mtv_tree_t *tree, int B, int Hkv, int D, int n_layers, uint8_t *const *k_pools,
                                             uint8_t *const *v_pools, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                             const int32_t *seq_lens, int32_t *new_lens, const int32_t *accept_len, const int32_t *acc_nodes,
                                             int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_compact_accepted_paged_fp8");
    return compact<1>(tree, B, Hkv, D, n_layers, untyped(k_pools), untyped(v_pools), pool, page_table, max_pages, seq_lens, new_lens, accept_len, acc_nodes,
                      status, stream);
}

extern "C" int kv_read_paged_fp8(int B, int n_rows, int Hkv, int D, int n_layers, const uint8_t *const *k_pools, const uint8_t *const *v_pools,
                                 const mtv_pool_layout *pool, const int32_t *page_table, int max_pages, const int32_t *first,
                                 const int32_t *row_starts, const float *k_scale, const float *v_scale, mtv_bf16 *k_out_layers,
                                 mtv_bf16 *v_out_layers, int32_t *status, void *stream) {
    using namespace mtv;
    MTV_RANGE("kv_read_paged_fp8");
    if (!k_pools || !v_pools || !row_starts || !k_scale || !v_scale || B < 1 || n_rows < 0 || Hkv < 1 || n_layers < 1) return MTV_ERR_INVALID_ARG;
    if (n_rows && (!k_out_layers || !v_out_layers || (((uintptr_t)k_out_layers | (uintptr_t)v_out_layers) & 15))) return MTV_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || n_layers > 65535 || Hkv > PAGED_MAX_HEADS || n_rows > 1 << 30) return MTV_ERR_UNSUPPORTED_SHAPE;
    ReadParams p = {};
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D, 16);
    if (rc != MTV_OK) return rc;
    p.B = B; p.n_rows = n_rows; p.Hkv = Hkv; p.n_layers = n_layers;
    p.k_pools = k_pools; p.v_pools = v_pools; p.k_scale = k_scale; p.v_scale = v_scale;
    p.first = first; p.starts = row_starts;
    p.k_out = reinterpret_cast<__nv_bfloat16 *>(k_out_layers);
    p.v_out = reinterpret_cast<__nv_bfloat16 *>(v_out_layers);
    p.status = status;
    p.row_blocks = (n_rows + READ_ROWS - 1) / READ_ROWS;
    // as in the appending: enough blocks to fill the device a few times over, as many layers per block as that leaves
    long per = (long)p.row_blocks * n_layers / (12L * sm_count());
    per = per < 1 ? 1 : per > n_layers ? n_layers : per;
    p.layers_per_block = (int)per;
    const int report = status || !p.row_blocks ? (B + PAGED_THREADS / 32 - 1) / (PAGED_THREADS / 32) : 0;
    const bool wide = (((uintptr_t)k_out_layers | (uintptr_t)v_out_layers) & 31) == 0;
    auto kernel = D == 128 ? (wide ? kv_read_paged_kernel<128, true> : kv_read_paged_kernel<128, false>)
                           : (wide ? kv_read_paged_kernel<64, true> : kv_read_paged_kernel<64, false>);
    MTV_CUDA_CHECK(launch_dependent(kernel, dim3(p.row_blocks + report, (unsigned)((n_layers + per - 1) / per)), PAGED_THREADS, 0, (cudaStream_t)stream, p));
    return MTV_OK;
}
