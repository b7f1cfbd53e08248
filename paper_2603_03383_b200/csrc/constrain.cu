// Penalties for repeated tokens, biases and grammar masks on the base model's logits at the tree's nodes, in front of the acceptance
// (Section 3.2; the paper accepts on the plain argmax).  For row (b, i) and token v, with c = occurrences of v in sequence b's generated
// text and on the path from the root to node i, seen = c > 0 or v in the prompt:
//   x = logit;  seen: x = x > 0 ? x / repetition : x * repetition;  c > 0: x = x - frequency * c, x = x - presence;
//   x = x + bias;  not allowed by the row's mask: -inf
// every operation rounded to fp32 by itself (no contraction), so that equal inputs give equal keys whatever the order they are met in.
//
// The logits are read once (and written once in the form that writes).  What a token was counted, and whether it is allowed, are bits
// (1/16 of the logits' bytes per sequence, 1/16 per mask); only the few tokens that are counted, biased or on the path go through the
// formula.  A block takes a slab of 2048 tokens of the vocabulary for some of a sequence's nodes.  It first lists the slab's counted and biased
// tokens; then a warp per row makes a dense pass over the allowed tokens that are in no list (16-byte loads, masks laid over whole
// vectors, packed maxima or copies) and a sparse one over the list.  Rows may begin at any element: vectors are cut at the addresses' 16-byte
// boundaries, and the two that a slab shares with its neighbours are taken element by element.
// A slab's entries of the bias list are sorted by token and place, so that a token's entries are summed in the list's order in one go: up to 32 by a warp
// beside the listing, more by the block (4096 entries of one token, 4 x 64 rows of 40000: 0.18 ms; of 2000 tokens in one slab: 0.07).
// Measured: argmax of 8 x 64 rows of 131072 bf16 logits, 64 masks, 4000 tokens of text a sequence, with the acceptance 49 us (134 MB: 21 us at the
// memory's rate); written, 5 x 64 rows of 50003: 25 us (9.9).  Bound by instructions and their latency: about 950 a warp for a row's slab at
// 0.63 an instruction a cycle and scheduler, a third of them the list's (a division each, on lanes that the list only partly fills; it is gone through for
// every row, though few listed tokens can be the maximum); written, 1000 blocks on 740 places are 1.35 waves, and the kernel spills (40 bytes a thread).  Blocks of 8 rows cost
// 8 us more (every block lists anew, three loads deep), of 32 rows 8 us (the last wave is short); five blocks per SM rather than the four that
// the compiler's choice of registers leaves: 66 -> 47; rows staged in shared memory by asynchronous copies: 75, as two blocks fit then.
#include <cuda_bf16.h>

#include "common.cuh"

namespace mtv {

constexpr int CN_THREADS = 256, CN_WARPS = CN_THREADS / 32;
constexpr int CN_SLAB = 2048, CN_WORDS = CN_SLAB / 32, CN_PER = CN_WORDS / 32;
constexpr int CN_ROWS = 32;          // most rows of a block
constexpr int CN_PATH = MTV_MAX_K + 1;
constexpr int CN_BLOCKS = 8;
constexpr int CN_MAX_BIAS = 4096;    // a power of two
constexpr uint32_t CN_PROMPT = 0x80000000u;

struct ConstrainParams {
    const void *logits;
    void *out;                       // or null: keys
    int64_t ld_in, ld_out;           // elements from row to row
    unsigned long long *keys;        // [B*T], zero before the launch where there is more than one slab
    const uint32_t *counts, *seen;   // [B][V], [B][words], or null
    const float *repetition, *presence, *frequency;   // [B] or null
    const int32_t *bias_ids;         // [B][n_bias]
    const float *bias;
    const uint32_t *mask;            // [n_masks][words]
    const int32_t *mask_of;          // [B*T] or null
    const int32_t *tree_tok;         // [B][T] or null
    const uint64_t *anc;             // [T][2]
    int32_t *dev_error;
    int B, T, V, words, n_bias, n_masks, rows_per_block, groups;
    bool one_slab;                   // a row's key is written once
};

// bits 0-3 -> the top bits of bytes 0-3 (the products of a bit with the factor's four fall on places of their own; other bits hold anything)
__device__ __forceinline__ uint32_t signs_of(uint32_t bits) { return (bits & 0xfu) * 0x10204080u; }
// every byte of the result: the sign of the byte of x that its digit of the selector names (8 + byte), eight times.  (__byte_perm leaves the digits'
// top bit out.)
__device__ __forceinline__ uint32_t spread(uint32_t x, uint32_t selector) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %1, %2;" : "=r"(r) : "r"(x), "r"(selector));
    return r;
}
// where a bit is 0: -inf
__device__ __forceinline__ uint32_t keep(uint32_t x, uint32_t mask, uint32_t hidden) { return (x & mask) | (hidden & ~mask); }

template <typename E> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static constexpr int VEC = 8;
    static __device__ __forceinline__ float get(const __nv_bfloat16 *p) { return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(p) << 16); }
    static __device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
    static __device__ __forceinline__ uint4 masked(const uint4 &u, uint32_t bits) {
        const uint32_t a = signs_of(bits), b = signs_of(bits >> 4), hidden = 0xff80ff80u;
        return make_uint4(keep(u.x, spread(a, 0x9988u), hidden), keep(u.y, spread(a, 0xbbaau), hidden),
                          keep(u.z, spread(b, 0x9988u), hidden), keep(u.w, spread(b, 0xbbaau), hidden));
    }
    // running maximum of vectors; NaN counts for nothing
    using Top = __nv_bfloat162;
    static __device__ __forceinline__ Top none() { return __float2bfloat162_rn(-INFINITY); }
    static __device__ __forceinline__ Top more(Top m, const uint4 &u) {
        const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&u);
        return __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
    }
    static __device__ __forceinline__ float value(Top m) { return fmaxf(__low2float(m), __high2float(m)); }
};
template <> struct Elem<float> {
    static constexpr int VEC = 4;
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    static __device__ __forceinline__ uint4 masked(const uint4 &u, uint32_t bits) {
        const uint32_t a = signs_of(bits), hidden = 0xff800000u;
        return make_uint4(keep(u.x, spread(a, 0x8888u), hidden), keep(u.y, spread(a, 0x9999u), hidden),
                          keep(u.z, spread(a, 0xaaaau), hidden), keep(u.w, spread(a, 0xbbbbu), hidden));
    }
    using Top = float;
    static __device__ __forceinline__ Top none() { return -INFINITY; }
    static __device__ __forceinline__ Top more(Top m, const uint4 &u) {
        return fmaxf(m, fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))));
    }
    static __device__ __forceinline__ float value(Top m) { return m; }
};

// Order-preserving image of a value that is no NaN; both zeros are one.
__device__ __forceinline__ uint32_t value_image(float v) {
    const uint32_t u = __float_as_uint(v);
    return v == 0.f ? 0x80000000u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Penalties {
    float r, p, f;
    __device__ __forceinline__ float apply(float x, int c, bool seen, float bias) const {
        if (seen) x = x > 0.f ? __fdiv_rn(x, r) : __fmul_rn(x, r);
        if (c > 0) x = __fsub_rn(__fsub_rn(x, __fmul_rn(f, (float)c)), p);
        return __fadd_rn(x, bias);
    }
};

// n <= 32 words ascending, by one warp; n of them, with room for the next power of two, by the block: a bitonic sort.
__device__ __forceinline__ void sort_warp(uint32_t *w, int n, int lane) {
    uint32_t x = lane < n ? w[lane] : 0xffffffffu;
#pragma unroll
    for (int k = 2; k <= 32; k *= 2)
#pragma unroll
        for (int j = k / 2; j > 0; j /= 2) {
            const uint32_t y = __shfl_xor_sync(0xffffffffu, x, j);
            x = ((lane & j) == 0) == ((lane & k) == 0) ? min(x, y) : max(x, y);
        }
    if (lane < n) w[lane] = x;
}
__device__ __noinline__ void sort_block(uint32_t *w, int n, int tid) {
    int size = 64;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += CN_THREADS) w[i] = 0xffffffffu;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int i = tid; i < size / 2; i += CN_THREADS) {
                const int a = 2 * i - (i & (j - 1));
                const uint32_t x = w[a], y = w[a + j];
                if ((x > y) == ((a & k) == 0)) {
                    w[a] = y;
                    w[a + j] = x;
                }
            }
            __syncthreads();
        }
}

template <typename E, bool WRITE>
__global__ void __launch_bounds__(CN_THREADS, 5)
constrain_kernel(const ConstrainParams p) {
    using El = Elem<E>;
    constexpr int VEC = El::VEC;
    __shared__ uint32_t listed[CN_WORDS], biased[CN_WORDS], known[CN_WORDS], allowed_of[CN_WARPS][CN_WORDS], dense_of[CN_WARPS][CN_WORDS + 1];
    __shared__ uint32_t list_count[CN_SLAB];
    __shared__ float list_bias[CN_SLAB];
    __shared__ uint16_t list_at[CN_SLAB];
    __shared__ uint32_t match[CN_MAX_BIAS];      // the slab's entries of the bias list: token << 16 | place in the list; sorted before they are used
    __shared__ int n_listed, n_match;
    __shared__ int32_t path[CN_ROWS][CN_PATH];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    // slabs are the slowest: vocabularies give their frequent tokens low numbers, and the slabs with long lists start first
    const int group = (int)blockIdx.x % p.groups, b = (int)blockIdx.x / p.groups % p.B, base = (int)blockIdx.x / p.groups / p.B * CN_SLAB;
    const int row0 = group * p.rows_per_block, n_rows = min(p.rows_per_block, p.T - row0), n_tok = min(CN_SLAB, p.V - base);
    let_next_start();
    previous_done();
    // ---- the slab's counted and biased tokens, and the path of every row.  Loads that wait for nothing are issued first: a block's start is
    // a chain of three or four of them, one behind the other.
    int mask_at = -1;                           // lane i: the mask of this warp's i-th row
    if (p.mask_of && warp + lane * CN_WARPS < n_rows) mask_at = p.mask_of[(size_t)b * p.T + row0 + warp + lane * CN_WARPS];
    uint32_t seen = 0u;
    if (tid < CN_WORDS && p.seen && base / 32 + tid < p.words) seen = p.seen[(size_t)b * p.words + base / 32 + tid];
    int biased_at = -1;
    auto bias_at = [&](int k) { return (int)((uint32_t)p.bias_ids[(size_t)b * p.n_bias + k] - (uint32_t)base); };   // any number may stand there
    if (tid < p.n_bias) biased_at = bias_at(tid);
    const Penalties pen = {p.repetition ? p.repetition[b] : 1.f, p.presence ? p.presence[b] : 0.f, p.frequency ? p.frequency[b] : 0.f};
    for (int e = tid; e < n_rows * CN_PATH; e += CN_THREADS) {
        const int r = e / CN_PATH;
        int k = e - r * CN_PATH, node = -1;
        if (p.tree_tok) {                                   // the k-th node of the path
            uint64_t lo = p.anc[(row0 + r) * 2], hi = p.anc[(row0 + r) * 2 + 1];
            for (; k > 0 && (lo | hi); --k) {
                if (lo) lo &= lo - 1;
                else hi &= hi - 1;
            }
            node = lo ? __ffsll((long long)lo) - 1 : hi ? 63 + __ffsll((long long)hi) : -1;
        }
        path[r][e - r * CN_PATH] = node >= 0 ? p.tree_tok[(size_t)b * p.T + node] : -1;
    }
    if (mask_at >= p.n_masks) {
        if (p.mask_of) atomicExch(p.dev_error, MTV_ERR_BOUNDS);
        mask_at = -1;
    }
    // the words of the mask of this warp's i-th row: bit t % 32 of word t / 32 for the slab's token t, word k * 32 + lane here
    auto mask_words = [&](int i, uint32_t (&w)[CN_PER]) {
        const int m = __shfl_sync(0xffffffffu, mask_at, i);
#pragma unroll
        for (int k = 0; k < CN_PER; ++k)
            w[k] = m >= 0 && (k * 32 + lane) * 32 < n_tok ? p.mask[(size_t)m * p.words + base / 32 + k * 32 + lane] : 0xffffffffu;
    };
    uint32_t next[CN_PER];
    mask_words(0, next);
    if (tid < CN_WORDS) {
        listed[tid] = known[tid] = seen;
        biased[tid] = 0u;
    }
    if (tid == 0) n_match = 0;
    __syncthreads();
    for (int k = tid; k < p.n_bias; k += CN_THREADS) {
        if (k != tid) biased_at = bias_at(k);
        if (biased_at >= 0 && biased_at < n_tok) {
            atomicOr(&listed[biased_at / 32], 1u << (biased_at % 32));
            atomicOr(&biased[biased_at / 32], 1u << (biased_at % 32));
            match[atomicAdd(&n_match, 1)] = (uint32_t)biased_at << 16 | (uint32_t)k;
        }
    }
    if (p.n_bias) __syncthreads();
    if (warp == 0) {
        int start = 0;
#pragma unroll
        for (int i = 0; i < CN_PER; ++i) {
            uint32_t w = listed[i * 32 + lane];
            const int mine = __popc(w);
            int before = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int x = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += x;
            }
            const int all = __shfl_sync(0xffffffffu, before, 31);
            before += start - mine;
            for (; w; w &= w - 1) list_at[before++] = (uint16_t)((i * 32 + lane) * 32 + __ffs((int)w) - 1);
            start += all;
        }
        if (lane == 0) n_listed = start;
    }
    if (warp == 1 && n_match > 1 && n_match <= 32) sort_warp(match, n_match, lane);
    __syncthreads();
    if (n_match > 32) sort_block(match, n_match, tid);
    for (int e = tid; e < n_listed; e += CN_THREADS) {
        const int at = list_at[e], v = base + at;
        float sum = 0.f;
        if (biased[at / 32] >> (at % 32) & 1) {             // its entries lie side by side, in the list's order
            int lo = 0;
            for (int hi = n_match; lo < hi;) {
                const int mid = (lo + hi) / 2;
                if (match[mid] < (uint32_t)at << 16) lo = mid + 1;
                else hi = mid;
            }
            bool more = true;
            for (; more; lo += 8) {                         // (eight at a time, so that their loads do not wait for one another)
                float x[8];
                bool is[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t m = lo + k < n_match ? match[lo + k] : 0xffffffffu;
                    is[k] = m >> 16 == (uint32_t)at;
                    x[k] = is[k] ? p.bias[(size_t)b * p.n_bias + (m & 0xffffu)] : 0.f;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (is[k]) sum = __fadd_rn(sum, x[k]);
                more = is[7];
            }
        }
        list_bias[e] = sum;
        // (a count whose bit in `seen` is 0 may be an earlier sequence's)
        list_count[e] = known[at / 32] >> (at % 32) & 1u && v < p.V ? p.counts[(size_t)b * p.V + v] : 0u;
    }
    __syncthreads();
    // ---- a warp per row; its mask is requested while the row before is worked on
    uint32_t *words = dense_of[warp];
    for (int r = warp, turn = 0; r < n_rows; r += CN_WARPS, ++turn) {
        uint32_t allowed[CN_PER], any = 0u;
#pragma unroll
        for (int i = 0; i < CN_PER; ++i) {
            const int left = n_tok - (i * 32 + lane) * 32;
            any |= allowed[i] = left >= 32 ? next[i] : left > 0 ? next[i] & ((1u << left) - 1u) : 0u;
        }
        mask_words(turn + 1, next);
        // (nothing allowed: the argmax need not look at the logits)
        const size_t row = (size_t)b * p.T + row0 + r;
        if (!WRITE && !__any_sync(0xffffffffu, any != 0u)) {
            if (p.one_slab && lane == 0) p.keys[row] = 0ull;
            continue;
        }
        const E *in = static_cast<const E *>(p.logits) + (int64_t)row * p.ld_in + base;
        E *out = WRITE ? static_cast<E *>(p.out) + (int64_t)row * p.ld_out + base : nullptr;
        int here = lane < CN_PATH ? path[r][lane] : -1;       // this lane's token of the path, where it lies in this slab
        here = here >= base && here - base < n_tok ? here - base : -1;
        const uint32_t on_path = __ballot_sync(0xffffffffu, here >= 0);
        // The vectors of the row's addresses: vector j holds tokens [j * VEC - off, (j + 1) * VEC - off); bit j * VEC + e of the words belongs to its
        // element e.
        const int off = (int)((uintptr_t)in / sizeof(E) % VEC);
        uint32_t dense[CN_PER];
#pragma unroll
        for (int i = 0; i < CN_PER; ++i) {
            allowed_of[warp][i * 32 + lane] = allowed[i];
            dense[i] = WRITE ? allowed[i] : allowed[i] & ~listed[i * 32 + lane];
        }
        if (!WRITE)
            for (uint32_t some = on_path; some; some &= some - 1) {
                const int at = __shfl_sync(0xffffffffu, here, __ffs((int)some) - 1);
#pragma unroll
                for (int i = 0; i < CN_PER; ++i)
                    if (at / 32 == i * 32 + lane) dense[i] &= ~(1u << (at % 32));
            }
        if (off == 0) {
#pragma unroll
            for (int i = 0; i < CN_PER; ++i) words[i * 32 + lane] = dense[i];
        } else {
            uint32_t carry = 0u;
#pragma unroll
            for (int i = 0; i < CN_PER; ++i) {
                uint32_t below = __shfl_up_sync(0xffffffffu, dense[i], 1);
                if (lane == 0) below = carry;
                words[i * 32 + lane] = __funnelshift_l(below, dense[i], off);
                carry = __shfl_sync(0xffffffffu, dense[i], 31);
            }
            if (lane == 0) words[CN_WORDS] = carry >> (32 - off);
        }
        __syncwarp();
        auto bits_of = [&](int j) {
            const uint32_t x = reinterpret_cast<const uint8_t *>(words)[j * VEC / 8];
            return VEC == 8 ? x : x >> (j % 2 * 4) & 0xfu;
        };
        auto is_dense = [&](int t) { return words[(t + off) >> 5] >> ((t + off) & 31) & 1u; };
        auto is_allowed = [&](int t) { return allowed_of[warp][t >> 5] >> (t & 31) & 1u; };
        // the largest of the tokens taken one by one and the first that has it; the largest of the vectors and the first DEEP that have it
        float best = -INFINITY, best_v = -INFINITY;
        int at = -1, at_v = -1;
        auto one = [&](int t, float x) {
            if (x > best || (x == best && t < at)) { best = x; at = t; }
        };
        // ---- whole vectors
        const int j_lo = off > 0, j_hi = (off + n_tok) / VEC;
        const bool out_vec = WRITE && (int)((uintptr_t)out / sizeof(E) % VEC) == off;
        constexpr int DEEP = 4;
        for (int j0 = j_lo + lane; j0 < j_hi; j0 += 32 * DEEP) {
            uint4 x[DEEP];
            uint32_t bits[DEEP];
#pragma unroll
            for (int k = 0; k < DEEP; ++k) {
                const int j = j0 + 32 * k;
                bits[k] = j < j_hi ? bits_of(j) : 0u;
                x[k] = make_uint4(0u, 0u, 0u, 0u);
                if (bits[k]) x[k] = *reinterpret_cast<const uint4 *>(in + (j * VEC - off));
            }
            typename El::Top top = El::none();
#pragma unroll
            for (int k = 0; k < DEEP; ++k) {
                const int j = j0 + 32 * k, t0 = j * VEC - off;
                const uint4 y = El::masked(x[k], bits[k]);
                if (!WRITE) {
                    top = El::more(top, y);
                } else if (j < j_hi) {
                    if (out_vec) {
                        *reinterpret_cast<uint4 *>(out + t0) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) out[t0 + e] = reinterpret_cast<const E *>(&y)[e];
                    }
                }
            }
            const float v = El::value(top);
            if (!WRITE && v > best_v) { best_v = v; at_v = j0; }     // strictly: the first ones stay
        }
        // the first token that has the vectors' largest value: the elements of the DEEP vectors of each lane that has it, one to a lane
        uint32_t top_v = value_image(best_v), first_v = 0xffffffffu;
        if (!WRITE) {
            const uint32_t mine = top_v;
            top_v = __reduce_max_sync(0xffffffffu, mine);
            if (top_v != value_image(-INFINITY))
                for (uint32_t some = __ballot_sync(0xffffffffu, mine == top_v); some; some &= some - 1) {
                    const int j0 = __shfl_sync(0xffffffffu, at_v, __ffs((int)some) - 1);
#pragma unroll
                    for (int i = lane; i < DEEP * VEC; i += 32) {
                        const int j = j0 + i / VEC * 32, t = j * VEC - off + i % VEC;
                        if (j < j_hi && is_dense(t) && value_image(El::get(in + t)) == top_v) first_v = min(first_v, (uint32_t)t);
                    }
                }
        }
        // ---- the tokens of the two vectors that the row shares with others
        {
            const int head = min(n_tok, j_lo * VEC - off), tail = max(head, j_hi * VEC - off);
            const int t = lane < VEC ? lane : tail + lane - VEC;
            if (lane < VEC ? t < head : t < n_tok && lane < 2 * VEC) {
                const bool is = is_dense(t);
                if (!WRITE) {
                    if (is) one(t, El::get(in + t));
                } else if (is) {
                    out[t] = in[t];
                } else {
                    El::put(out + t, -INFINITY);
                }
            }
        }
        // ---- listed tokens, then those of the path that are in no list
        if (WRITE) __syncwarp();
        auto special = [&](int t, uint32_t counted, float bias) {
            int c = (int)(counted & ~CN_PROMPT);
            if (on_path)
                for (int k = 0; k < CN_PATH; ++k) c += path[r][k] == base + t;
            return pen.apply(El::get(in + t), c, c > 0 || counted & CN_PROMPT, bias);
        };
        for (int e = lane; e < n_listed; e += 32) {
            const int t = list_at[e];
            if (!is_allowed(t)) continue;
            const float x = special(t, list_count[e], list_bias[e]);
            if (WRITE) El::put(out + t, x);
            else one(t, x);
        }
        if (here >= 0 && is_allowed(here) && !(listed[here / 32] >> (here % 32) & 1)) {
            bool first = true;          // the same token twice on a path: once
            for (int k = 0; k < lane; ++k) first = first && path[r][k] != base + here;
            if (first) {
                const float x = special(here, 0u, 0.f);
                if (WRITE) El::put(out + here, x);
                else one(here, x);
            }
        }
        if (WRITE) {
            __syncwarp();
            continue;
        }
        // ---- the row's largest value in this slab, and the first token that has it
        const uint32_t image = value_image(best);         // (of -inf where this lane has nothing)
        const uint32_t top = max(top_v, __reduce_max_sync(0xffffffffu, image));
        uint32_t first = top_v == top ? first_v : 0xffffffffu;
        if (top != value_image(-INFINITY)) {
            if (image == top) first = min(first, (uint32_t)at);
        } else {
            // nothing but -inf and NaN: the first allowed -inf
            first = 0xffffffffu;
            for (int t = lane; t < n_tok && first == 0xffffffffu; t += 32)
                if (is_allowed(t)) {
                    float x = El::get(in + t), bias = 0.f;
                    uint32_t counted = 0u;
                    const bool in_list = listed[t / 32] >> (t % 32) & 1;
                    bool walked = false;
                    for (int k = 0; k < CN_PATH; ++k) walked = walked || path[r][k] == base + t;
                    for (int e = 0; in_list && e < n_listed; ++e)
                        if (list_at[e] == t) { bias = list_bias[e]; counted = list_count[e]; }
                    if (in_list || walked) x = special(t, counted, bias);
                    if (x == -INFINITY) first = (uint32_t)t;
                }
        }
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0 && first != 0xffffffffu) {
            const unsigned long long key = (unsigned long long)top << 32 | (0xffffffffu - ((uint32_t)base + first));
            if (p.one_slab) p.keys[row] = key;
            else atomicMax(p.keys + row, key);
        }
        if (p.one_slab && lane == 0 && first == 0xffffffffu) p.keys[row] = 0ull;
        __syncwarp();       // before the next row's bits
    }
}

// The keys' zeros: a kernel, so that the one behind it is launched while it runs.
__global__ void __launch_bounds__(256)
clear_keys_kernel(int n, unsigned long long *keys) {
    let_next_start();
    previous_done();
    const int i = (int)blockIdx.x * 256 + threadIdx.x;
    if (i < n) keys[i] = 0ull;
}

// ---------------------------------------------------------------------------------------- counts
// grid = (chunks of tokens, B).  Integer atomics: the order does not matter.
__global__ void __launch_bounds__(256)
token_counts_add_kernel(int V, int words, int n, int prompt, const int32_t *__restrict__ tokens, const int32_t *__restrict__ lens,
                        uint32_t *counts, uint32_t *seen) {
    let_next_start();
    previous_done();
    const int b = blockIdx.y, i = (int)blockIdx.x * 256 + threadIdx.x;
    const int end = lens ? min(lens[b], n) : n;
    if (i >= end) return;
    const int v = tokens[(size_t)b * n + i];
    if (v < 0 || v >= V) return;
    if (prompt) atomicOr(counts + (size_t)b * V + v, CN_PROMPT);
    else atomicAdd(counts + (size_t)b * V + v, 1u);
    atomicOr(seen + (size_t)b * words + v / 32, 1u << (v % 32));
}

static int constrain(const mtv_tree_t *tree, int B, int V, int dtype, const void *logits, int64_t ld_in, void *out, int64_t ld_out,
                     unsigned long long *keys, const mtv_logit_rules *rules, const int32_t *tree_tok, cudaStream_t stream) {
    if (!tree || !tree->on_device || !logits || !rules || (!out && !keys) || B < 1 || V < 1) return MTV_ERR_INVALID_ARG;
    if (dtype != MTV_LOGITS_BF16 && dtype != MTV_LOGITS_F32) return MTV_ERR_INVALID_ARG;
    const size_t size = dtype == MTV_LOGITS_BF16 ? 2 : 4;
    if (ld_in < V || (out && ld_out < V) || (uintptr_t)logits % size || (uintptr_t)out % size) return MTV_ERR_INVALID_ARG;
    if (out == logits && ld_out != ld_in) return MTV_ERR_INVALID_ARG;
    if (!rules->counts != !rules->seen || rules->n_bias < 0 || rules->n_masks < 0) return MTV_ERR_INVALID_ARG;
    if (rules->n_bias > 0 && (!rules->bias_ids || !rules->bias)) return MTV_ERR_INVALID_ARG;
    if (rules->n_masks > 0 && (!rules->mask || !rules->mask_of)) return MTV_ERR_INVALID_ARG;
    if (rules->n_bias > CN_MAX_BIAS || B > 65535 || V > 0x7fffffff - CN_SLAB) return MTV_ERR_UNSUPPORTED_SHAPE;
    ConstrainParams p = {};
    p.logits = logits; p.out = out; p.ld_in = ld_in; p.ld_out = ld_out; p.keys = keys;
    p.counts = rules->counts; p.seen = rules->seen;
    p.repetition = rules->repetition; p.presence = rules->presence; p.frequency = rules->frequency;
    p.bias_ids = rules->bias_ids; p.bias = rules->bias; p.n_bias = rules->n_bias;
    p.mask = rules->mask; p.mask_of = rules->n_masks > 0 ? rules->mask_of : nullptr; p.n_masks = rules->n_masks;
    p.tree_tok = tree_tok; p.anc = tree->d_anc; p.dev_error = tree->d_error;
    p.T = tree->T; p.V = V; p.words = (V + 31) / 32;
    // A row per warp at least; every block lists its slab's tokens anew, so more where that still leaves a few blocks per SM.
    const int64_t slabs = (V + CN_SLAB - 1) / CN_SLAB;
    int per = CN_WARPS;
    while (per < CN_ROWS && slabs * B * ((p.T + 2 * per - 1) / (2 * per)) >= CN_BLOCKS * sm_count()) per *= 2;
    p.B = B; p.rows_per_block = per; p.groups = (p.T + per - 1) / per;
    if (slabs * B * p.groups > 0x7fffffff) return MTV_ERR_UNSUPPORTED_SHAPE;
    const dim3 grid((unsigned)(slabs * B * p.groups));
    p.one_slab = slabs == 1;
    if (keys && !p.one_slab) MTV_CUDA_CHECK(launch_dependent(clear_keys_kernel, dim3((B * p.T + 255) / 256), 256, 0, stream, B * p.T, keys));
    auto kernel = dtype == MTV_LOGITS_BF16 ? (keys ? constrain_kernel<__nv_bfloat16, false> : constrain_kernel<__nv_bfloat16, true>)
                                           : (keys ? constrain_kernel<float, false> : constrain_kernel<float, true>);
    MTV_CUDA_CHECK(launch_dependent(kernel, grid, CN_THREADS, 0, stream, p));
    return MTV_OK;
}

}  // namespace mtv

extern "C" int logits_constrain(const mtv_tree_t *tree, int B, int V, int dtype, const void *logits, int64_t stride_in, void *out,
                                int64_t stride_out, const mtv_logit_rules *rules, const int32_t *tree_tok, void *stream) {
    MTV_RANGE("logits_constrain");
    if (!out) return MTV_ERR_INVALID_ARG;
    return mtv::constrain(tree, B, V, dtype, logits, stride_in, out, stride_out, nullptr, rules, tree_tok, (cudaStream_t)stream);
}

extern "C" int constrained_argmax_keys(const mtv_tree_t *tree, int B, int V, int dtype, const void *logits, int64_t stride_in,
                                       const mtv_logit_rules *rules, const int32_t *tree_tok, unsigned long long *keys, void *stream) {
    MTV_RANGE("constrained_argmax_keys");
    if (!keys || (uintptr_t)keys % 8) return MTV_ERR_INVALID_ARG;
    return mtv::constrain(tree, B, V, dtype, logits, stride_in, nullptr, 0, keys, rules, tree_tok, (cudaStream_t)stream);
}

extern "C" int token_counts_add(int B, int V, int n, const int32_t *tokens, const int32_t *lens, int prompt, uint32_t *counts, uint32_t *seen,
                                void *stream) {
    using namespace mtv;
    MTV_RANGE("token_counts_add");
    if (B < 1 || V < 1 || n < 0 || (n > 0 && !tokens) || !counts || !seen) return MTV_ERR_INVALID_ARG;
    if (B > 65535) return MTV_ERR_UNSUPPORTED_SHAPE;
    if (n == 0) return MTV_OK;
    MTV_CUDA_CHECK(launch_dependent(token_counts_add_kernel, dim3((n + 255) / 256, B), 256, 0, (cudaStream_t)stream, V, (V + 31) / 32, n, prompt ? 1 : 0,
                                    tokens, lens, counts, seen));
    return MTV_OK;
}
