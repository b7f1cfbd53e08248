// Tree attention over a K/V cache in pages, of a batch whose first keys are the same (Section 3.2 / Fig. 2(b)).
// A warp per query row, keys one after the other with a running maximum and sum.
#include "attn_common.cuh"
#include "paged_common.cuh"

namespace mtv {

struct PagedAttnParams {
    PagedRef pages;
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16 *out;
    const int32_t *seq_lens;
    const uint64_t *anc;
    int32_t *status;
    float scale_log2;
    int B, T, Hq, G, D, shared;
};

__global__ void __launch_bounds__(256)
paged_attn_kernel(const PagedAttnParams p) {
    previous_done();
    let_next_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int b = blockIdx.y;
    const int L = p.seq_lens[b];
    const bool fits = p.pages.fits(L, p.T) && L >= p.shared;
    if (blockIdx.x == 0 && warp == 0 && p.status) {
        int code = fits ? p.pages.check(b, p.shared, L - p.shared + p.T, lane) : MTV_ERR_CAPACITY;
        if (code == MTV_OK) code = p.pages.check(0, 0, p.shared, lane);
        if (lane == 0) p.status[b] = code;
    }
    const int row = (int)blockIdx.x * 8 + warp;
    if (!fits || row >= p.T * p.Hq) return;
    const int i = row / p.Hq, h = row % p.Hq;
    const int per = p.D / 32;
    const __nv_bfloat16 *qr = p.q + ((size_t)b * p.T * p.Hq + row) * p.D;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    for (int d = 0; d < per; ++d) q[d] = __bfloat162float(qr[d * 32 + lane]) * p.scale_log2;
    for (int s = 0; s < L + p.T; ++s) {
        const int a = s - L;
        if (a >= 0 && !(p.anc[i * 2 + a / 64] >> (a % 64) & 1)) continue;
        const int64_t at = p.pages.row(s < p.shared ? 0 : b, s);
        const int64_t off = at + (int64_t)(h / p.G) * p.pages.stride_h + lane;
        float x = 0.f;
        if (at >= 0)
            for (int d = 0; d < per; ++d) x += q[d] * __bfloat162float(p.k[off + d * 32]);
        for (int k = 16; k; k /= 2) x += __shfl_xor_sync(0xffffffffu, x, k);
        const float m_new = fmaxf(m, x), w = exp2f(x - m_new), keep = exp2f(m - m_new);
        l = l * keep + w;
        for (int d = 0; d < per; ++d) o[d] = o[d] * keep + (at >= 0 ? w * __bfloat162float(p.v[off + d * 32]) : 0.f);
        m = m_new;
    }
    for (int d = 0; d < per; ++d) p.out[((size_t)b * p.T * p.Hq + row) * p.D + d * 32 + lane] = __float2bfloat16_rn(o[d] / l);
}

}  // namespace mtv

extern "C" size_t tree_attention_paged_workspace_bytes(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, int shared_len) {
    if (!tree || B < 1 || B > 1024 || Hkv < 1 || Hq < Hkv || Hq % Hkv || Hq / Hkv > 8 || (D != 64 && D != 128) || shared_len < 0) return 0;
    return 256;
}

extern "C" int tree_verify_attention_paged(const mtv_tree_t *tree, int B, int Hq, int Hkv, int D, const mtv_bf16 *q, const mtv_bf16 *k_pool,
                                           const mtv_bf16 *v_pool, const mtv_pool_layout *pool, const int32_t *page_table, int max_pages,
                                           int shared_len, const int32_t *seq_lens, float scale, mtv_bf16 *out, int32_t *status,
                                           void *ws, size_t ws_bytes, void *stream) {
    using namespace mtv;
    MTV_RANGE("tree_verify_attention_paged");
    if (!tree || !tree->on_device || !q || !k_pool || !v_pool || !seq_lens || !out || !ws) return MTV_ERR_INVALID_ARG;
    if (B < 1 || Hq < 1 || Hkv < 1 || shared_len < 0 || !(scale >= 0.f)) return MTV_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || Hq % Hkv || Hq / Hkv > 8 || B > 1024) return MTV_ERR_UNSUPPORTED_SHAPE;
    PagedAttnParams p = {};
    const int rc = paged_ref(p.pages, pool, page_table, max_pages, D);
    if (rc != MTV_OK) return rc;
    if (shared_len % pool->page_size || ((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_pool | (uintptr_t)v_pool) & 15) return MTV_ERR_INVALID_ARG;
    if (ws_bytes < tree_attention_paged_workspace_bytes(tree, B, Hq, Hkv, D, shared_len)) return MTV_ERR_WORKSPACE;
    p.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    p.k = reinterpret_cast<const __nv_bfloat16 *>(k_pool);
    p.v = reinterpret_cast<const __nv_bfloat16 *>(v_pool);
    p.out = reinterpret_cast<__nv_bfloat16 *>(out);
    p.seq_lens = seq_lens; p.anc = tree->d_anc; p.status = status;
    p.scale_log2 = (scale == 0.f ? 1.f / sqrtf((float)D) : scale) * 1.4426950408889634f;
    p.B = B; p.T = tree->T; p.Hq = Hq; p.G = Hq / Hkv; p.D = D; p.shared = shared_len;
    MTV_CUDA_CHECK(launch_dependent(paged_attn_kernel, dim3((tree->T * Hq + 7) / 8, B), 256, 0, (cudaStream_t)stream, p));
    return MTV_OK;
}
