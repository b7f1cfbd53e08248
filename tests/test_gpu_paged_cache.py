"""Rows appended to pages with the rotary embedding, and the accepted rows moved, against the oracle in 64 bits.

A rotated value a cos - b sin: fp32 with an angle below pi that was reduced in double precision and rounded (2^-23), sine and cosine good to
2^-22, two products and a sum (2^-24 each): off by less than 2^-20 (|a| + |b|), then one rounding to bf16, at most 2^-8 of the value."""
import pytest
import torch

from oracle import reference as ref
from paper_2603_03383_b200 import binding
from tests._cases import make_tree
from tests._paged import contiguous, pools, table

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
CAPACITY, BOUNDS = -6, -7


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def tree_of(K, T):
    if T == 1:
        return dict(mask=[[1]], depth=[0], T=1), binding.tree_build_static(1, [])
    return make_tree("rank_prior", K, (), T)


def close(got, want, x):
    """got bf16, want fp64 rotations of x, last dimension D."""
    h = x.shape[-1] // 2
    pair = x.double().abs()
    pair = (pair[..., :h] + pair[..., h:]).repeat_interleave(1, -1)
    pair = torch.cat([pair, pair], -1)
    return ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * pair + 1e-38).all()


def appended(g, n_layers, rows, Hq, Hkv, D, offset=0):
    """q, k_new, v_new [n_layers, *rows, heads, D] on the CPU and on the device; there they begin `offset` elements behind a boundary."""
    cpu = [torch.randn(n_layers, *rows, h, D, generator=g).to(BF16) for h in (Hq, Hkv, Hkv)]
    dev = []
    for x in cpu:
        buf = torch.zeros(x.numel() + offset, dtype=BF16, device=DEV)
        dev.append(buf[offset:].view(x.shape))
        dev[-1].copy_(x)
    return cpu, dev


@pytest.mark.parametrize("K,T,Hq,Hkv,D,page,lens,theta,layers,outside,offset", [
    (1, 1, 1, 1, 64, 16, [0], 0.0, 1, False, 0),
    (1, 1, 28, 4, 128, 16, [0, 15, 16, 700], 0.0, 3, False, 0),
    (3, 29, 8, 2, 64, 16, [0, 517, 30000], 500000.0, 2, False, 0),
    (4, 64, 32, 8, 128, 64, [100, 63, 64, 65, 1], 0.0, 2, True, 0),
    (4, 65, 7, 1, 128, 32, [5, 31], 10000.0, 5, True, 0),
    (5, 128, 5, 5, 64, 1024, [1000, 3], 0.0, 1, False, 3),       # rows at odd addresses
    (2, 3, 4, 2, 128, 65536, [65534], 0.0, 70, False, 0),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_tree_rows(K, T, Hq, Hkv, D, page, lens, theta, layers, outside, offset, in_place):
    tb, tree = tree_of(K, T)
    g = torch.Generator().manual_seed(4)
    B = len(lens)
    t, n_pages = table(g, B, max(lens) + T, page)
    if page == 65536:                 # one page is enough to read back
        kp, vp = ([torch.randn(n_pages, Hkv, page, D, device=DEV).to(BF16)] * layers for _ in range(2))
        layers_kept = [layers - 1]
    else:
        kp, vp = (pools(g, layers, n_pages, Hkv, page, D, outside, DEV) for _ in range(2))
        layers_kept = range(layers)
    before = [(kp[l].cpu(), vp[l].cpu()) for l in layers_kept]
    (q, kn, vn), (qd, knd, vnd) = appended(g, layers, (B, T), Hq, Hkv, D, offset)
    if page == 65536:                 # all layers write the same buffers: the same rows
        for x, y in ((q, qd), (kn, knd), (vn, vnd)):
            x[:] = x[-1:].clone()
            y.copy_(x)
    out = qd if in_place else torch.full_like(qd, 7.0)
    status = i32([5] * B)
    binding.tree_kv_append_rope_paged(tree, qd, out, knd, vnd, binding.cache_pointer_array(kp, DEV), binding.cache_pointer_array(vp, DEV),
                                      binding.pool_layout(kp[0]), t.to(DEV), i32(lens), rope_theta=theta, status=status)
    assert status.tolist() == [0] * B
    for l, (k0, v0) in zip(layers_kept, before):
        q_ref, k_ref = ref.rope(q[l], kn[l], lens, tb["depth"], theta or 10000.0)
        assert close(out[l].cpu(), q_ref, q[l])
        k1, v1 = kp[l].cpu(), vp[l].cpu()
        for b, L in enumerate(lens):
            for i in range(T):
                pg, r = int(t[b, (L + i) // page]), (L + i) % page
                assert close(k1[pg, :, r], k_ref[b, i], kn[l, b, i])
                assert torch.equal(v1[pg, :, r], vn[l, b, i])
                k0[pg, :, r], v0[pg, :, r] = k1[pg, :, r], v1[pg, :, r]
        assert torch.equal(k0, k1) and torch.equal(v0, v1)          # nothing else was written


@pytest.mark.parametrize("Hq,Hkv,D,page,lens,counts,front,back", [
    (4, 1, 128, 16, [0], [1], 0, 0),
    (28, 4, 128, 16, [0, 3, 15, 100], [40, 1, 17, 0], 0, 0),
    (8, 2, 64, 32, [5, 0, 0, 31, 64], [0, 0, 33, 1, 0], 3, 5),     # padding in front and behind; sequences without rows
    (2, 2, 64, 16, [7] * 300, [i % 3 for i in range(300)], 0, 9),
    (6, 2, 128, 64, [0, 0], [0, 0], 0, 4),                          # padding alone
])
@pytest.mark.parametrize("in_place", [False, True])
def test_ragged_rows(Hq, Hkv, D, page, lens, counts, front, back, in_place):
    g = torch.Generator().manual_seed(8)
    B, layers = len(lens), 2
    t, n_pages = table(g, B, max(L + n for L, n in zip(lens, counts)) + 1, page)
    kp, vp = (pools(g, layers, n_pages, Hkv, page, D, False, DEV) for _ in range(2))
    k0, v0 = [x.cpu() for x in kp], [x.cpu() for x in vp]
    starts = [front]
    for n in counts:
        starts.append(starts[-1] + n)
    (q, kn, vn), (qd, knd, vnd) = appended(g, layers, (starts[-1] + back,), Hq, Hkv, D)
    out = qd if in_place else torch.full_like(qd, 7.0)
    status = i32([5] * B)
    binding.kv_append_rope_paged(qd, out, knd, vnd, binding.cache_pointer_array(kp, DEV), binding.cache_pointer_array(vp, DEV),
                                 binding.pool_layout(kp[0]), t.to(DEV), i32(lens), i32(starts), status=status)
    assert status.tolist() == [0] * B
    for l in range(layers):
        k1, v1, got = kp[l].cpu(), vp[l].cpu(), out[l].cpu()
        for b, (L, n) in enumerate(zip(lens, counts)):
            s = slice(starts[b], starts[b + 1])
            if n:
                q_ref, k_ref = ref.rope(q[l, s][None], kn[l, s][None], [L], list(range(n)))
                assert close(got[s], q_ref[0], q[l, s])
            for i in range(n):
                pg, r = int(t[b, (L + i) // page]), (L + i) % page
                assert close(k1[pg, :, r], k_ref[0, i], kn[l, starts[b] + i])
                assert torch.equal(v1[pg, :, r], vn[l, starts[b] + i])
                k0[l][pg, :, r], v0[l][pg, :, r] = k1[pg, :, r], v1[pg, :, r]
        assert torch.equal(k0[l], k1) and torch.equal(v0[l], v1)
        for s in (slice(0, front), slice(starts[-1], None)):        # padding
            assert torch.equal(got[s], q[l, s] if in_place else torch.full_like(got[s], 7.0))


def test_no_rows_at_all():
    g = torch.Generator().manual_seed(8)
    t, n_pages = table(g, 3, 32, 16)
    kp, vp = (pools(g, 1, n_pages, 2, 16, 64, False, DEV) for _ in range(2))
    k0 = kp[0].clone()
    q, k = torch.empty(1, 0, 4, 64, dtype=BF16, device=DEV), torch.empty(1, 0, 2, 64, dtype=BF16, device=DEV)
    some = torch.zeros(8, dtype=BF16, device=DEV)
    status = i32([5] * 3)
    L = binding.lib()
    pool, td, lens, starts = binding.pool_layout(kp[0]), t.to(DEV), i32([0, 33, -1]), i32([0, 0, 0, 0])
    ptrs = [binding.cache_pointer_array(x, DEV) for x in (kp, vp)]
    assert L.kv_append_rope_paged(3, 0, 4, 2, 64, 1, *[some.data_ptr()] * 4, ptrs[0].data_ptr(), ptrs[1].data_ptr(), pool, td.data_ptr(),
                                  td.shape[1], lens.data_ptr(), starts.data_ptr(), 0.0, status.data_ptr(), 0) == 0
    assert status.tolist() == [0, CAPACITY, CAPACITY]
    assert torch.equal(kp[0], k0) and (q.numel(), k.numel()) == (0, 0)


def test_append_to_what_is_not_there():
    """Sequences that do not fit are left alone; rows of a page that is not there are left out; the others have what they would have alone."""
    tb, tree = tree_of(3, 20)
    g = torch.Generator().manual_seed(2)
    page, T, B, Hq, Hkv, D = 16, 20, 5, 4, 2, 64
    t, n_pages = table(g, B, 64, page)
    lens = [10, 45, -1, 20, 44]                 # 64 slots: 45 + 20 does not fit, 44 + 20 does
    t[3, 2] = n_pages                           # slots 32 .. 47 of sequence 3
    t[0, 3] = -7                                # behind sequence 0's last slot: never followed
    kp, vp = (pools(g, 1, n_pages, Hkv, page, D, False, DEV) for _ in range(2))
    k0, v0 = kp[0].cpu(), vp[0].cpu()
    (q, kn, vn), (qd, knd, vnd) = appended(g, 1, (B, T), Hq, Hkv, D)
    status = i32([5] * B)
    binding.tree_kv_append_rope_paged(tree, qd, qd, knd, vnd, binding.cache_pointer_array(kp, DEV), binding.cache_pointer_array(vp, DEV),
                                      binding.pool_layout(kp[0]), t.to(DEV), i32(lens), status=status)
    assert status.tolist() == [0, CAPACITY, CAPACITY, BOUNDS, 0]
    k1, v1 = kp[0].cpu(), vp[0].cpu()
    q_ref, k_ref = ref.rope(q[0], kn[0], [max(0, L) for L in lens], tb["depth"])
    for b in range(B):
        if status[b] == CAPACITY:
            assert torch.equal(qd[0, b].cpu(), q[0, b])
            continue
        assert close(qd[0, b].cpu(), q_ref[b], q[0, b])
        for i in range(T):
            s = lens[b] + i
            if b == 3 and 32 <= s < 48:
                continue
            pg, r = int(t[b, s // page]), s % page
            assert close(k1[pg, :, r], k_ref[b, i], kn[0, b, i])
            k0[pg, :, r], v0[pg, :, r] = k1[pg, :, r], vn[0, b, i]
    assert torch.equal(k0, k1) and torch.equal(v0, v1)


def test_pools_beyond_32_bits():
    """Pages whose offsets pass 2^32 elements, on strides that leave gaps between few rows."""
    tb, tree = tree_of(2, 4)
    T, Hq, Hkv, D, page = 4, 4, 2, 64, 16
    n_pages, stride_page = 5, (1 << 30) + 8
    g = torch.Generator().manual_seed(3)
    buf = [torch.empty((n_pages - 1) * stride_page + Hkv * page * D, dtype=BF16, device=DEV) for _ in range(2)]
    kp, vp = (x.as_strided((n_pages, Hkv, page, D), (stride_page, page * D, D, 1)) for x in buf)
    for x in (kp, vp):
        x.copy_(torch.randn(n_pages, Hkv, page, D, generator=g).to(BF16))
    k0, v0 = kp.cpu(), vp.cpu()
    t = torch.tensor([[3, 4, 2]], dtype=torch.int32)
    (q, kn, vn), (qd, knd, vnd) = appended(g, 1, (1, T), Hq, Hkv, D)
    ptrs = [binding.cache_pointer_array([x], DEV) for x in (kp, vp)]
    pool = binding.pool_layout(kp)
    status, sl = i32([5]), i32([30])
    binding.tree_kv_append_rope_paged(tree, qd, qd, knd, vnd, *ptrs, pool, t.to(DEV), sl, status=status)
    assert status.tolist() == [0]
    _, k_ref = ref.rope(q[0], kn[0], [30], tb["depth"])
    k1, v1 = kp.cpu(), vp.cpu()
    for i in range(T):
        pg, r = int(t[0, (30 + i) // page]), (30 + i) % page
        assert close(k1[pg, :, r], k_ref[0, i], kn[0, 0, i]) and torch.equal(v1[pg, :, r], vn[0, 0, i])
        k0[pg, :, r], v0[pg, :, r] = k1[pg, :, r], vn[0, 0, i]
    assert torch.equal(k0, k1) and torch.equal(v0, v1)
    ws = torch.empty(binding.paged_workspace_bytes(tree, 1, Hq, Hkv, D), dtype=torch.uint8, device=DEV)
    out = torch.empty(1, T, Hq, D, dtype=BF16, device=DEV)
    binding.tree_verify_attention_paged(tree, qd[0], kp, vp, t.to(DEV), sl, out, ws, status=status)
    assert status.tolist() == [0]
    want = ref.tree_attention(qd[0].cpu(), contiguous(k1, t), contiguous(v1, t), torch.tensor([30], dtype=torch.int32), tb["mask"])
    assert (out.cpu().double() - want).abs().max().item() <= 2.0 ** -7 * v1.abs().max().item()
    node = 3 if tb["depth"][3] == 1 else 2
    binding.kv_compact_accepted_paged(tree, *ptrs, 1, Hkv, D, pool, t.to(DEV), sl, sl, i32([1]), i32([[0, node, -1]]), status)
    assert status.tolist() == [0] and sl.tolist() == [32]
    at = lambda s: (int(t[0, s // page]), slice(None), s % page)  # noqa: E731
    k1[at(31)], v1[at(31)] = k1[at(30 + node)], v1[at(30 + node)]
    assert torch.equal(kp.cpu(), k1) and torch.equal(vp.cpu(), v1)


@pytest.mark.parametrize("K,T,Hkv,D,page,outside,layers", [
    (4, 64, 8, 128, 64, False, 2), (4, 64, 3, 64, 16, True, 3), (8, 9, 40, 128, 16, False, 1), (1, 1, 2, 64, 16, False, 2), (5, 128, 1, 128, 32, True, 1),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_compaction(K, T, Hkv, D, page, outside, layers, in_place):
    """Every length of a path, rows that are another's destination, nodes in no order a tree would give them."""
    tb, tree = make_tree("cartesian", K, (1,) * K) if T == K + 1 else tree_of(K, T)
    g = torch.Generator().manual_seed(6)
    K = tree.K
    B = 2 * (K + 1) + 1
    lens = [(7 * b * b) % 90 for b in range(B)]
    n = [min(b % (K + 1), T - 1) for b in range(B)]
    nodes = torch.full((B, K + 1), -1, dtype=torch.int32)
    for b in range(B):
        order = torch.randperm(T - 1, generator=g)[:n[b]] + 1 if b % 3 else torch.arange(2, n[b] + 2).clamp(max=T - 1)   # slot j + 1 to slot j
        nodes[b, 0], nodes[b, 1:n[b] + 1] = 0, order.to(torch.int32)
    t, n_pages = table(g, B, max(lens) + T, page)
    kp, vp = (pools(g, layers, n_pages, Hkv, page, D, outside, DEV) for _ in range(2))
    k0, v0 = [x.cpu() for x in kp], [x.cpu() for x in vp]
    sl, status = i32(lens), i32([5] * B)
    new = sl if in_place else i32([-3] * B)
    binding.kv_compact_accepted_paged(tree, binding.cache_pointer_array(kp, DEV), binding.cache_pointer_array(vp, DEV), layers, Hkv, D,
                                      binding.pool_layout(kp[0]), t.to(DEV), sl, new, i32(n), nodes.to(DEV), status)
    assert status.tolist() == [0] * B and new.tolist() == [L + m + 1 for L, m in zip(lens, n)]
    for l in range(layers):
        for x0, x1 in ((k0[l], kp[l].cpu()), (v0[l], vp[l].cpu())):
            want, lens_ref = ref.kv_compact(contiguous(x0, t), lens, n, nodes)
            assert torch.equal(contiguous(x1, t), want) and lens_ref.tolist() == new.tolist()
            held = torch.zeros(n_pages, dtype=torch.bool)
            held[t.long().view(-1)] = True
            assert torch.equal(x1[~held], x0[~held])


@pytest.mark.parametrize("in_place", [False, True])
def test_compaction_that_cannot_be(in_place):
    tb, tree = tree_of(3, 20)
    g = torch.Generator().manual_seed(2)
    page, T, Hkv, D = 16, 20, 2, 64
    lens = [10, 45, -1, 20, 12, 14, 8, 9, 30]
    n = [2, 1, 0, 2, 4, -1, 2, 3, 1]
    nodes = [[0, 3, 9, -1], [0, 1, -1, -1], [0, -1, -1, -1], [0, 5, 15, -1], [0, 1, 2, 3], [0, 1, 2, 3], [0, 20, 2, -1], [0, 1, -1, 2], [0, 7, 99, 99]]
    B = len(lens)
    t, n_pages = table(g, B, 64, page)
    t[3, 2] = n_pages                        # node 15 of sequence 3 lies there
    t[8, 3] = -1                             # needed by no accepted node
    want_status = [0, CAPACITY, CAPACITY, BOUNDS, BOUNDS, BOUNDS, BOUNDS, BOUNDS, 0]
    kp, vp = (pools(g, 1, n_pages, Hkv, page, D, False, DEV) for _ in range(2))
    k0 = kp[0].cpu()
    sl, status = i32(lens), i32([5] * B)
    new = sl if in_place else i32([-3] * B)
    binding.kv_compact_accepted_paged(tree, binding.cache_pointer_array(kp, DEV), binding.cache_pointer_array(vp, DEV), 1, Hkv, D,
                                      binding.pool_layout(kp[0]), t.to(DEV), sl, new, i32(n), i32(nodes), status)
    assert status.tolist() == want_status
    old = lens if in_place else [-3] * B
    assert new.tolist() == [L + m + 1 if s == 0 else o for L, m, s, o in zip(lens, n, want_status, old)]
    moved = []
    for b in range(B):
        for j in range(1, n[b] + 1):
            if want_status[b] == 0:
                src, dst = lens[b] + nodes[b][j], lens[b] + j
                moved.append((int(t[b, dst // page]), dst % page, k0[int(t[b, src // page]), :, src % page].clone()))
    for pg, r, x in moved:
        k0[pg, :, r] = x
    assert torch.equal(kp[0].cpu(), k0)


def test_no_rows_in_empty_tensors():
    """Tensors without rows have no address: the call reports the lengths all the same."""
    g = torch.Generator().manual_seed(8)
    t, n_pages = table(g, 3, 32, 16)
    kp, vp = (pools(g, 2, n_pages, 2, 16, 64, False, DEV) for _ in range(2))
    before = [x.clone() for x in kp + vp]
    q, k = torch.empty(2, 0, 4, 64, dtype=BF16, device=DEV), torch.empty(2, 0, 2, 64, dtype=BF16, device=DEV)
    assert q.data_ptr() == 0
    status = i32([5] * 3)
    binding.kv_append_rope_paged(q, q, k, k, binding.cache_pointer_array(kp, DEV), binding.cache_pointer_array(vp, DEV), binding.pool_layout(kp[0]),
                                 t.to(DEV), i32([0, 33, -1]), i32([0, 0, 0, 0]), status=status)
    assert status.tolist() == [0, CAPACITY, CAPACITY]
    assert all(torch.equal(x, y) for x, y in zip(before, kp + vp))
