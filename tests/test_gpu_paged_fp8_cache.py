"""Rows quantised into pages of e4m3 codes, read back, and the accepted rows moved.

A code stands next to the value that is stored: half a step, 2^-4 of a value or 2^-10 at the smallest.  In front of it a rotated value is off by less than
2^-19 of its pair's sum of sizes (see the bf16 cache), and the factor 1 / scale and the product with it by 2^-24 each."""
import pytest
import torch

from oracle import reference as ref
from paper_2603_03383_b200 import binding
from tests import _fp8
from tests._cases import make_tree
from tests._paged import contiguous, table

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, U8 = torch.bfloat16, torch.uint8
CAPACITY, BOUNDS = -6, -7


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def tree_of(K, T):
    if T == 1:
        return dict(mask=[[1]], depth=[0], T=1), binding.tree_build_static(1, [])
    return make_tree("rank_prior", K, (), T)


def numbers(codes):
    return codes.view(_fp8.FP8).float().double()


def stored(codes, want, scale, x=None):
    """Codes [..., heads, D] (bytes) next to want / scale [heads]; x: what was rotated."""
    s = scale.double()[:, None]
    v = want / s
    slack = 2.0 ** -22 * v.abs()
    if x is not None:
        h = x.shape[-1] // 2
        pair = x.double().abs()
        pair = pair[..., :h] + pair[..., h:]
        slack = slack + 2.0 ** -19 * torch.cat([pair, pair], -1) / s
    v = v.clamp(-_fp8.MAX, _fp8.MAX)
    return ((numbers(codes) - v).abs() <= 2.0 ** -4 * v.abs() + 2.0 ** -10 + slack).all()


def rotated(got, want, x):
    h = x.shape[-1] // 2
    pair = x.double().abs()
    pair = pair[..., :h] + pair[..., h:]
    return ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * torch.cat([pair, pair], -1) + 1e-38).all()


def byte_pools(g, n, n_pages, Hkv, page, D, outside=False):
    out = []
    for _ in range(n):
        x = torch.randint(0, 256, (n_pages, page, Hkv, D) if outside else (n_pages, Hkv, page, D), generator=g, dtype=torch.int32).to(U8).to(DEV)
        out.append(x.transpose(1, 2) if outside else x)
    return out


def layout(pool):
    return binding.pool_layout(pool.view(_fp8.FP8))


def ptrs(*pools):
    return [binding.cache_pointer_array(p, DEV) for p in pools]


def rows(g, n_layers, shape, Hq, Hkv, D, offset=0):
    cpu = [torch.randn(n_layers, *shape, h, D, generator=g).to(BF16) for h in (Hq, Hkv, Hkv)]
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
])
@pytest.mark.parametrize("in_place", [False, True])
def test_tree_rows(K, T, Hq, Hkv, D, page, lens, theta, layers, outside, offset, in_place):
    tb, tree = tree_of(K, T)
    g = torch.Generator().manual_seed(4)
    B = len(lens)
    t, n_pages = table(g, B, max(lens) + T, page)
    kp, vp = byte_pools(g, layers, n_pages, Hkv, page, D, outside), byte_pools(g, layers, n_pages, Hkv, page, D, outside)
    before = [(k.cpu(), v.cpu()) for k, v in zip(kp, vp)]
    (q, kn, vn), (qd, knd, vnd) = rows(g, layers, (B, T), Hq, Hkv, D, offset)
    ks, vs = _fp8.scales(g, layers, Hkv), _fp8.scales(g, layers, Hkv)
    ks[0, 0], vs[-1, -1] = 0.001, 0.0015                           # many values beyond the largest code
    ks[-1, -1], vs[0, 0] = 3.0, 20.0                               # many below the smallest
    out = qd if in_place else torch.full_like(qd, 7.0)
    status = i32([5] * B)
    binding.tree_kv_append_rope_paged_fp8(tree, qd, out, knd, vnd, *ptrs(kp, vp), layout(kp[0]), t.to(DEV), i32(lens), ks.to(DEV), vs.to(DEV),
                                          rope_theta=theta, status=status)
    assert status.tolist() == [0] * B
    for l, (k0, v0) in enumerate(before):
        q_ref, k_ref = ref.rope(q[l], kn[l], lens, tb["depth"], theta or 10000.0)
        assert rotated(out[l].cpu(), q_ref, q[l])
        k1, v1 = kp[l].cpu(), vp[l].cpu()
        for b, L in enumerate(lens):
            s = L + torch.arange(T)
            pg, r = t[b][s // page].long(), s % page
            assert stored(k1[pg, :, r], k_ref[b], ks[l], kn[l, b]) and stored(v1[pg, :, r], vn[l, b].double(), vs[l])
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
def test_ragged_rows_and_back(Hq, Hkv, D, page, lens, counts, front, back, in_place):
    """Runs of tokens are quantised; the same runs read back are what their codes stand for, rounded once; padding stays as it was on either way."""
    g = torch.Generator().manual_seed(8)
    B, layers = len(lens), 2
    t, n_pages = table(g, B, max(L + n for L, n in zip(lens, counts)) + 1, page)
    kp, vp = byte_pools(g, layers, n_pages, Hkv, page, D), byte_pools(g, layers, n_pages, Hkv, page, D)
    k0, v0 = [x.cpu() for x in kp], [x.cpu() for x in vp]
    starts = [front]
    for n in counts:
        starts.append(starts[-1] + n)
    (q, kn, vn), (qd, knd, vnd) = rows(g, layers, (starts[-1] + back,), Hq, Hkv, D)
    ks, vs = _fp8.scales(g, layers, Hkv), _fp8.scales(g, layers, Hkv)
    out = qd if in_place else torch.full_like(qd, 7.0)
    status = i32([5] * B)
    args = (*ptrs(kp, vp), layout(kp[0]), t.to(DEV))
    binding.kv_append_rope_paged_fp8(qd, out, knd, vnd, *args, i32(lens), i32(starts), ks.to(DEV), vs.to(DEV), status=status)
    assert status.tolist() == [0] * B
    back_k, back_v = torch.full_like(knd, 7.0), torch.full_like(vnd, 7.0)
    status.fill_(5)
    binding.kv_read_paged_fp8(*args, i32(starts), ks.to(DEV), vs.to(DEV), back_k, back_v, first=i32(lens), status=status)
    assert status.tolist() == [0] * B
    for l in range(layers):
        k1, v1, got = kp[l].cpu(), vp[l].cpu(), out[l].cpu()
        for b, (L, n) in enumerate(zip(lens, counts)):
            if not n:
                continue
            s = slice(starts[b], starts[b + 1])
            q_ref, k_ref = ref.rope(q[l, s][None], kn[l, s][None], [L], list(range(n)))
            assert rotated(got[s], q_ref[0], q[l, s])
            at = L + torch.arange(n)
            pg, r = t[b][at // page].long(), at % page
            assert stored(k1[pg, :, r], k_ref[0], ks[l], kn[l, s]) and stored(v1[pg, :, r], vn[l, s].double(), vs[l])
            for codes, scale, x in ((k1, ks, back_k), (v1, vs, back_v)):
                want = (codes[pg, :, r].view(_fp8.FP8).float() * scale[l][:, None]).to(BF16)
                assert torch.equal(x[l, s].cpu(), want)
            k0[l][pg, :, r], v0[l][pg, :, r] = k1[pg, :, r], v1[pg, :, r]
        assert torch.equal(k0[l], k1) and torch.equal(v0[l], v1)
        for s in (slice(0, front), slice(starts[-1], None)):        # padding
            assert torch.equal(got[s], q[l, s] if in_place else torch.full_like(got[s], 7.0))
            assert (back_k[l, s] == 7.0).all() and (back_v[l, s] == 7.0).all()


def test_what_has_no_code():
    """NaN stays NaN, infinities and what is too large become the largest code; zeros keep their sign."""
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([nan, -nan, inf, -inf, 3e38, -3e38, 449.0, 480.0, 448.0, 0.0, -0.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, -1.0, 17.0], dtype=BF16)
    want = torch.tensor([0x7f, 0x7f, 0x7e, 0xfe, 0x7e, 0xfe, 0x7e, 0x7e, 0x7e, 0x00, 0x80, 0x01, 0x00, 0x01, 0xb8, 0x58], dtype=torch.int32)   # 2^-10, 17: ties to even
    kp, vp = torch.zeros(2, 1, 16, 64, dtype=U8, device=DEV), torch.zeros(2, 1, 16, 64, dtype=U8, device=DEV)
    row = torch.zeros(1, 1, 1, 64, dtype=BF16)
    row[..., :16] = x
    row = row.to(DEV)
    one = torch.ones(1, 1, device=DEV)
    t = i32([[1]])
    binding.kv_append_rope_paged_fp8(row.clone(), row.clone(), row, row, *ptrs([kp], [vp]), layout(kp), t, i32([0]), i32([0, 1]), one, one)
    for p in (kp, vp):                                             # (position 0: nothing turns, but inf * 0 is NaN)
        got = p[1, 0, 0, :16].cpu().to(torch.int32)
        same = (got == want) | (((got & 0x7f) == 0x7f) & ((want & 0x7f) == 0x7f))
        if p is kp:
            same[2:4] = True
        assert same.all(), got
    k, v = torch.zeros(1, 1, 1, 64, dtype=BF16, device=DEV), torch.zeros(1, 1, 1, 64, dtype=BF16, device=DEV)
    binding.kv_read_paged_fp8(*ptrs([kp], [vp]), layout(kp), t, i32([0, 1]), one, one, k, v)
    assert torch.isnan(v[0, 0, 0, :2]).all() and v[0, 0, 0, 2:6].tolist() == [448.0, -448.0, 448.0, -448.0]


def test_every_code_is_read():
    """All 256 codes with a scale that fp32 has no short form of, and one whose products pass bf16's middle."""
    for D in (64, 128):
        codes = torch.arange(256, dtype=torch.int32).to(U8).view(1, 1, 256 // D, D).repeat(1, 1, 16 * D // 256, 1).to(DEV)
        for scale in (1.0, 0.1, 1.00390625, 1e30):
            s = torch.full((1, 1), scale, device=DEV)
            k, v = (torch.zeros(1, 16, 1, D, dtype=BF16, device=DEV) for _ in range(2))
            binding.kv_read_paged_fp8(*ptrs([codes], [codes]), layout(codes), i32([[0]]), i32([0, 16]), s, s, k, v)
            want = (codes.cpu()[0, 0].view(_fp8.FP8).float() * s.cpu()).to(BF16)
            for x in (k, v):
                got = x[0, :, 0].cpu()
                assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_rows_that_are_not_there():
    """Sequences that do not fit are left alone; rows of a page that is not there are left out, on the way in and back."""
    g = torch.Generator().manual_seed(2)
    page, Hq, Hkv, D = 16, 4, 2, 64
    lens, counts = [10, 45, -1, 20, 44, 0], [20, 20, 3, 20, 20, 64]
    B = len(lens)
    t, n_pages = table(g, B, 64, page)
    t[3, 2] = n_pages                           # slots 32 .. 47 of sequence 3
    t[0, 3] = -7                                # behind sequence 0's last slot: never followed
    t[5, 1] = -1
    want_status = [0, CAPACITY, CAPACITY, BOUNDS, 0, BOUNDS]
    kp, vp = byte_pools(g, 1, n_pages, Hkv, page, D), byte_pools(g, 1, n_pages, Hkv, page, D)
    k0, v0 = kp[0].cpu(), vp[0].cpu()
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    (q, kn, vn), (qd, knd, vnd) = rows(g, 1, (starts[-1],), Hq, Hkv, D)
    ks, vs = _fp8.scales(g, 1, Hkv).to(DEV), _fp8.scales(g, 1, Hkv).to(DEV)
    status = i32([5] * B)
    args = (*ptrs(kp, vp), layout(kp[0]), t.to(DEV))
    binding.kv_append_rope_paged_fp8(qd, qd, knd, vnd, *args, i32(lens), i32(starts), ks, vs, status=status)
    assert status.tolist() == want_status
    back_k, back_v = torch.full_like(knd, 7.0), torch.full_like(vnd, 7.0)
    binding.kv_read_paged_fp8(*args, i32(starts), ks, vs, back_k, back_v, first=i32(lens), status=status)
    assert status.tolist() == want_status
    k1, v1 = kp[0].cpu(), vp[0].cpu()
    for b in range(B):
        s = slice(starts[b], starts[b + 1])
        if want_status[b] == CAPACITY:
            assert torch.equal(qd[0, s].cpu(), q[0, s]) and (back_k[0, s] == 7.0).all() and (back_v[0, s] == 7.0).all()
            continue
        for i in range(counts[b]):
            slot = lens[b] + i
            pg, r = int(t[b, slot // page]), slot % page
            if not 0 <= pg < n_pages:
                assert (back_k[0, starts[b] + i] == 7.0).all() and (back_v[0, starts[b] + i] == 7.0).all()
                continue
            assert stored(v1[pg, :, r], vn[0, starts[b] + i].double(), vs[0].cpu())
            assert torch.equal(back_v[0, starts[b] + i].cpu(), (v1[pg, :, r].view(_fp8.FP8).float() * vs[0].cpu()[:, None]).to(BF16))
            k0[pg, :, r], v0[pg, :, r] = k1[pg, :, r], v1[pg, :, r]
    assert torch.equal(k0, k1) and torch.equal(v0, v1)


@pytest.mark.parametrize("layers", [1, 40])
def test_reading_many_layers_from_the_start(layers):
    """first is left out; more layers than a block takes; heads inside a page; outputs that begin between 32-byte boundaries."""
    g = torch.Generator().manual_seed(12)
    page, Hkv, D, counts = 32, 3, 128, [0, 70, 1, 300]
    t, n_pages = table(g, 4, 300, page)
    kp, vp = byte_pools(g, layers, n_pages, Hkv, page, D, True), byte_pools(g, layers, n_pages, Hkv, page, D, True)
    ks, vs = _fp8.scales(g, layers, Hkv).to(DEV), _fp8.scales(g, layers, Hkv).to(DEV)
    starts = [0, 0, 70, 71, 371]
    out = [torch.zeros(layers * 371 * Hkv * D + 8, dtype=BF16, device=DEV)[8:].view(layers, 371, Hkv, D) for _ in range(2)]
    binding.kv_read_paged_fp8(*ptrs(kp, vp), layout(kp[0]), t.to(DEV), i32(starts), ks, vs, *out)
    for l in range(layers):
        for pool, scale, x in ((kp, ks, out[0]), (vp, vs, out[1])):
            want = (pool[l].contiguous().view(_fp8.FP8).float() * scale[l][None, :, None, None]).to(BF16).cpu()
            for b, n in enumerate(counts):
                got, exp = x[l, starts[b]:starts[b + 1]].cpu().transpose(0, 1), contiguous(want, t)[b][:, :n]
                assert torch.equal(torch.isnan(got), torch.isnan(exp)) and torch.equal(got.nan_to_num(), exp.nan_to_num())


def test_no_rows_at_all():
    g = torch.Generator().manual_seed(8)
    t, n_pages = table(g, 3, 32, 16)
    kp, vp = byte_pools(g, 2, n_pages, 2, 16, 64), byte_pools(g, 2, n_pages, 2, 16, 64)
    before = [x.clone() for x in kp + vp]
    q, k = torch.empty(2, 0, 4, 64, dtype=BF16, device=DEV), torch.empty(2, 0, 2, 64, dtype=BF16, device=DEV)
    s = torch.ones(2, 2, device=DEV)
    status, lens, starts = i32([5] * 3), i32([0, 33, -1]), i32([0, 0, 0, 0])
    args = (*ptrs(kp, vp), layout(kp[0]), t.to(DEV))
    binding.kv_append_rope_paged_fp8(q, q, k, k, *args, lens, starts, s, s, status=status)
    assert status.tolist() == [0, CAPACITY, CAPACITY]
    status.fill_(5)
    binding.kv_read_paged_fp8(*args, starts, s, s, k, k, first=lens, status=status)
    assert status.tolist() == [0, CAPACITY, CAPACITY]
    assert all(torch.equal(x, y) for x, y in zip(before, kp + vp))


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
    kp, vp = byte_pools(g, layers, n_pages, Hkv, page, D, outside), byte_pools(g, layers, n_pages, Hkv, page, D, outside)
    k0, v0 = [x.cpu() for x in kp], [x.cpu() for x in vp]
    sl, status = i32(lens), i32([5] * B)
    new = sl if in_place else i32([-3] * B)
    binding.kv_compact_accepted_paged_fp8(tree, *ptrs(kp, vp), layers, Hkv, D, layout(kp[0]), t.to(DEV), sl, new, i32(n), nodes.to(DEV), status)
    assert status.tolist() == [0] * B and new.tolist() == [L + m + 1 for L, m in zip(lens, n)]
    for l in range(layers):
        for x0, x1 in ((k0[l], kp[l].cpu()), (v0[l], vp[l].cpu())):
            want = x0.clone()
            for b, L in enumerate(lens):
                for j in range(1, n[b] + 1):
                    src, dst = L + int(nodes[b, j]), L + j
                    want[int(t[b, dst // page]), :, dst % page] = x0[int(t[b, src // page]), :, src % page]
            assert torch.equal(x1, want)


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
    kp, vp = byte_pools(g, 1, n_pages, Hkv, page, D), byte_pools(g, 1, n_pages, Hkv, page, D)
    k0 = kp[0].cpu()
    sl, status = i32(lens), i32([5] * B)
    new = sl if in_place else i32([-3] * B)
    binding.kv_compact_accepted_paged_fp8(tree, *ptrs(kp, vp), 1, Hkv, D, layout(kp[0]), t.to(DEV), sl, new, i32(n), i32(nodes), status)
    assert status.tolist() == want_status
    old = lens if in_place else [-3] * B
    assert new.tolist() == [L + m + 1 if s == 0 else o for L, m, s, o in zip(lens, n, want_status, old)]
    want = k0.clone()
    for b in range(B):
        for j in range(1, n[b] + 1):
            if want_status[b] == 0:
                src, dst = lens[b] + nodes[b][j], lens[b] + j
                want[int(t[b, dst // page]), :, dst % page] = k0[int(t[b, src // page]), :, src % page]
    assert torch.equal(kp[0].cpu(), want)


def test_pools_beyond_32_bits():
    """Pages whose offsets pass 2^32 bytes, on strides that leave gaps between few rows: appended, attended to, read back, moved."""
    tb, tree = tree_of(2, 4)
    T, Hq, Hkv, D, page = 4, 4, 2, 64, 16
    n_pages, stride_page = 5, (1 << 30) + (1 << 28) + 16
    g = torch.Generator().manual_seed(3)
    buf = [torch.empty((n_pages - 1) * stride_page + Hkv * page * D, dtype=U8, device=DEV) for _ in range(2)]
    kp, vp = (x.as_strided((n_pages, Hkv, page, D), (stride_page, page * D, D, 1)) for x in buf)
    for x in (kp, vp):
        x.copy_((100.0 * torch.randn(n_pages, Hkv, page, D, generator=g)).clamp(-448, 448).to(_fp8.FP8).view(U8))
    k0, v0 = kp.cpu(), vp.cpu()
    t = torch.tensor([[3, 4, 2]], dtype=torch.int32)
    (q, kn, vn), (qd, knd, vnd) = rows(g, 1, (1, T), Hq, Hkv, D)
    ks, vs = _fp8.scales(g, 1, Hkv), _fp8.scales(g, 1, Hkv)
    ksd, vsd = ks.to(DEV), vs.to(DEV)
    at, pool = ptrs([kp], [vp]), binding.pool_layout(kp.view(_fp8.FP8))
    status, sl = i32([5]), i32([30])
    binding.tree_kv_append_rope_paged_fp8(tree, qd, qd, knd, vnd, *at, pool, t.to(DEV), sl, ksd, vsd, status=status)
    assert status.tolist() == [0]
    _, k_ref = ref.rope(q[0], kn[0], [30], tb["depth"])
    k1, v1 = kp.cpu(), vp.cpu()
    s = 30 + torch.arange(T)
    pg, r = t[0][s // page].long(), s % page
    assert stored(k1[pg, :, r], k_ref[0], ks[0], kn[0, 0]) and stored(v1[pg, :, r], vn[0, 0].double(), vs[0])
    k0[pg, :, r], v0[pg, :, r] = k1[pg, :, r], v1[pg, :, r]
    assert torch.equal(k0, k1) and torch.equal(v0, v1)
    ws = torch.empty(binding.paged_workspace_bytes(tree, 1, Hq, Hkv, D), dtype=U8, device=DEV)
    out = torch.empty(1, T, Hq, D, dtype=BF16, device=DEV)
    binding.tree_verify_attention_paged_fp8(tree, qd[0], kp.view(_fp8.FP8), vp.view(_fp8.FP8), t.to(DEV), sl, out, ws, ksd[0], vsd[0], status=status)
    assert status.tolist() == [0]
    want, absolute = _fp8.attention(qd[0].cpu(), k1, v1, ks[0], vs[0], t, [30], tb["mask"])
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3 * absolute).all()
    k, v = (torch.zeros(1, 34, Hkv, D, dtype=BF16, device=DEV) for _ in range(2))
    binding.kv_read_paged_fp8(*at, pool, t.to(DEV), i32([0, 34]), ksd, vsd, k, v, status=status)
    for x, codes, scale in ((k, k1, ks), (v, v1, vs)):
        assert torch.equal(x[0].cpu().transpose(0, 1), contiguous((codes.view(_fp8.FP8).float() * scale[0][None, :, None, None]).to(BF16), t)[0][:, :34])
    node = 3 if tb["depth"][3] == 1 else 2
    binding.kv_compact_accepted_paged_fp8(tree, *at, 1, Hkv, D, pool, t.to(DEV), sl, sl, i32([1]), i32([[0, node, -1]]), status)
    assert status.tolist() == [0] and sl.tolist() == [32]
    to, of = ((int(t[0, x // page]), slice(None), x % page) for x in (31, 30 + node))
    k1[to], v1[to] = k1[of], v1[of]
    assert torch.equal(kp.cpu(), k1) and torch.equal(vp.cpu(), v1)


def test_layouts_of_another_type():
    """A layout that was made of a bf16 pool is refused where codes are meant, and the other way round; strides of 8 elements by the library."""
    g = torch.Generator().manual_seed(8)
    t, n_pages = table(g, 2, 64, 16)
    kp, vp = byte_pools(g, 1, n_pages, 2, 16, 64), byte_pools(g, 1, n_pages, 2, 16, 64)
    half = torch.zeros(n_pages, 2, 16, 64, dtype=BF16, device=DEV)
    tree = tree_of(3, 20)[1]
    (_, _, _), (q, k, v) = rows(g, 1, (2, 20), 4, 2, 64)
    s = torch.ones(1, 2, device=DEV)
    at, sl = ptrs(kp, vp), i32([0, 0])

    def code(f, *a, **kw):
        with pytest.raises(binding.MtvError) as e:
            f(*a, **kw)
        return e.value.code
    good, bad = layout(kp[0]), binding.pool_layout(half)
    assert code(binding.tree_kv_append_rope_paged_fp8, tree, q, q, k, v, *at, bad, t.to(DEV), sl, s, s) == -1
    assert code(binding.tree_kv_append_rope_paged, tree, q, q, k, v, *at, good, t.to(DEV), sl) == -1
    assert code(binding.kv_compact_accepted_paged_fp8, tree, *at, 1, 2, 64, bad, t.to(DEV), sl, sl, sl, i32([[0] * 4] * 2)) == -1
    assert code(binding.kv_read_paged_fp8, *at, bad, t.to(DEV), i32([0, 1, 2]), s, s, k[:, 0], v[:, 0]) == -1
    for kw in (dict(stride_t=72), dict(stride_h=1032), dict(stride_page=2056)):
        odd = layout(kp[0])
        for name, x in kw.items():
            setattr(odd, name, x)
        assert code(binding.tree_kv_append_rope_paged_fp8, tree, q, q, k, v, *at, odd, t.to(DEV), sl, s, s) == -1
    off = torch.zeros(k[:, 0].numel() + 8, dtype=BF16, device=DEV)[1:1 + k[:, 0].numel()].view(k[:, 0].shape)
    assert code(binding.kv_read_paged_fp8, *at, good, t.to(DEV), i32([0, 1, 2]), s, s, off, off) == -1
