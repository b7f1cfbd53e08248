"""Tree attention over pages of e4m3 codes, against the formula in 64 bits on the values that the codes stand for.

Element by element, with A = sum of the weights times |v| (the formula on |v|): the output's rounding to bf16 is at most 2^-8 of the result, a
weight's rounding to fp16 at most 2^-11 of it (the weights that lose more are below 2^-22 of the largest, and vanish in the rest), an exponential off by at
most 7.5e-5, in the weights and in their sum.  Scores are fp32 sums of exact products: 1e-4 of A covers them at the scores of these inputs (below 2^6)."""
import random

import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _fp8
from tests._cases import make_tree
from tests._paged import table

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 2.0 ** -8
NAN = float("nan")


def bound(want, absolute):
    return EPS * want.abs() + (1 + EPS) * (2.0 ** -11 + 2 * 7.5e-5 + 1e-4) * absolute + 1e-30


def tree_of(K, T):
    if T == 1:
        return dict(mask=[[1]]), binding.tree_build_static(1, [])
    return make_tree("rank_prior", K, (), T)


def want_of(q, kp, vp, ks, vs, t, lens, mask, scale=None):
    return _fp8.attention(q, kp, vp, ks, vs, t, lens, mask, scale)


def run(tree, q, kp, vp, ks, vs, t, lens, shared, out=None, scale=0.0, status=None, stream=None):
    B, T, Hq, D = q.shape
    ws = torch.full((binding.paged_workspace_bytes(tree, B, Hq, kp.shape[1], D, shared),), 0xff, dtype=torch.uint8, device=DEV)   # NaN
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out

    def moved(p):         # with its strides
        return p if p.is_cuda else p.view(torch.uint8).to(DEV).view(_fp8.FP8) if p.is_contiguous() else p.transpose(1, 2).to(DEV).transpose(1, 2)
    binding.tree_verify_attention_paged_fp8(tree, q.to(DEV), moved(kp), moved(vp), t.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out, ws,
                                            ks.to(DEV), vs.to(DEV), shared_len=shared, scale=scale, status=status, stream=stream)
    torch.cuda.synchronize()
    assert binding.mtv_device_error(tree) == 0
    return out.cpu()


def inputs(T, Hq, Hkv, D, page, shared, lens, room=0, seed=1, tokens_outside=False):
    g = torch.Generator().manual_seed(seed)
    t, n_pages = table(g, len(lens), max(lens) - shared + T + room, page, shared)
    kp, vp = _fp8.pools(g, 2, n_pages, Hkv, page, D, tokens_outside)
    ks, vs = _fp8.scales(g, Hkv), _fp8.scales(g, Hkv)
    return t, n_pages, kp, vp, ks, vs, torch.randn(len(lens), T, Hq, D, generator=g).to(torch.bfloat16)


def check(tree, tb, Hq, Hkv, D, page, shared, lens, seed=1, tokens_outside=False, scale=None):
    t, _, kp, vp, ks, vs, q = inputs(tree.T, Hq, Hkv, D, page, shared, lens, seed=seed, tokens_outside=tokens_outside)
    status = torch.full((len(lens),), 5, dtype=torch.int32, device=DEV)
    out = run(tree, q, kp, vp, ks, vs, t, lens, shared, scale=scale or 0.0, status=status)
    assert status.tolist() == [0] * len(lens)
    want, absolute = want_of(q, kp, vp, ks, vs, t, lens, tb["mask"], scale)
    worst = ((out.double() - want).abs() / bound(want, absolute)).max().item()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("K,T,Hq,Hkv,D,page,shared,lens", [
    (1, 1, 4, 1, 128, 16, 0, [0]),                       # one key
    (1, 1, 4, 1, 64, 16, 0, [0, 1, 15, 16, 31, 32, 127, 128, 129]),
    (1, 1, 8, 2, 128, 16, 16, [16, 17, 31, 300]),        # the shared prefix alone in front of the token
    (1, 1, 32, 8, 128, 64, 512, [512 + 17 * i for i in range(40)]),   # more rows than a tile behind the prefix: packed across sequences
    (3, 29, 8, 2, 64, 16, 0, [128]),
    (3, 29, 28, 4, 128, 16, 48, [48, 700, 49]),          # groups of seven; a tile of the prefix ends inside
    (4, 64, 32, 8, 128, 64, 256, [256, 383, 384, 900]),  # two row tiles per sequence
    (4, 64, 12, 4, 128, 32, 128, [200, 500]),            # groups of three
    (4, 65, 6, 1, 64, 128, 384, [384, 400]),             # an odd number of row tiles: pairs and a single one
    (5, 128, 8, 1, 128, 256, 512, [600, 1000]),          # eight row tiles, pages longer than a tile, tree across three key tiles
    (5, 128, 16, 2, 64, 1024, 0, [5, 3000]),
    (5, 128, 5, 5, 128, 16, 160, [161, 161, 161]),       # groups of one
    (4, 20, 4, 1, 128, 64, 0, [9000]),                   # one row tile alone: its keys over all workers
    (4, 64, 4, 1, 128, 64, 0, [20000]),
    (1, 1, 4, 1, 64, 16, 0, [9000] + [1] * 300 + [5000] + [3] * 200),      # long pieces beside many short ones
    (1, 1, 2, 2, 128, 32, 32, [40 + i % 50 for i in range(150)] + [6000]),
    (1, 1, 2, 1, 64, 16, 32, [32 + 7 * i % 40 for i in range(1024)]),          # the largest batch
    (2, 3, 64, 64, 64, 16, 0, [3, 100]),                                        # many KV heads
    (2, 2, 8, 1, 128, 16, 0, [0, 5, 14, 15, 16, 63, 64, 500]),                 # at most 16 query rows a KV head: of a sequence, and of all behind the prefix
    (3, 16, 2, 2, 64, 32, 64, [64, 80, 1001]),
    (3, 4, 16, 4, 128, 64, 128, [128, 129, 2047]),
    (2, 3, 10, 2, 128, 16, 16, [17, 300]),
    (1, 1, 16, 4, 128, 128, 2048, [2048, 2100, 2049, 5000]),
])
def test_against_the_formula(K, T, Hq, Hkv, D, page, shared, lens):
    tb, tree = tree_of(K, T)
    check(tree, tb, Hq, Hkv, D, page, shared, lens)


@pytest.mark.parametrize("seed", range(24))
def test_sizes_at_random(seed):
    """Trees, groups, batches, prefixes and lengths as they come, short ones more often than long ones."""
    r = random.Random(seed)
    K, T = r.choice([2, 3, 4, 5]), 1 if seed % 4 == 0 else int(2 ** r.uniform(1, 7))
    D, page, Hkv, G = r.choice([64, 128]), r.choice([16, 32, 64, 128, 256]), r.choice([1, 2, 3]), r.randint(1, 8)
    B = int(2 ** r.uniform(0, 5))
    shared = r.choice([0, 0, int(2 ** r.uniform(4, 11))]) // page * page
    lens = [shared + int(2 ** r.uniform(0, 11)) - 1 for _ in range(B)]
    tb, tree = tree_of(K, T)
    check(tree, tb, Hkv * G, Hkv, D, page, shared, lens, seed=seed, tokens_outside=bool(seed & 1))


@pytest.mark.parametrize("T,Hq,Hkv,D,page,shared,lens", [
    (64, 32, 8, 128, 64, 256, [256, 383, 900]), (29, 8, 2, 64, 16, 48, [700, 49]), (1, 8, 2, 128, 16, 32, [33, 32, 400]), (4, 4, 1, 64, 16, 0, [77]),
])
def test_pages_with_the_heads_inside(T, Hq, Hkv, D, page, shared, lens):
    tb, tree = tree_of(4, T)
    check(tree, tb, Hq, Hkv, D, page, shared, lens, tokens_outside=True)
    check(tree, tb, Hq, Hkv, D, page, shared, lens, scale=0.3)


@pytest.mark.parametrize("D,T,G", [(128, 64, 4), (64, 1, 8), (128, 20, 3), (128, 4, 4), (64, 64, 8)])
@pytest.mark.parametrize("size", [1.0, 30.0, 300.0])
def test_scores_that_grow_along_the_keys(D, T, G, size):
    """Keys that get longer: the reference has to move from tile to tile, by up to hundreds; the softmax ends up on few keys."""
    tb, tree = tree_of(4, T)
    shared, lens, page, Hkv = 320, [700, 1500], 32, 2
    t, n_pages, kp, vp, ks, vs, q = inputs(T, Hkv * G, Hkv, D, page, shared, lens, seed=7)
    grow = torch.ones(n_pages, page)
    for b in range(2):
        for i, pg in enumerate(t[b].tolist()):
            grow[pg] = (0.05 + (i * page + torch.arange(page)) / 1500.0) / 1.1
    kp = (kp.float() * grow[:, None, :, None]).to(_fp8.FP8)
    ks = ks * size / 0.014 / 100                           # values of `size` units at the end
    out = run(tree, q, kp, vp, ks, vs, t, lens, shared)
    want, absolute = want_of(q, kp, vp, ks, vs, t, lens, tb["mask"])
    # scores up to S = 9 * size in natural units (six deviations, the scales up to 1.43 of their middle), their fp32 sums off by at most 128 products' rounding
    # and the factor's two (2^-24 each, of S): relative error of a weight up to 130 * 2^-24 * S in front of the softmax; twice (numerator and sum)
    slop = 2 * 130 * 2.0 ** -24 * 9 * size * absolute
    assert ((out.double() - want).abs() / (bound(want, absolute) + slop)).max().item() <= 1.0


@pytest.mark.parametrize("T,G", [(1, 4), (20, 3), (64, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [-60, -16, 14, 60])
def test_queries_of_any_size(D, T, G, power):
    """Queries far outside fp16's range, rows of one sequence of different sizes: the scores' factor makes up for it."""
    tb, tree = tree_of(4, T)
    shared, lens, page, Hkv = 64, [64, 200, 517], 16, 2
    t, _, kp, vp, ks, vs, q = inputs(T, Hkv * G, Hkv, D, page, shared, lens, seed=9)
    out = run(tree, (q.float() * 2.0 ** power).to(torch.bfloat16), kp, vp, ks, vs, t, lens, shared, scale=D ** -0.5 * 2.0 ** -power)
    assert torch.equal(out, run(tree, q, kp, vp, ks, vs, t, lens, shared, scale=D ** -0.5))
    size = 2.0 ** torch.randint(-30, 4, (len(lens), T, Hkv * G, 1), generator=torch.Generator().manual_seed(3)).float()
    q = (q.float() * size).to(torch.bfloat16)
    q[0, 0, 0] = 0.0
    q[1, 0, 0, 1:] *= 2.0 ** -9                               # the largest far in front of the rest
    out = run(tree, q, kp, vp, ks, vs, t, lens, shared)
    want, absolute = want_of(q, kp, vp, ks, vs, t, lens, tb["mask"])
    # rows of size up to 8: scores up to 2^6 * 8 / 4 at the deviations of these inputs; 130 * 2^-24 of them, twice
    assert ((out.double() - want).abs() / (bound(want, absolute) + 2 * 130 * 2.0 ** -24 * 128 * absolute)).max().item() <= 1.0


@pytest.mark.parametrize("T,G", [(1, 4), (20, 3), (64, 4)])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_are_all_zero(D, T, G):
    """Queries and a scale so small that their factor is none of fp32's: every visible key weighs the same."""
    tb, tree = tree_of(4, T)
    shared, lens, page, Hkv = 64, [64, 200, 517], 16, 2
    t, _, kp, vp, ks, vs, q = inputs(T, Hkv * G, Hkv, D, page, shared, lens, seed=9)
    out = run(tree, (q.float() * 2.0 ** -120).to(torch.bfloat16), kp, vp, ks, vs, t, lens, shared, scale=1e-20)
    want, absolute = want_of(torch.zeros_like(q), kp, vp, ks, vs, t, lens, tb["mask"])
    assert ((out.double() - want).abs() / bound(want, absolute)).max().item() <= 1.0


@pytest.mark.parametrize("K,T,Hq,Hkv,D,page,shared,lens", [
    (3, 20, 32, 8, 64, 16, 0, [(37 * i) % 400 for i in range(300)]),       # single row tiles, eight items a worker
    (3, 20, 32, 8, 128, 16, 32, [32 + (91 * i) % 300 for i in range(150)]),
    (4, 64, 32, 8, 128, 32, 0, [(53 * i) % 500 for i in range(100)]),      # pairs, five a worker, ten
    (4, 64, 16, 4, 64, 16, 64, [64 + (29 * i) % 200 for i in range(400)]),
    (5, 100, 24, 8, 128, 16, 0, [(17 * i) % 300 for i in range(60)]),      # three row tiles: pairs and single ones
])
def test_many_short_pieces(K, T, Hq, Hkv, D, page, shared, lens):
    """More pieces a worker than are handed out at a time."""
    tb, tree = tree_of(K, T)
    check(tree, tb, Hq, Hkv, D, page, shared, lens)


@pytest.mark.parametrize("T", [20, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_row_tiles_beyond_32_bits(D, T):
    """Pages whose offsets pass 2^32 bytes, with a NaN in a V row that some nodes see."""
    tb, tree = tree_of(4, T)
    Hq, Hkv, page, n_pages, stride = 8, 2, 64, 4, (1 << 30) + (1 << 29) + 48
    g = torch.Generator().manual_seed(3)
    small = _fp8.pools(g, 2, n_pages, Hkv, page, D)
    t, lens = torch.tensor([[3, 1, 2]], dtype=torch.int32), [70]
    mask = torch.tensor(tb["mask"], dtype=torch.bool)
    ks, vs = _fp8.scales(g, Hkv), _fp8.scales(g, Hkv)
    q = torch.randn(1, T, Hq, D, generator=g).to(torch.bfloat16)
    want, absolute = want_of(q, *small, ks, vs, t, lens, tb["mask"])
    node = T - 1
    pg, r = int(t[0, (lens[0] + node) // page]), (lens[0] + node) % page
    _fp8.put(small[1], (pg, 0, r, 5), NAN)
    want[0][mask[:, node], :Hq // Hkv, 5] = NAN
    big = []
    for x in small:
        buf = torch.empty((n_pages - 1) * stride + Hkv * page * D, dtype=torch.uint8, device=DEV)
        y = buf.as_strided((n_pages, Hkv, page, D), (stride, page * D, D, 1))
        y.copy_(x.view(torch.uint8))
        big.append(y.view(_fp8.FP8))
    out = run(tree, q, *big, ks, vs, t, lens, 0).double()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert ((out - want).abs() / bound(want, absolute))[fine].max().item() <= 1.0


@pytest.mark.parametrize("T", [1, 4, 29, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_rows_reach_those_who_see_them(D, T):
    """NaN codes in K and V rows of single nodes and behind the last node: nodes that do not see them have the results of a cache without them."""
    tb, tree = tree_of(4, T)
    shared, lens, page, Hkv, G = 64, [130, 300, 64], 16, 2, 4
    t, _, kp, vp, ks, vs, q = inputs(T, Hkv * G, Hkv, D, page, shared, lens, room=40, seed=11)
    clean, absolute = want_of(q, kp, vp, ks, vs, t, lens, tb["mask"])
    mask = torch.tensor(tb["mask"], dtype=torch.bool)
    at = lambda b, s: (int(t[b, s // page]), s % page)  # noqa: E731
    bad_v = {} if T == 1 else {0: min(5, T - 1), 1: T - 1, 2: T // 2}
    want = clean.clone()
    for b, L in enumerate(lens):
        for s in range(L + T, L + T + 30):       # behind the last node
            pg, r = at(b, s)
            _fp8.put(kp, (pg, slice(None), r), NAN)
            _fp8.put(vp, (pg, slice(None), r), -NAN)
        if b in bad_v:
            pg, r = at(b, L + bad_v[b])
            _fp8.put(vp, (pg, 1, r, slice(3, None, 7)), NAN if b else -NAN)
            want[b][mask[:, bad_v[b]], G:, 3::7] = NAN
    if T > 1:                                    # a K row of NaN: every row that sees it is NaN
        pg, r = at(0, lens[0] + T - 2)
        _fp8.put(kp, (pg, 0, r), NAN)
        want[0][mask[:, T - 2], :G] = NAN
    out = run(tree, q, kp, vp, ks, vs, t, lens, shared).double()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert ((out - want).abs() / bound(want, absolute))[fine].max().item() <= 1.0


@pytest.mark.parametrize("T", [64, 20, 3, 1])
@pytest.mark.parametrize("D", [64, 128])
def test_non_finite_queries_and_prefix(D, T):
    """A NaN or an infinity in a query row makes that row NaN and no other; a NaN in a prefix key every row of its head, one in a prefix value its column."""
    tb, tree = tree_of(4, T)
    shared, lens, page, Hkv, G = 128, [400, 200], 16, 2, 4
    t, _, kp, vp, ks, vs, q = inputs(T, Hkv * G, Hkv, D, page, shared, lens, seed=13)
    clean, absolute = want_of(q, kp, vp, ks, vs, t, lens, tb["mask"])
    for col, x in ((0, NAN), (15, float("inf")), (D // 2 - 1, float("-inf")), (D - 1, NAN)):
        y = q.clone()
        y[1, T - 1, 5, col] = x
        out = run(tree, y, kp, vp, ks, vs, t, lens, shared).double()
        want = clean.clone()
        want[1, T - 1, 5] = NAN
        assert torch.equal(torch.isnan(out), torch.isnan(want)), (col, x)
        fine = ~torch.isnan(want)
        assert ((out - want).abs() / bound(want, absolute))[fine].max().item() <= 1.0
    pg = int(t[0, 2])
    _fp8.put(kp, (pg, 1, 3, 17), NAN)
    _fp8.put(vp, (pg, 0, 5, 9), NAN)
    out = run(tree, q, kp, vp, ks, vs, t, lens, shared)
    want = torch.zeros(out.shape, dtype=torch.bool)
    want[:, :, G:] = True
    want[:, :, :G, 9] = True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("T,G", [(64, 4), (20, 3), (1, 4), (4, 4)])
@pytest.mark.parametrize("D", [64, 128])
def test_sequences_that_cannot_be(D, T, G):
    """Lengths that do not fit or end inside the prefix: out stays as it was.  A page that is not there: BOUNDS, and the other sequences have
    what they would have alone.  Table entries behind the last slot are never followed."""
    tb, tree = tree_of(4, T)
    page, shared, Hkv = 16, 64, 2
    lens = [130, 63, -1, 300, 400, 210, 416 - T, 417 - T]
    g = torch.Generator().manual_seed(5)
    t, n_pages = table(g, len(lens), 416 - shared, page, shared)
    kp, vp = _fp8.pools(g, 2, n_pages, Hkv, page, D)
    ks, vs = _fp8.scales(g, Hkv), _fp8.scales(g, Hkv)
    q = torch.randn(len(lens), T, Hkv * G, D, generator=g).to(torch.bfloat16)
    bad = t.clone()
    bad[3, 100 // page] = n_pages
    bad[0, -(-(130 + T) // page):] = -1
    bad[5, (210 + T - 1) // page] = -3
    status = torch.full((len(lens),), 5, dtype=torch.int32, device=DEV)
    out = run(tree, q, kp, vp, ks, vs, bad, lens, shared, status=status)
    cap = -6
    assert status.tolist() == [0, cap, cap, -7, cap if 400 + T > 416 else 0, -7, 0, cap]
    ok = [b for b in range(len(lens)) if status[b] == 0]
    want, absolute = want_of(q[ok], kp, vp, ks, vs, t[ok], [lens[b] for b in ok], tb["mask"])
    assert ((out[ok].double() - want).abs() / bound(want, absolute)).max().item() <= 1.0
    for b in range(len(lens)):
        if status[b] == cap:
            assert (out[b] == 7.0).all()
    bad = t.clone()
    bad[0, 1] = n_pages + 5                      # a page of the prefix: it is missing for all
    run(tree, q, kp, vp, ks, vs, bad, lens, shared, status=status)
    assert all(s in (-7, cap) for s in status.tolist()[:1])


@pytest.mark.parametrize("T", [64, 20, 1])
def test_two_streams_and_a_graph(T):
    """Calls with workspaces of their own on two streams at once, and two graphs over one workspace replayed in turn, with other lengths and
    scales than at their capture; every pass gives the same bits."""
    tb, tree = tree_of(4, T)
    Hq, Hkv, D, page, shared = 16, 4, 128, 16, 96
    lens = [[96, 500, 1000], [700, 97, 333]]
    t, _, kp, vp, ks, vs, q = inputs(T, Hq, Hkv, D, page, shared, [96, 500, 1000], seed=5)
    kd, vd, td, ksd, vsd = kp.view(torch.uint8).to(DEV).view(_fp8.FP8), vp.view(torch.uint8).to(DEV).view(_fp8.FP8), t.to(DEV), ks.to(DEV), vs.to(DEV)
    qd = [q.to(DEV), q.flip(0).to(DEV)]
    ld = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in lens]
    n = binding.paged_workspace_bytes(tree, 3, Hq, Hkv, D, shared)
    ws = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [torch.zeros_like(x) for x in qd]

    def right():
        torch.cuda.synchronize()
        for i in range(2):
            want = want_of(qd[i].cpu(), kp, vp, ksd.cpu(), vsd.cpu(), t, ld[i].tolist(), tb["mask"])
            assert ((outs[i].cpu().double() - want[0]).abs() / bound(*want)).max().item() <= 1.0
    call = lambda i, w, stream=None: binding.tree_verify_attention_paged_fp8(tree, qd[i], kd, vd, td, ld[i], outs[i], ws[w], ksd, vsd, shared_len=shared, stream=stream)  # noqa: E731
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for i in range(2):
            call(i, i, streams[i])
    right()
    eager = [o.clone() for o in outs]
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=streams[0]):
            call(i, 0, streams[0])
    ws[0].fill_(0xff)
    for changed in (False, True):
        if changed:
            ld[0].copy_(torch.tensor(lens[1])), ld[1].copy_(torch.tensor(lens[0]))
            ksd.mul_(1.25), vsd.mul_(0.5)
        for o in outs:
            o.fill_(9.0)
        for _ in range(3):
            graphs[0].replay()
            graphs[1].replay()
        right()
        if not changed:
            assert all(torch.equal(a, b) for a, b in zip(eager, outs))
    assert binding.mtv_device_error(tree) == 0


@pytest.mark.parametrize("T,G", [(1, 4), (20, 8), (64, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_that_vanish(D, T, G):
    """A visible key whose score is 300 below the others' adds nothing, whatever its V row and its column; a key far above them all leaves nothing of them."""
    tb, tree = tree_of(4, T)
    page, Hkv, lens = 16, 2, [300 + i for i in range(16)]
    t, _, kp, vp, ks, vs, q = inputs(T, Hkv * G, Hkv, D, page, 0, lens, seed=19)
    ks[:] = 300.0 * D ** 0.5 / 16 / 448
    kp = (kp.float() * 0.002).to(_fp8.FP8)
    kp.view(torch.uint8)[..., 0] = 0
    q[..., 0] = 16.0
    clean = vp.clone()
    for sign in (-1, 1):
        for b, L in enumerate(lens):
            for s in (5 + b, 130 + b, L - 1):
                pg, r = int(t[b, s // page]), s % page
                _fp8.put(kp, (pg, slice(None), r, 0), sign * 448.0)
                _fp8.put(vp, (pg, slice(None), r), 448.0)
                _fp8.put(clean, (pg, slice(None), r), 0.0 if sign < 0 else 448.0)
        want, absolute = want_of(q, kp, clean, ks, vs, t, lens, tb["mask"])
        out = run(tree, q, kp, vp, ks, vs, t, lens, 0)
        # scores up to 302: 130 * 2^-24 of them, twice
        assert ((out.double() - want).abs() / (bound(want, absolute) + 2 * 130 * 2.0 ** -24 * 302 * absolute)).max().item() <= 1.0


def test_refusals():
    tb, tree = tree_of(4, 20)
    page, Hkv, Hq, D, lens = 16, 2, 4, 64, [70, 80]
    t, _, kp, vp, ks, vs, q = inputs(20, Hq, Hkv, D, page, 0, lens, seed=5)
    kp, vp, ks, vs, q = kp.to(DEV), vp.to(DEV), ks.to(DEV), vs.to(DEV), q.to(DEV)
    td, ld, out = t.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), torch.full_like(q, 7.0)
    n = binding.paged_workspace_bytes(tree, 2, Hq, Hkv, D)
    ws = torch.zeros(n + 512, dtype=torch.uint8, device=DEV)
    ws = ws[-ws.data_ptr() % 256:]

    def code(q=q, out=out, ws=ws[:n], shared=0, scale=0.0, kp=kp, vp=vp, ks=ks, vs=vs):
        with pytest.raises(binding.MtvError) as e:
            binding.tree_verify_attention_paged_fp8(tree, q, kp, vp, td, ld, out, ws, ks, vs, shared_len=shared, scale=scale)
        return e.value.code
    assert code(ws=ws[:n - 1]) == -3 and code(ws=ws[16:n + 16]) in (-1, -3)
    assert code(shared=8) == -1 and code(shared=-16) == -1 and code(shared=16 * (t.shape[1] + 1)) == -1
    for s in (-1.0, NAN, float("inf")):
        assert code(scale=s) == -1
    off = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device=DEV)[1:1 + q.numel()].view(q.shape)
    assert code(q=off) == -1 and code(out=off) == -1
    wide = torch.zeros(2, 20, 5, D, dtype=torch.bfloat16, device=DEV)
    assert code(q=wide, out=torch.zeros_like(wide)) in (-1, -2)
    byte = torch.zeros(kp.numel() + 16, dtype=torch.uint8, device=DEV)[8:8 + kp.numel()].view(kp.shape).view(_fp8.FP8)
    assert code(kp=byte) == -1 and code(vp=byte) == -1
    eight = torch.zeros(kp.shape[0], Hkv, page, D + 8, dtype=torch.uint8, device=DEV).view(_fp8.FP8)[..., :D]      # rows at multiples of 8 bytes
    assert code(kp=eight, vp=eight) == -1
    assert code(kp=kp.view(torch.uint8)) == -1 and code(ks=ks[:1]) == -1 and code(vs=vs.double()) == -1 and code(ks=None) == -1
    torch.cuda.synchronize()
    assert (out == 7.0).all() and binding.mtv_device_error(tree) == 0
