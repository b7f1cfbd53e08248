"""Tree attention over pages with a shared prefix, against the oracle on the contiguous cache that the page table stands for.

Element by element, with A = sum of the weights times |v| (the oracle on |v|): the output's rounding to bf16 is at most 2^-8 of the
result, the weights' rounding to bf16 in front of the second product at most 2^-8 of A.  Scores are fp32 sums of exact products, exponentials
good to 2^-21: 1e-4 of A covers them at the scores of these inputs (below 2^6)."""
import pytest
import torch

from oracle import reference as ref
from paper_2603_03383_b200 import binding
from tests._cases import make_tree
from tests._paged import contiguous, pools, table

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 2.0 ** -8


def bound(want, absolute):
    return EPS * want.abs() + 1.02 * EPS * absolute + 1e-4 * absolute + 1e-30


def want_of(q, kp, vp, t, lens, mask, scale=None):
    k, v = contiguous(kp, t), contiguous(vp, t)
    want = ref.tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32), mask, scale)
    return want, ref.tree_attention(q, k, v.abs(), torch.tensor(lens, dtype=torch.int32), mask, scale)


def run(tree, q, kp, vp, t, lens, shared, out=None, scale=0.0, status=None, stream=None):
    B, T, Hq, D = q.shape
    ws = torch.full((binding.paged_workspace_bytes(tree, B, Hq, kp.shape[1], D, shared),), 0xff, dtype=torch.uint8, device=DEV)   # NaN
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    binding.tree_verify_attention_paged(tree, q.to(DEV), kp.to(DEV) if kp.device.type == "cpu" else kp,
                                        vp.to(DEV) if vp.device.type == "cpu" else vp, t.to(DEV),
                                        torch.tensor(lens, dtype=torch.int32, device=DEV), out, ws, shared_len=shared, scale=scale,
                                        status=status, stream=stream)
    torch.cuda.synchronize()
    assert binding.mtv_device_error(tree) == 0
    return out.cpu()


def check(tree, tb, Hq, Hkv, D, page, shared, lens, seed=1, tokens_outside=False, scale=None):
    g = torch.Generator().manual_seed(seed)
    B, T = len(lens), tree.T
    t, n_pages = table(g, B, max(lens) - shared + T, page, shared)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D, tokens_outside)
    q = torch.randn(B, T, Hq, D, generator=g).to(torch.bfloat16)
    status = torch.full((B,), 5, dtype=torch.int32, device=DEV)
    out = run(tree, q, kp, vp, t, lens, shared, scale=scale or 0.0, status=status)
    assert status.tolist() == [0] * B
    want, absolute = want_of(q, kp, vp, t, lens, tb["mask"], scale)
    err = (out.double() - want).abs()
    worst = (err / bound(want, absolute)).max().item()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("K,T,Hq,Hkv,D,page,shared,lens", [
    (1, 1, 4, 1, 128, 16, 0, [0]),                       # one key
    (1, 1, 4, 1, 64, 16, 0, [0, 1, 15, 16, 127, 128, 129]),
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
    (1, 1, 4, 1, 64, 16, 0, [9000] + [1] * 300 + [5000] + [3] * 200),      # long pieces beside many short ones
    (1, 1, 2, 2, 128, 32, 32, [40 + i % 50 for i in range(150)] + [6000]),
    (1, 1, 2, 1, 64, 16, 32, [32 + 7 * i % 40 for i in range(1024)]),          # the largest batch
    (2, 3, 64, 64, 64, 16, 0, [3, 100]),                                        # many KV heads
    # at most 16 query rows a KV head: of a sequence, and of all behind the prefix (2 x 8, 4 x 4)
    (2, 2, 8, 1, 128, 16, 0, [0, 5, 14, 15, 16, 63, 64, 500]),
    (3, 16, 2, 2, 64, 32, 64, [64, 80, 1001]),
    (3, 4, 16, 4, 128, 64, 128, [128, 129, 2047]),
    (2, 3, 10, 2, 128, 16, 16, [17, 300]),
    (1, 1, 8, 1, 64, 16, 160, [160, 333]),
    (1, 1, 16, 4, 128, 128, 2048, [2048, 2100, 2049, 5000]),
])
def test_against_the_oracle(K, T, Hq, Hkv, D, page, shared, lens):
    tb, tree = make_tree("rank_prior", K, (), T) if T > 1 else make_tree("cartesian", 1, (1,))
    if T == 1:
        tree = binding.tree_build_static(1, [])
        tb = dict(mask=[[1]])
    check(tree, tb, Hq, Hkv, D, page, shared, lens)


def _tree(K, T):
    if T == 1:
        return dict(mask=[[1]]), binding.tree_build_static(1, [])
    return make_tree("rank_prior", K, (), T)


@pytest.mark.parametrize("D,T,G", [(128, 64, 4), (64, 1, 8), (128, 20, 3), (128, 4, 4)])
@pytest.mark.parametrize("size", [1.0, 30.0, 300.0])
def test_scores_that_grow_along_the_keys(D, T, G, size):
    """Keys that get longer: the running maximum of most rows rises from tile to tile, by up to hundreds, so that the reference has to
    move; the softmax ends up on few keys."""
    tb, tree = _tree(4, T)
    g = torch.Generator().manual_seed(7)
    shared, lens, page, Hkv = 320, [700, 1500], 32, 2
    t, n_pages = table(g, 2, 1500 - shared + T, page, shared)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D)
    grow = torch.ones(n_pages, page)
    for b in range(2):
        for i, pg in enumerate(t[b].tolist()):
            grow[pg] = 0.05 + size * ((i * page + torch.arange(page)) / 1500.0)
    kp = (kp.float() * grow[:, None, :, None]).to(torch.bfloat16)
    q = torch.randn(2, T, Hkv * G, D, generator=g).to(torch.bfloat16)
    out = run(tree, q, kp, vp, t, lens, shared)
    want, absolute = want_of(q, kp, vp, t, lens, tb["mask"])
    # scores up to S = 6 * size in natural units, their fp32 sums off by at most 128 products' rounding (2^-24 each, of S): relative error of a weight
    # up to 128 * 2^-24 * S in front of the softmax; twice (numerator and sum)
    slop = 2 * 128 * 2.0 ** -24 * 6 * size * absolute
    assert ((out.double() - want).abs() / (bound(want, absolute) + slop)).max().item() <= 1.0


@pytest.mark.parametrize("T", [1, 4, 29, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_non_finite_rows_reach_those_who_see_them(D, T):
    """NaN and infinities in K and V rows of single nodes and behind the last node: nodes that do not see them have the results of a cache
    without them, the others NaN or infinite where the oracle has it."""
    tb, tree = _tree(4, T)
    g = torch.Generator().manual_seed(11)
    shared, lens, page, Hkv, G = 64, [130, 300, 64], 16, 2, 4
    t, n_pages = table(g, 3, 300 - shared + T + 40, page, shared)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D)
    q = torch.randn(3, T, Hkv * G, D, generator=g).to(torch.bfloat16)
    clean, _ = want_of(q, kp, vp, t, lens, tb["mask"])
    mask = torch.tensor(tb["mask"], dtype=torch.bool)
    at = lambda b, s: (int(t[b, s // page]), s % page)  # noqa: E731
    bad_v = {} if T == 1 else {0: (min(5, T - 1), float("nan")), 1: (T - 1, float("inf")), 2: (T // 2, float("-inf"))}
    for b, L in enumerate(lens):
        for s in range(L + T, L + T + 30):       # behind the last node
            pg, r = at(b, s)
            kp[pg, :, r] = vp[pg, :, r] = float("nan")
        if b in bad_v:
            pg, r = at(b, L + bad_v[b][0])
            vp[pg, 1, r, 3::7] = bad_v[b][1]
    if T > 1:                                    # a K row of NaN: every row that sees it is NaN
        pg, r = at(0, lens[0] + T - 2)
        kp[pg, 0, r] = float("nan")
    out = run(tree, q, kp, vp, t, lens, shared).double()
    for b in range(3):
        want = clean[b].clone()
        if b in bad_v:
            a, x = bad_v[b]
            want[mask[:, a], G:, 3::7] = x
        if b == 0 and T > 1:
            want[mask[:, T - 2], :G] = float("nan")
        fine = torch.isfinite(want)
        assert torch.equal(torch.isnan(out[b]), torch.isnan(want)) and torch.equal(torch.isinf(out[b]), torch.isinf(want))
        assert torch.equal(out[b][torch.isinf(want)], want[torch.isinf(want)])
        assert (out[b][fine] - want[fine]).abs().max().item() <= 2e-2


@pytest.mark.parametrize("T", [64, 3])
@pytest.mark.parametrize("where", ["q", "k", "k_inf"])
def test_non_finite_scores(where, T):
    """A NaN in a query row makes that row NaN; a NaN or an infinity in a prefix key every row of its head that has a finite query."""
    tb, tree = _tree(4, T)
    g = torch.Generator().manual_seed(13)
    shared, lens, page, Hkv, G, D = 128, [400, 200], 16, 2, 4, 128
    for col in (0, 6, 12, 13, 14, 15, 70, 127):              # columns of either exponential
        t, n_pages = table(g, 2, 400 - shared + T, page, shared)
        kp, vp = pools(g, 2, n_pages, Hkv, page, D)
        q = torch.randn(2, T, Hkv * G, D, generator=g).to(torch.bfloat16)
        want = torch.zeros(2, T, Hkv * G, dtype=torch.bool)
        if where == "q":
            q[1, T - 2, 5, col] = float("nan")
            want[1, T - 2, 5] = True
        else:
            s = 128 + 128 + col if where == "k" else 128 + col      # sequence 0 alone, second or first own tile
            pg, r = int(t[0, s // page]), s % page
            kp[pg, 1, r, 17] = float("nan") if where == "k" else float("inf")
            q[..., 17] = 1.0                                  # +inf scores
            want[0, :, G:] = True
        out = run(tree, q, kp, vp, t, lens, shared)
        assert torch.equal(torch.isnan(out).all(-1), want) and torch.equal(torch.isnan(out).any(-1), want), col


def sequences_of(t, n_pages, page, Hkv, D, lens, shared, T, Hq, seed=21):
    g = torch.Generator().manual_seed(seed)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D)
    return kp, vp, torch.randn(len(lens), T, Hq, D, generator=g).to(torch.bfloat16)


@pytest.mark.parametrize("T,Hq,Hkv,D,page,shared,lens", [
    (64, 32, 8, 128, 64, 256, [256, 383, 900]), (29, 8, 2, 64, 16, 48, [700, 49]), (1, 8, 2, 128, 16, 32, [33, 32, 400]), (4, 4, 1, 64, 16, 0, [77]),
])
def test_pages_with_the_heads_inside(T, Hq, Hkv, D, page, shared, lens):
    tb, tree = _tree(4, T)
    check(tree, tb, Hq, Hkv, D, page, shared, lens, tokens_outside=True)
    check(tree, tb, Hq, Hkv, D, page, shared, lens, scale=0.3)


@pytest.mark.parametrize("T,G", [(64, 4), (20, 3), (1, 4), (4, 4)])
@pytest.mark.parametrize("D", [64, 128])
def test_sequences_that_cannot_be(D, T, G):
    """Lengths that do not fit or end inside the prefix: out stays as it was.  A page that is not there: BOUNDS, and the other sequences have
    what they would have alone.  Table entries behind the last slot are never followed."""
    tb, tree = _tree(4, T)
    page, shared, Hkv = 16, 64, 2
    lens = [130, 63, -1, 300, 400, 210, 416 - T, 417 - T]
    g = torch.Generator().manual_seed(5)
    t, n_pages = table(g, len(lens), 416 - shared, page, shared)
    kp, vp, q = sequences_of(t, n_pages, page, Hkv, D, lens, shared, T, Hkv * G)
    assert t.shape[1] * page == 416
    bad = t.clone()
    bad[3, 100 // page] = n_pages
    bad[0, -(-(130 + T) // page):] = -1
    bad[5, (210 + T - 1) // page] = -3
    status = torch.full((len(lens),), 5, dtype=torch.int32, device=DEV)
    out = run(tree, q, kp, vp, bad, lens, shared, status=status)
    cap = -6
    assert status.tolist() == [0, cap, cap, -7, cap if 400 + T > 416 else 0, -7, 0, cap]
    ok = [b for b in range(len(lens)) if status[b] == 0]
    want, absolute = want_of(q[ok], kp, vp, t[ok], [lens[b] for b in ok], tb["mask"])
    assert ((out[ok].double() - want).abs() / bound(want, absolute)).max().item() <= 1.0
    for b in range(len(lens)):
        if status[b] == cap:
            assert (out[b] == 7.0).all()
    bad = t.clone()
    bad[0, 1] = n_pages + 5                      # a page of the prefix: it is missing for all
    run(tree, q, kp, vp, bad, lens, shared, status=status)
    assert all(s in (-7, cap) for s in status.tolist()[:1])


@pytest.mark.parametrize("T", [64, 1])
def test_two_streams_and_a_graph(T):
    """Calls with workspaces of their own on two streams at once, and two graphs over one workspace replayed in turn, with other lengths and
    pages than at their capture."""
    tb, tree = _tree(4, T)
    Hq, Hkv, D, page, shared = 16, 4, 128, 16, 96
    lens = [[96, 500, 1000], [700, 97, 333]]
    g = torch.Generator().manual_seed(5)
    t, n_pages = table(g, 3, 1000 + T - shared, page, shared)
    kp, vp, q = sequences_of(t, n_pages, page, Hkv, D, lens[0], shared, T, Hq)
    kd, vd, td, qd = kp.to(DEV), vp.to(DEV), t.to(DEV), [q.to(DEV), q.flip(0).to(DEV)]
    ld = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in lens]
    n = binding.paged_workspace_bytes(tree, 3, Hq, Hkv, D, shared)
    ws = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [torch.zeros_like(x) for x in qd]
    want = [want_of(x.cpu(), kp, vp, t, ls, tb["mask"]) for x, ls in zip(qd, lens)]

    def right(order=(0, 1)):
        torch.cuda.synchronize()
        for i, j in enumerate(order):
            assert ((outs[i].cpu().double() - want[j][0]).abs() / bound(*want[j])).max().item() <= 1.0
    call = lambda i, w, stream=None: binding.tree_verify_attention_paged(tree, qd[i], kd, vd, td, ld[i], outs[i], ws[w], shared_len=shared, stream=stream)  # noqa: E731
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for i in range(2):
            call(i, i, streams[i])
    right()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=streams[0]):
            call(i, 0, streams[0])
    ws[0].fill_(0xff)
    for swapped in (False, True):
        if swapped:
            ld[0].copy_(torch.tensor(lens[1])), ld[1].copy_(torch.tensor(lens[0]))
            a, b = qd[0].clone(), qd[1].clone()
            qd[0].copy_(b), qd[1].copy_(a)
        for o in outs:
            o.fill_(9.0)
        for _ in range(3):
            graphs[0].replay()
            graphs[1].replay()
        right((1, 0) if swapped else (0, 1))
    assert binding.mtv_device_error(tree) == 0


def test_refusals():
    tb, tree = _tree(4, 20)
    page, Hkv, Hq, D, lens = 16, 2, 4, 64, [70, 80]
    g = torch.Generator().manual_seed(5)
    t, n_pages = table(g, 2, 100, page)
    kp, vp, q = (x.to(DEV) for x in sequences_of(t, n_pages, page, Hkv, D, lens, 0, 20, Hq))
    td, ld, out = t.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), torch.full_like(q, 7.0)
    n = binding.paged_workspace_bytes(tree, 2, Hq, Hkv, D)
    ws = torch.zeros(n + 512, dtype=torch.uint8, device=DEV)
    ws = ws[-ws.data_ptr() % 256:]

    def code(q=q, out=out, ws=ws[:n], shared=0, scale=0.0):
        with pytest.raises(binding.MtvError) as e:
            binding.tree_verify_attention_paged(tree, q, kp, vp, td, ld, out, ws, shared_len=shared, scale=scale)
        return e.value.code
    assert code(ws=ws[:n - 1]) == -3 and code(ws=ws[16:n + 16]) in (-1, -3)
    assert code(shared=8) == -1 and code(shared=-16) == -1 and code(shared=16 * (t.shape[1] + 1)) == -1
    for s in (-1.0, float("nan"), float("inf")):
        assert code(scale=s) == -1
    off = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device=DEV)[1:1 + q.numel()].view(q.shape)
    assert code(q=off) == -1 and code(out=off) == -1
    wide = torch.zeros(2, 20, 5, D, dtype=torch.bfloat16, device=DEV)
    assert code(q=wide, out=torch.zeros_like(wide)) in (-1, -2)
    torch.cuda.synchronize()
    assert (out == 7.0).all() and binding.mtv_device_error(tree) == 0


@pytest.mark.parametrize("K,T,Hq,Hkv,D,page,shared,lens", [
    (1, 1, 8, 1, 64, 16, 0, [3, 9, 40, 700]),             # at most 16 rows a KV head, of a sequence and of all behind the prefix
    (1, 1, 16, 2, 128, 64, 0, [3, 9, 40, 700]),
    (1, 1, 16, 4, 128, 64, 128, [130, 128, 900]),
    (2, 2, 8, 1, 128, 16, 0, [0, 5, 14, 63, 500]),
    (3, 4, 16, 4, 64, 32, 32, [32, 47, 333]),
    (3, 29, 8, 2, 64, 16, 0, [128, 5]),                   # row tiles of head size 64
    (4, 64, 32, 8, 64, 32, 256, [256, 383, 900]),
    (4, 64, 32, 8, 64, 32, 4096, [4100, 5000]),
    (4, 65, 6, 1, 64, 128, 384, [384, 400]),
    (5, 128, 16, 2, 64, 32, 0, [5, 3000]),
    (1, 1, 32, 8, 64, 64, 1024, [1024 + 17 * i for i in range(40)]),
])
def test_weights_in_two_terms(K, T, Hq, Hkv, D, page, shared, lens):
    """Where weights have two bf16 terms their own rounding stays out of the result: two bf16 terms leave at most 2^-16 of a weight.  The exponentials are good to 7.5e-5,
    above and below the fraction, the scores as in bound(); beside them there is the output's rounding alone."""
    tb, tree = _tree(K, T)
    g = torch.Generator().manual_seed(23)
    B = len(lens)
    t, n_pages = table(g, B, max(lens) - shared + T, page, shared)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D)
    q = torch.randn(B, T, Hq, D, generator=g).to(torch.bfloat16)
    out = run(tree, q, kp, vp, t, lens, shared)
    want, absolute = want_of(q, kp, vp, t, lens, tb["mask"])
    most = EPS * want.abs() + (1 + EPS) * (2.0 ** -16 + 2 * 7.5e-5 + 1e-4) * absolute + 1e-30
    worst = ((out.double() - want).abs() / most).max().item()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("T", [3, 20, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_large_values_of_nodes_that_are_not_seen(D, T):
    """The largest finite V rows in every leaf, the leaves in every column of a tile: they reach the leaves alone."""
    tb, tree = _tree(4, T)
    g = torch.Generator().manual_seed(17)
    mask = torch.tensor(tb["mask"], dtype=torch.bool)
    leaf = mask.sum(0) == 1                                # nobody else sees it
    shared, page, Hkv, G = 64, 16, 2, 8
    lens = [64 + i for i in range(16)] + [190 + 16 * i for i in range(8)]
    t, n_pages = table(g, len(lens), max(lens) - shared + T, page, shared)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D)
    q = torch.randn(len(lens), T, Hkv * G, D, generator=g).to(torch.bfloat16)
    want, absolute = want_of(q, kp, vp, t, lens, tb["mask"])
    for b, L in enumerate(lens):
        for i in leaf.nonzero()[:, 0].tolist():
            vp[int(t[b, (L + i) // page]), :, (L + i) % page] = torch.finfo(torch.bfloat16).max * (-1) ** (i + b)
    out = run(tree, q, kp, vp, t, lens, shared)
    assert ((out.double() - want).abs() / bound(want, absolute))[:, ~leaf].max().item() <= 1.0


@pytest.mark.parametrize("T,G", [(1, 4), (20, 8), (64, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_that_vanish(D, T, G):
    """A visible key whose score is 300 below the others' (a weight of 2^-430) adds nothing, whatever its V row and its column."""
    tb, tree = _tree(4, T)
    g = torch.Generator().manual_seed(19)
    shared, page, Hkv = 0, 16, 2
    lens = [300 + i for i in range(16)]
    t, n_pages = table(g, len(lens), max(lens) + T, page, shared)
    kp, vp = pools(g, 2, n_pages, Hkv, page, D)
    kp[..., 0] = 0
    q = torch.randn(len(lens), T, Hkv * G, D, generator=g).to(torch.bfloat16)
    q[..., 0] = 16.0
    clean = vp.clone()
    for b, L in enumerate(lens):
        for s in (5 + b, 130 + b, L - 1):
            pg, r = int(t[b, s // page]), s % page
            kp[pg, :, r, 0] = -300.0 * D ** 0.5 / 16
            clean[pg, :, r], vp[pg, :, r] = 0.0, torch.finfo(torch.bfloat16).max
    want, absolute = want_of(q, kp, clean, t, lens, tb["mask"])
    out = run(tree, q, kp, vp, t, lens, shared)
    assert ((out.double() - want).abs() / bound(want, absolute)).max().item() <= 1.0
