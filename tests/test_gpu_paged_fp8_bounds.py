"""What the header says that the attention over codes loses: of small weights 2^-33 of a row's largest, of small values of a query row of a row tile 2^-17 of its largest."""
import math

import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _fp8
from tests._cases import make_tree
from tests._paged import table

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 2.0 ** -8


def tree_of(T):
    return (dict(mask=[[1]]), binding.tree_build_static(1, [])) if T == 1 else make_tree("rank_prior", 4, (), T)


def run(tree, q, kp, vp, ks, vs, t, lens, shared=0, scale=0.0):
    B, T, Hq, D = q.shape
    ws = torch.full((binding.paged_workspace_bytes(tree, B, Hq, kp.shape[1], D, shared),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    move = lambda p: p.view(torch.uint8).to(DEV).view(_fp8.FP8)  # noqa: E731
    binding.tree_verify_attention_paged_fp8(tree, q.to(DEV), move(kp), move(vp), t.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out, ws,
                                            ks.to(DEV), vs.to(DEV), shared_len=shared, scale=scale)
    torch.cuda.synchronize()
    assert binding.mtv_device_error(tree) == 0
    return out.cpu().double()


@pytest.mark.parametrize("T,G", [(1, 4), (4, 4), (20, 3), (64, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shared", [0, 64])
def test_small_weights(D, T, G, shared):
    """Keys of weight 2^-30 to 2^-36 among many of weight 1, each with a column of V of its own.  In front of the bound, as everywhere: the output's rounding, 2^-11 of
    a weight, an exponential off by at most 7.5e-5 in it and in the sum, a score of 36 off by 2^-22 of itself."""
    tb, tree = tree_of(T)
    Hkv, page, lens = 2, 16, [700, 300]
    t, n_pages = table(torch.Generator().manual_seed(4), 2, max(lens) - shared + T, page, shared)
    kp, vp = (torch.zeros(n_pages, Hkv, page, D).to(_fp8.FP8) for _ in range(2))
    ks, vs = torch.ones(Hkv), torch.ones(Hkv)
    q = torch.zeros(2, T, Hkv * G, D, dtype=torch.bfloat16)
    q[..., :4] = 1.0
    for b, L in enumerate(lens):
        for i in range(48):
            s = shared + (17 * i + 5) % (L - shared)
            pg, r = int(t[b, s // page]), s % page
            for c, x in enumerate((16.0, 14.0, i // 8, i % 8 / 8)):
                _fp8.put(kp, (pg, slice(None), r, c), -x)
            _fp8.put(vp, (pg, slice(None), r, i), 448.0)
    out = run(tree, q, kp, vp, ks, vs, t, lens, shared, math.log(2.0))
    want, _ = _fp8.attention(q, kp, vp, ks, vs, t, lens, tb["mask"], math.log(2.0))
    largest = 1.0 / (torch.tensor(lens).double()[:, None, None, None] - 48)            # of a row's weights, at most: all others are as large
    bound = EPS * want + (1 + EPS) * ((2.0 ** -11 + 2 * 7.5e-5 + 36 * 2.0 ** -22) * want + 2.0 ** -33 * 448.0 * largest)
    worst = ((out - want).abs() / bound)[..., :48].max().item()
    assert worst <= 1.0, worst
    assert (out[..., 48:] == 0).all()


@pytest.mark.parametrize("T,G", [(20, 3), (64, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [-9, -11, -13, -15])
def test_small_values_of_a_query_row(D, T, G, power):
    """One value of a row is far above the rest and meets zeros in K: the scores are the small values' alone, of which each is off by 2^-17 of the largest at most."""
    tb, tree = tree_of(T)
    Hkv, page, lens = 2, 16, [300, 77]
    g = torch.Generator().manual_seed(5)
    t, n_pages = table(g, 2, max(lens) + T, page)
    kp, vp = _fp8.pools(g, 2, n_pages, Hkv, page, D)
    kp.view(torch.uint8)[..., 7] = 0
    ks, vs = torch.tensor([0.01, 0.012]), torch.tensor([0.01, 0.012])
    small = (torch.randn(2, T, Hkv * G, D, generator=g).clamp(-2.5, 2.5) * 2.0 ** power).to(torch.bfloat16)
    q = small.clone()
    q[..., 7] = -3.0
    scale = 2.0 ** (-power) / D ** 0.5
    out = run(tree, q, kp, vp, ks, vs, t, lens, 0, scale)
    want, absolute = _fp8.attention(q, kp, vp, ks, vs, t, lens, tb["mask"], scale)
    # a score is off by at most 2^-17 * 3 * scale * k_scale * sum |K8| = d; a weight by a factor of e^d, and so is their sum
    size = _fp8.values(kp, ks).abs().sum(-1).max().item()
    d = 2.0 ** -17 * 3.0 * scale * size
    bound = EPS * want.abs() + (1 + EPS) * (2.0 ** -11 + 2 * 7.5e-5 + 1e-4 + math.expm1(2 * d)) * absolute
    worst = ((out - want).abs() / bound).max().item()
    assert worst <= 1.0, worst
