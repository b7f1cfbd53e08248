"""Scores far from zero, where fp32 holds their differences to whole steps alone: keys whose scores differ by a few steps weigh as in 64 bits, and no weight is beyond fp16."""
import math

import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _fp8
from tests._cases import make_tree
from tests._paged import table

pytestmark = pytest.mark.gpu
DEV = "cuda"


# (in row tiles a query row's values are held to 2^-17 of its largest: no differences beside scores beyond 2^11 there)
@pytest.mark.parametrize("T,G,power", [(T, G, p) for T, G in ((1, 4), (1, 8), (4, 4)) for p in (0, 16, 20, 21, 22, 24, 26)] + [(T, G, p) for T, G in ((20, 3), (64, 4)) for p in (0, 8, 11)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_differences_of_large_scores(D, T, G, power, sign):
    """Scores (of base 2) sign * 2^power + d: every one is a number of fp32 with two bits to spare, as are the products and sums that it comes from, so that only the
    weights' rounding is left (2^-11 and 7.5e-5 of a weight, in the sum too) and the output's.  d grows along the keys by up to 8 at a time, in steps of that size."""
    tb, tree = (dict(mask=[[1]]), binding.tree_build_static(1, [])) if T == 1 else make_tree("rank_prior", 4, (), T)
    Hkv, page, lens = 8, 16, [1500 - 3 * i for i in range(8)]          # several blocks of keys a warp, whatever the division
    g = torch.Generator().manual_seed(4)
    t, n_pages = table(g, len(lens), max(lens) + T, page)
    kp = torch.zeros(n_pages, Hkv, page, D)
    vp = _fp8.pools(g, 1, n_pages, Hkv, page, D)[0]
    step = max(0.25, 2.0 ** (power - 21))
    q = torch.zeros(len(lens), T, Hkv * G, D, dtype=torch.bfloat16)
    q[..., 0], q[..., 1], q[..., 2], q[..., 3] = 2.0 ** (power - 4), step, 64 * step, step
    kp[..., 0] = 16.0 * sign
    d, steps = 0, []
    for run, up in ((37, 8.0), (150, 7.75), (5, 8.0), (130, 7.5), (64, 8.0), (300, 1.0), (16, 8.0), (10000, 8.0)):
        steps += [d] * run
        d += max(1, int(up / step))
    for b, L in enumerate(lens):
        i = torch.arange(L + T)
        pg, r, d = t[b, i // page].long(), i % page, torch.tensor(steps)[i]
        kp[pg, :, r, 1], kp[pg, :, r, 2], kp[pg, :, r, 3] = ((d % 64 // 4 * 4)[:, None].float(), (d // 64)[:, None].float(), (d % 4)[:, None].float())
    kp = kp.to(_fp8.FP8)
    ks, vs = torch.ones(Hkv), torch.full((Hkv,), 0.01)
    ws = torch.full((binding.paged_workspace_bytes(tree, len(lens), Hkv * G, Hkv, D),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    move = lambda p: p.view(torch.uint8).to(DEV).view(_fp8.FP8)  # noqa: E731
    scale = math.log(2.0)
    binding.tree_verify_attention_paged_fp8(tree, q.to(DEV), move(kp), move(vp), t.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out, ws,
                                            ks.to(DEV), vs.to(DEV), scale=scale)
    torch.cuda.synchronize()
    assert binding.mtv_device_error(tree) == 0
    want, absolute = _fp8.attention(q, kp, vp, ks, vs, t, lens, tb["mask"], scale)
    out = out.cpu().double()
    assert not torch.isnan(out).any()
    bound = 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (2.0 ** -11 + 2 * 7.5e-5 + 1e-4) * absolute
    worst = ((out - want).abs() / bound).max().item()
    assert worst <= 1.0, worst
