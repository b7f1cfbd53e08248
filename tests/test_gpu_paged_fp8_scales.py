"""Scales of the 8-bit cache over the whole range of fp32, its subnormal numbers too.

A code stands next to the value over the scale: half a step, which is 2^-4 of its power of two, or 2^-10 at the smallest.  In front of it 1 / scale (which has at
least 21 bits) and the product with it are off by 2^-21 of the value at most, together less than 2^-20."""
import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _fp8
from tests._cases import make_tree
from tests._paged import table

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, U8 = torch.bfloat16, torch.uint8
SCALES = [2.0 ** -149, 3 * 2.0 ** -149, 1.37 * 2.0 ** -140, 2.0 ** -133, 1.9 * 2.0 ** -130, 2.0 ** -129, 2.0 ** -128, 1.01 * 2.0 ** -128, 1.99 * 2.0 ** -127, 2.0 ** -126,
          1.3 * 2.0 ** -100, 1.0, 1.7 * 2.0 ** 90, 2.0 ** 118, 1.9 * 2.0 ** 126, 1.99 * 2.0 ** 127]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def append(k, v, ks, vs, page, layers, Hkv, D, tree=None):
    """Rows k, v [n][Hkv][D] of one sequence at the front of its pages (rows at position 0 are not rotated) -> codes [n][Hkv][D] of either."""
    n, n_pages = k.shape[0], -(-k.shape[0] // page)
    kp, vp = (torch.zeros(n_pages, Hkv, page, D, dtype=U8, device=DEV) for _ in range(2))
    q = torch.zeros(layers, n, Hkv, D, dtype=BF16, device=DEV)
    t = torch.arange(n_pages, dtype=torch.int32, device=DEV)[None]
    args = (q, torch.zeros_like(q), k[None].to(DEV), v[None].to(DEV), binding.cache_pointer_array([kp], DEV), binding.cache_pointer_array([vp], DEV),
            binding.pool_layout(kp.view(_fp8.FP8)), t)
    ks, vs = (x[None].to(DEV) for x in (ks, vs))
    if tree is None:
        binding.kv_append_rope_paged_fp8(*args, i32([0]), i32([0, n]), ks, vs)
    else:
        binding.tree_kv_append_rope_paged_fp8(tree, *(x.unsqueeze(1) for x in args[:4]), *args[4:], i32([0]), ks, vs)
    return [x.cpu().transpose(1, 2).reshape(-1, Hkv, D)[:n].view(_fp8.FP8).float().double() for x in (kp, vp)]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("whole_tree", [False, True])
def test_codes(scale, D, whole_tree):
    """Values around the scale, and beyond what its codes reach; zeros are the code of zero whatever the scale."""
    g = torch.Generator().manual_seed(2)
    Hkv, n = 2, 1 if whole_tree else 5
    s = torch.tensor([scale, 0.75], dtype=torch.float32)
    assert s[0].double() == torch.tensor(scale, dtype=torch.float64).float().double() > 0
    tree = binding.tree_build_static(1, []) if whole_tree else None

    def some():
        x = torch.randn(n, Hkv, D, generator=g, dtype=torch.float64) * 2.0 ** torch.randint(-11, 12, (n, Hkv, D), generator=g).double()
        x = (x * s.double()[:, None]).clamp(-3e38, 3e38).float().to(BF16)
        x[..., ::7] = 0.0
        x[..., 3::7] = -0.0
        return x
    k, v = some(), some()
    v[0, :, 5], v[0, :, 6], v[0, :, 8], v[0, :, 9] = float("inf"), float("-inf"), 3e38, -3e38
    v[0, :, 11] = float("nan")
    kc, vc = append(k, v, s, s, 16, 1, Hkv, D, tree)
    for x, c, first in ((k, kc, 1), (v, vc, n)):
        # (keys behind position 0 are rotated: their zeros are not zeros any more)
        y = (x.double() / s.double()[:, None])[:first]
        c = c[:first]
        assert torch.equal(torch.isnan(c), torch.isnan(y))
        y = y.clamp(-_fp8.MAX, _fp8.MAX)
        step = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        ok = (c - y).abs() <= step / 2 + 2.0 ** -20 * y.abs()
        assert (ok | torch.isnan(y)).all(), (x[:first][~ok & ~torch.isnan(y)][:4], c[~ok & ~torch.isnan(y)][:4])
    assert not torch.isnan(kc).any()


def attend(tree, q, kp, vp, ks, vs, t, lens, scale):
    B, T, Hq, D = q.shape
    ws = torch.full((binding.paged_workspace_bytes(tree, B, Hq, kp.shape[1], D),), 0xff, dtype=U8, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=BF16, device=DEV)
    move = lambda p: p.view(U8).to(DEV).view(_fp8.FP8)  # noqa: E731
    binding.tree_verify_attention_paged_fp8(tree, q.to(DEV), move(kp), move(vp), t.to(DEV), i32(lens), out, ws, ks.to(DEV), vs.to(DEV), scale=scale)
    torch.cuda.synchronize()
    assert binding.mtv_device_error(tree) == 0
    return out.cpu().double()


def bound(want, absolute):
    """As for other scales: the output's rounding, weights in fp16 and their exponentials (in the weights and in their sum), fp32 sums."""
    return 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (2.0 ** -11 + 2 * 7.5e-5 + 1e-4) * absolute


@pytest.mark.parametrize("T,G", [(1, 4), (4, 4), (20, 3), (64, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("large", [False, True])
def test_scores_whose_scales_have_no_product(D, T, G, large):
    """scale * k_scale is below fp32's normal numbers, or beyond its largest; with the queries, which make up for it, the scores are ordinary."""
    g = torch.Generator().manual_seed(6)
    Hkv, page, lens = 2, 16, [300, 77]
    tb, tree = (dict(mask=[[1]]), binding.tree_build_static(1, [])) if T == 1 else make_tree("rank_prior", 4, (), T)
    t, n_pages = table(g, len(lens), max(lens) + T, page)
    kp, vp = _fp8.pools(g, 2, n_pages, Hkv, page, D)
    vs = torch.tensor([0.01, 0.02])
    if large:
        q = (torch.randn(2, T, Hkv * G, D, generator=g) * 2.0 ** -66).mul(2.0 ** -64).to(BF16)       # a few steps of the smallest bf16
        kp = (kp.float() / 1600).to(_fp8.FP8)
        ks, scale = torch.tensor([2.0 ** 110, 1.5 * 2.0 ** 110]), 2.0 ** 20
    else:
        # keys of +-448 along or against the queries; V has the sign of a key's score, so that a factor that is off shows at first order
        sign = torch.where(torch.rand(n_pages, Hkv, page, 1, generator=g) < 0.5, -1.0, 1.0)
        kp = (448.0 * sign).expand(n_pages, Hkv, page, D).contiguous().to(_fp8.FP8)
        vp = (100.0 * sign).expand(n_pages, Hkv, page, D).contiguous().to(_fp8.FP8)
        q = torch.full((2, T, Hkv * G, D), 1.9921875 * 2.0 ** 127).to(BF16)
        ks, scale = torch.tensor([2.0 ** -100, 1.25 * 2.0 ** -100]), 1.0625 / 1.4426950408889634 * 2.0 ** -46
    out = attend(tree, q, kp, vp, ks, vs, t, lens, scale)
    want, absolute = _fp8.attention(q, kp, vp, ks, vs, t, lens, tb["mask"], scale)
    assert want.isfinite().all()
    worst = ((out - want).abs() / bound(want, absolute)).max().item()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("T,G", [(1, 4), (4, 4), (20, 3), (64, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("of_v", [False, True])
def test_a_scale_that_is_no_number_shows(D, T, G, of_v):
    """NaN as a head's scale: that head's rows are NaN, the other's as ever."""
    g = torch.Generator().manual_seed(6)
    Hkv, page, lens = 2, 16, [300, 77]
    tb, tree = (dict(mask=[[1]]), binding.tree_build_static(1, [])) if T == 1 else make_tree("rank_prior", 4, (), T)
    t, n_pages = table(g, len(lens), max(lens) + T, page)
    kp, vp = _fp8.pools(g, 2, n_pages, Hkv, page, D)
    q = torch.randn(2, T, Hkv * G, D, generator=g).to(BF16)
    ks, vs = torch.tensor([0.01, 0.012]), torch.tensor([0.01, 0.012])
    want, absolute = _fp8.attention(q, kp, vp, ks, vs, t, lens, tb["mask"])
    (vs if of_v else ks)[0] = float("nan")
    out = attend(tree, q, kp, vp, ks, vs, t, lens, 0.0)
    assert torch.isnan(out[:, :, :G]).all()
    assert ((out - want).abs() / bound(want, absolute))[:, :, G:].max().item() <= 1.0
