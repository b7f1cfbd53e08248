"""Scales of the 8-bit cache over the whole range of fp32, its subnormal numbers too.

A code stands next to the value over the scale: half a step, which is 2^-4 of its power of two, or 2^-10 at the smallest.  In front of it 1 / scale (which has at
least 21 bits) and the product with it are off by 2^-21 of the value at most, together less than 2^-20."""
import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _fp8

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
