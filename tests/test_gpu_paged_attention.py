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
])
def test_against_the_oracle(K, T, Hq, Hkv, D, page, shared, lens):
    tb, tree = make_tree("rank_prior", K, (), T) if T > 1 else make_tree("cartesian", 1, (1,))
    if T == 1:
        tree = binding.tree_build_static(1, [])
        tb = dict(mask=[[1]])
    check(tree, tb, Hq, Hkv, D, page, shared, lens)
