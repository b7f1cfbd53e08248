"""Status of the paged attention of either cache where pages of the shared prefix are missing: every sequence of the batch says so, except those that cannot be at all."""
import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _fp8, _paged
from tests._cases import make_tree

pytestmark = pytest.mark.gpu
DEV = "cuda"
CAPACITY, BOUNDS = -6, -7


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D,T,G", [(64, 64, 4), (128, 20, 3), (128, 1, 4), (64, 4, 4)])
@pytest.mark.parametrize("missing", ["first", "last", "negative", "far"])
def test_a_missing_page_of_the_prefix_is_missing_for_all(codes, D, T, G, missing):
    tree = binding.tree_build_static(1, []) if T == 1 else make_tree("rank_prior", 4, (), T)[1]
    page, shared, Hkv = 16, 64, 2
    lens = [130, 63, -1, 300, 400, 210, 416 - T, 417 - T, 64, 2 ** 31 - 1]
    g = torch.Generator().manual_seed(5)
    t, n_pages = _paged.table(g, len(lens), 416 - shared, page, shared)
    q = torch.randn(len(lens), T, Hkv * G, D, generator=g).to(torch.bfloat16).to(DEV)
    ws = torch.full((binding.paged_workspace_bytes(tree, len(lens), Hkv * G, Hkv, D, shared),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, 7.0)
    scales = torch.full((Hkv,), 0.01, device=DEV)
    if codes:
        kp, vp = (x.view(torch.uint8).to(DEV).view(_fp8.FP8) for x in _fp8.pools(g, 2, n_pages, Hkv, page, D))
    else:
        kp, vp = (x.to(DEV) for x in _paged.pools(g, 2, n_pages, Hkv, page, D))

    def status_of(t):
        status = torch.full((len(lens),), 5, dtype=torch.int32, device=DEV)
        args = (tree, q, kp, vp, t.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out, ws)
        if codes:
            binding.tree_verify_attention_paged_fp8(*args, scales, scales, shared_len=shared, status=status)
        else:
            binding.tree_verify_attention_paged(*args, shared_len=shared, status=status)
        assert binding.mtv_device_error(tree) == 0
        return status.tolist()
    fits = [shared <= L and L + T <= 416 for L in lens]
    assert status_of(t) == [0 if f else CAPACITY for f in fits]
    bad = t.clone()
    at = {"first": 0, "last": shared // page - 1}.get(missing, 1)
    bad[:, at] = {"negative": -1, "far": 2 ** 31 - 1}.get(missing, n_pages)
    assert status_of(bad) == [BOUNDS if f else CAPACITY for f in fits]
    torch.cuda.synchronize()
    for b, f in enumerate(fits):
        assert f or (out[b] == 7.0).all()
    # an own page is missing for its sequence alone
    bad = t.clone()
    bad[3, 100 // page] = n_pages
    assert status_of(bad) == [CAPACITY if not f else BOUNDS if b == 3 else 0 for b, f in enumerate(fits)]
