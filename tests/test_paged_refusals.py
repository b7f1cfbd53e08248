"""What the calls on paged caches and constrained logits refuse, before they touch a device."""
import pytest
import torch

from paper_2603_03383_b200 import binding, build

INVALID, SHAPE, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


P = 4096                        # an address that is aligned and never followed


def layout(stride_page=4096, stride_h=1024, stride_t=64, page_size=16, n_pages=9):
    return binding.PoolLayout(stride_page, stride_h, stride_t, page_size, n_pages)


BAD_POOLS = [
    (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(page_size=0), SHAPE),
    (dict(n_pages=0), INVALID), (dict(stride_t=56), INVALID), (dict(stride_t=68), INVALID), (dict(stride_h=1020), INVALID),
    (dict(stride_page=4100), INVALID), (dict(stride_page=-4096), INVALID), (dict(stride_h=0), INVALID),
]


def rows(**kw):
    a = dict(B=2, n_rows=5, Hq=4, Hkv=2, D=64, n_layers=1, q=P, q_out=P, k=P, v=P, kp=P, vp=P, pool=layout(), table=P, max_pages=4, lens=P, starts=P,
             theta=0.0)
    a.update(kw)
    return binding.lib().kv_append_rope_paged(a["B"], a["n_rows"], a["Hq"], a["Hkv"], a["D"], a["n_layers"], a["q"], a["q_out"], a["k"], a["v"],
                                              a["kp"], a["vp"], a["pool"], a["table"], a["max_pages"], a["lens"], a["starts"], a["theta"], None, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(kp=None), INVALID),
    (dict(vp=None), INVALID), (dict(pool=None), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(starts=None), INVALID),
    (dict(B=0), INVALID), (dict(B=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID),
    (dict(n_layers=0), INVALID), (dict(max_pages=0), INVALID), (dict(theta=-1.0), INVALID), (dict(theta=float("nan")), INVALID),
    (dict(D=96), SHAPE), (dict(D=256), SHAPE), (dict(n_layers=65536), SHAPE), (dict(n_rows=(1 << 30) + 1), SHAPE),
    (dict(max_pages=(1 << 27)), SHAPE), (dict(theta=float("inf")), INVALID), (dict(Hq=1 << 20), SHAPE), (dict(Hkv=1 << 20), SHAPE),
])
def test_ragged_append(kw, code):
    assert rows(**kw) == code


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_pools(kw, code):
    assert rows(pool=layout(**kw)) == code


def test_a_tree_that_is_not_on_a_device():
    tree = binding.tree_build_static(3, binding.tree_gen_rank_prior(3, 20), upload=False)
    L, h, r = binding.lib(), tree.handle, binding.LogitRules()
    assert L.tree_kv_append_rope_paged(h, 2, 4, 2, 64, 1, P, P, P, P, P, P, layout(), P, 4, P, 0.0, None, 0) == INVALID
    assert L.tree_verify_attention_paged(h, 2, 4, 2, 64, P, P, P, layout(), P, 4, 0, P, 0.0, P, None, P, 1 << 30, 0) == INVALID
    assert L.logits_constrain(h, 2, 100, 0, P, 100, P, 100, r, None, 0) == INVALID
    assert L.constrained_argmax_keys(h, 2, 100, 0, P, 100, r, None, P, 0) == INVALID
    assert L.tree_kv_append_rope_paged(None, 2, 4, 2, 64, 1, P, P, P, P, P, P, layout(), P, 4, P, 0.0, None, 0) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(n_layers=0), INVALID), (dict(kp=None), INVALID), (dict(vp=None), INVALID),
    (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(new=None), INVALID), (dict(n=None), INVALID), (dict(nodes=None), INVALID),
    (dict(pool=None), INVALID), (dict(max_pages=0), INVALID), (dict(tree=None), INVALID), (dict(D=32), SHAPE), (dict(B=65536), SHAPE),
    (dict(Hkv=1 << 20), SHAPE),
] + [(dict(pool=layout(**kw)), code) for kw, code in BAD_POOLS])
def test_compaction(kw, code):
    tree = binding.tree_build_static(3, binding.tree_gen_rank_prior(3, 20), upload=False)
    a = dict(tree=tree.handle, B=2, Hkv=2, D=64, n_layers=1, kp=P, vp=P, pool=layout(), table=P, max_pages=4, lens=P, new=P, n=P, nodes=P)
    a.update(kw)
    assert binding.lib().kv_compact_accepted_paged(a["tree"], a["B"], a["Hkv"], a["D"], a["n_layers"], a["kp"], a["vp"], a["pool"], a["table"],
                                                   a["max_pages"], a["lens"], a["new"], a["n"], a["nodes"], None, 0) == code


@pytest.mark.parametrize("B,V,n,tokens,counts,seen,code", [
    (0, 10, 1, P, P, P, INVALID), (1, 0, 1, P, P, P, INVALID), (1, 10, -1, P, P, P, INVALID), (1, 10, 1, None, P, P, INVALID),
    (1, 10, 1, P, None, P, INVALID), (1, 10, 1, P, P, None, INVALID), (65536, 10, 1, P, P, P, SHAPE), (1, 10, 0, None, P, P, 0),
])
def test_counts(B, V, n, tokens, counts, seen, code):
    assert binding.lib().token_counts_add(B, V, n, tokens, None, 0, counts, seen, 0) == code


@pytest.mark.parametrize("B,Hq,Hkv,D,shared", [(0, 4, 2, 64, 0), (1025, 4, 2, 64, 0), (2, 5, 2, 64, 0), (2, 4, 2, 96, 0), (2, 4, 2, 64, -16), (2, 0, 2, 64, 0)])
def test_workspaces_of_sizes_that_are_refused(B, Hq, Hkv, D, shared):
    tree = binding.tree_build_static(3, binding.tree_gen_rank_prior(3, 20), upload=False)
    assert binding.paged_workspace_bytes(tree, B, Hq, Hkv, D, shared) == 0


def test_layouts_that_the_wrappers_refuse():
    tree = binding.tree_build_static(3, binding.tree_gen_rank_prior(3, 20), upload=False)
    x, r = torch.zeros(2, 20, 64, dtype=torch.bfloat16), binding.logit_rules()
    for y in (x.transpose(1, 2).contiguous().transpose(1, 2), x[:, ::1].repeat(1, 2, 1)[:, :20], x.half(), torch.zeros(2, 20, 128, dtype=torch.bfloat16)[..., ::2]):
        with pytest.raises(binding.MtvError):
            binding._logit_rows(y, "constrained_argmax_keys")
    with pytest.raises(binding.MtvError):
        binding.logits_constrain(tree, x, x.float(), r)
    with pytest.raises(binding.MtvError):
        binding.logits_constrain(tree, x, torch.zeros(2, 20, 65, dtype=torch.bfloat16), r)
    pool = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    for p in (pool[..., ::2], pool.half(), pool[0]):
        with pytest.raises((binding.MtvError, AssertionError)):
            binding.pool_layout(p)


def test_rows_without_an_address():
    """Only a call without rows may leave their pointers out; what else it lacks is refused before a device is touched."""
    none = dict(q=None, q_out=None, k=None, v=None)
    assert rows(**none) == INVALID and rows(n_rows=1, **none) == INVALID
    for kw in (dict(kp=None), dict(table=None), dict(lens=None), dict(starts=None), dict(B=0), dict(D=96), dict(theta=-1.0)):
        assert rows(n_rows=0, **none, **kw) in (INVALID, SHAPE)
        assert rows(n_rows=0, **kw) == rows(n_rows=0, **none, **kw)
