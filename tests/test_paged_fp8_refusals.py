"""What the calls on caches in 8 bits refuse, before they touch a device."""
import pytest

from paper_2603_03383_b200 import binding, build
from tests.test_paged_refusals import BAD_POOLS, INVALID, P, SHAPE, layout

BAD_POOLS = BAD_POOLS + [(dict(stride_t=72), INVALID), (dict(stride_h=1032), INVALID), (dict(stride_page=4104), INVALID)]     # multiples of 8 alone


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.fixture(scope="module")
def tree():
    return binding.tree_build_static(3, binding.tree_gen_rank_prior(3, 20), upload=False)


def rows(**kw):
    a = dict(B=2, n_rows=5, Hq=4, Hkv=2, D=64, n_layers=1, q=P, q_out=P, k=P, v=P, kp=P, vp=P, pool=layout(), table=P, max_pages=4, lens=P, starts=P, ks=P, vs=P,
             theta=0.0)
    a.update(kw)
    return binding.lib().kv_append_rope_paged_fp8(a["B"], a["n_rows"], a["Hq"], a["Hkv"], a["D"], a["n_layers"], a["q"], a["q_out"], a["k"], a["v"],
                                                  a["kp"], a["vp"], a["pool"], a["table"], a["max_pages"], a["lens"], a["starts"], a["ks"], a["vs"],
                                                  a["theta"], None, 0)


def read(**kw):
    a = dict(B=2, n_rows=5, Hkv=2, D=64, n_layers=1, kp=P, vp=P, pool=layout(), table=P, max_pages=4, first=P, starts=P, ks=P, vs=P, k=P, v=P)
    a.update(kw)
    return binding.lib().kv_read_paged_fp8(a["B"], a["n_rows"], a["Hkv"], a["D"], a["n_layers"], a["kp"], a["vp"], a["pool"], a["table"], a["max_pages"],
                                           a["first"], a["starts"], a["ks"], a["vs"], a["k"], a["v"], None, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(kp=None), INVALID),
    (dict(vp=None), INVALID), (dict(pool=None), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(starts=None), INVALID),
    (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(B=0), INVALID), (dict(n_rows=-1), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID),
    (dict(n_layers=0), INVALID), (dict(max_pages=0), INVALID), (dict(theta=-1.0), INVALID), (dict(theta=float("nan")), INVALID),
    (dict(theta=float("inf")), INVALID), (dict(D=96), SHAPE), (dict(D=256), SHAPE), (dict(n_layers=65536), SHAPE), (dict(n_rows=(1 << 30) + 1), SHAPE),
    (dict(max_pages=(1 << 27)), SHAPE), (dict(Hq=1 << 20), SHAPE), (dict(Hkv=1 << 20), SHAPE),
] + [(dict(pool=layout(**kw)), code) for kw, code in BAD_POOLS])
def test_ragged_append(kw, code):
    assert rows(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(kp=None), INVALID), (dict(vp=None), INVALID), (dict(pool=None), INVALID), (dict(table=None), INVALID), (dict(starts=None), INVALID),
    (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=P + 8), INVALID), (dict(v=P + 2), INVALID),
    (dict(B=0), INVALID), (dict(n_rows=-1), INVALID), (dict(Hkv=0), INVALID), (dict(n_layers=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(n_rows=0, k=None, v=None, ks=None), INVALID), (dict(D=96), SHAPE), (dict(n_layers=65536), SHAPE), (dict(n_rows=(1 << 30) + 1), SHAPE),
    (dict(max_pages=(1 << 27)), SHAPE), (dict(Hkv=1 << 20), SHAPE), (dict(n_rows=0, k=None, v=None, D=32), SHAPE),
] + [(dict(pool=layout(**kw)), code) for kw, code in BAD_POOLS])
def test_reading(kw, code):
    assert read(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(n_layers=0), INVALID), (dict(kp=None), INVALID), (dict(vp=None), INVALID),
    (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(new=None), INVALID), (dict(n=None), INVALID), (dict(nodes=None), INVALID),
    (dict(pool=None), INVALID), (dict(max_pages=0), INVALID), (dict(h=None), INVALID), (dict(D=32), SHAPE), (dict(B=65536), SHAPE),
    (dict(Hkv=1 << 20), SHAPE),
] + [(dict(pool=layout(**kw)), code) for kw, code in BAD_POOLS])
def test_compaction(tree, kw, code):
    a = dict(h=tree.handle, B=2, Hkv=2, D=64, n_layers=1, kp=P, vp=P, pool=layout(), table=P, max_pages=4, lens=P, new=P, n=P, nodes=P)
    a.update(kw)
    assert binding.lib().kv_compact_accepted_paged_fp8(a["h"], a["B"], a["Hkv"], a["D"], a["n_layers"], a["kp"], a["vp"], a["pool"], a["table"],
                                                       a["max_pages"], a["lens"], a["new"], a["n"], a["nodes"], None, 0) == code


def test_a_tree_that_is_not_on_a_device(tree):
    L = binding.lib()
    for h in (tree.handle, None):
        assert L.tree_kv_append_rope_paged_fp8(h, 2, 4, 2, 64, 1, P, P, P, P, P, P, layout(), P, 4, P, P, P, 0.0, None, 0) == INVALID
        assert L.tree_verify_attention_paged_fp8(h, 2, 4, 2, 64, P, P, P, layout(), P, 4, 0, P, P, P, 0.0, P, None, P, 1 << 30, 0) == INVALID
