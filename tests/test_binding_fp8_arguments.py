"""What the wrappers of the calls on caches in 8 bits refuse by the tensors themselves, each by its argument's name, before an address goes to the
library.  On the host the good call is refused last, as one that is on no CUDA device."""
import pytest
import torch

from paper_2603_03383_b200 import binding, build
from tests import test_binding_arguments as other
from tests.test_binding_arguments import B, BF16, D, HKV, HQ, I32, LAYERS, N_PAGES, NOT_HERE, PAGE, T, bf, i32, refused

FP8 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.fixture(scope="module")
def tree():
    return binding.tree_build_static(3, binding.tree_gen_rank_prior(3, T), upload=False)


def codes(*n):
    return torch.zeros(n, dtype=torch.uint8).view(FP8)


def scales():
    return dict(k_scale=torch.ones(LAYERS, HKV), v_scale=torch.ones(LAYERS, HKV))


def cache():
    return dict(other.cache(), pool=binding.pool_layout(codes(N_PAGES, HKV, PAGE, D)))


def append_args():
    return dict(other.append_args(), **cache(), **scales())


def rows_args():
    return dict(other.rows_args(), **cache(), **scales())


def compact_args():
    return dict(other.compact_args(), **cache())


def read_args():
    c = cache()
    c["first"] = c.pop("seq_lens")
    return dict(c, **scales(), row_starts=i32(B + 1), k_out_layers=bf(LAYERS, 7, HKV, D), v_out_layers=bf(LAYERS, 7, HKV, D))


def attend_args():
    return dict(other.attend_args(), k_pool=codes(N_PAGES, HKV, PAGE, D), v_pool=codes(N_PAGES, HKV, PAGE, D), k_scale=torch.ones(HKV), v_scale=torch.ones(HKV))


CALLS = [(append_args, "tree_kv_append_rope_paged_fp8", True), (rows_args, "kv_append_rope_paged_fp8", False),
         (compact_args, "kv_compact_accepted_paged_fp8", True), (read_args, "kv_read_paged_fp8", False)]


@pytest.mark.parametrize("make,wrapper,of_tree", CALLS)
def test_appends_reading_and_compaction(tree, make, wrapper, of_tree):
    def call(**a):
        getattr(binding, wrapper)(*((tree,) if of_tree else ()), **a)
    assert NOT_HERE in refused(call, make())
    assert NOT_HERE in refused(call, dict(make(), status=None))
    for name, good in make().items():
        if not isinstance(good, torch.Tensor):
            continue
        for bad in other.wrong(name, good):
            if name in ("q_layers", "k_out_layers") and bad.dtype is BF16 and bad.shape[-1] < D:      # (then it is others that do not fit)
                continue
            if name == "page_table" and bad.is_contiguous() and bad.dtype is I32:
                continue                                    # (a table of fewer pages is a table)
            assert name in refused(call, dict(make(), **{name: bad})), (name, bad.dtype, bad.shape)
        if name not in ("status", "first"):
            with pytest.raises((binding.MtvError, AttributeError)):
                call(**dict(make(), **{name: None}))
    half = binding.pool_layout(bf(N_PAGES, HKV, PAGE, D))
    assert "pool" in refused(call, dict(make(), pool=half))


def test_reading_other_sizes():
    a = read_args()
    assert NOT_HERE in refused(binding.kv_read_paged_fp8, dict(a, first=None))
    assert NOT_HERE in refused(binding.kv_read_paged_fp8, dict(a, k_out_layers=a["k_out_layers"][:, :0], v_out_layers=a["v_out_layers"][:, :0]))
    assert "v_out_layers" in refused(binding.kv_read_paged_fp8, dict(a, v_out_layers=a["v_out_layers"][:, :6].contiguous()))
    assert "k_out_layers" in refused(binding.kv_read_paged_fp8, dict(a, k_out_layers=a["k_out_layers"][0]))
    assert "k_scale" in refused(binding.kv_read_paged_fp8, dict(a, k_scale=torch.ones(LAYERS * HKV - 1)))


def test_attention(tree):
    def call(**a):
        binding.tree_verify_attention_paged_fp8(tree, **a)
    assert NOT_HERE in refused(call, attend_args())
    for name, good in attend_args().items():
        bads = [bf(*good.shape), good.view(torch.uint8), good[..., :-1].contiguous()] if good.dtype is FP8 else other.wrong(name, good)
        for bad in bads:
            if name == "ws" and bad.is_contiguous() or name == "page_table" and bad.is_contiguous() and bad.dtype is I32:
                continue                                    # (the library looks at its size)
            if name == "q" and bad.dtype is BF16 and bad.shape[-1] < D:
                continue
            assert any(n in refused(call, dict(attend_args(), **{name: bad})) for n in ([name, "v_pool"] if name == "k_pool" else [name])), (name, bad.dtype)
    a = attend_args()
    assert "v_pool" in refused(call, dict(a, v_pool=codes(N_PAGES - 1, HKV, PAGE, D)))
    assert "v_pool" in refused(call, dict(a, v_pool=codes(N_PAGES, PAGE, HKV, D).transpose(1, 2)))
    assert "k_scale" in refused(call, dict(a, k_scale=None)) and "v_scale" in refused(call, dict(a, v_scale=None))


def test_bf16_calls_want_bf16_layouts(tree):
    pool = binding.pool_layout(codes(N_PAGES, HKV, PAGE, D))
    for make, wrapper, lead in ((other.append_args, binding.tree_kv_append_rope_paged, (tree,)), (other.rows_args, binding.kv_append_rope_paged, ()),
                                (other.compact_args, binding.kv_compact_accepted_paged, (tree,))):
        with pytest.raises(binding.MtvError) as e:
            wrapper(*lead, **dict(make(), pool=pool))
        assert e.value.code == -1 and "pool" in str(e.value)
    assert "k_pool" in refused(binding.tree_verify_attention_paged, dict(other.attend_args(), tree=tree, k_pool=codes(N_PAGES, HKV, PAGE, D)))
    for bad in (codes(N_PAGES, HKV, PAGE, D).view(torch.uint8), codes(N_PAGES, HKV, PAGE, 2 * D)[..., ::2], codes(HKV, PAGE, D)):
        with pytest.raises(binding.MtvError):
            binding.pool_layout(bad)


@pytest.mark.gpu
def test_one_tensor_on_the_host(tree):
    """Among tensors of the device, any one that is not there; it is refused before anything is launched."""
    on = lambda a: {k: x.to("cuda") if isinstance(x, torch.Tensor) else x for k, x in a.items()}  # noqa: E731
    for make, name_of, of_tree in CALLS + [(attend_args, "tree_verify_attention_paged_fp8", True)]:
        f = getattr(binding, name_of)
        for name, x in make().items():
            if isinstance(x, torch.Tensor):
                with pytest.raises(binding.MtvError) as e:
                    f(*((tree,) if of_tree else ()), **dict(on(make()), **{name: x}))
                assert e.value.code == -1 and f.__name__ in str(e.value)
