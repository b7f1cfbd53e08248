"""What the wrappers of the paged and constrained calls refuse by the tensors themselves, each by its argument's name, before an address
goes to the library.  On the host the good call is refused last, as one that is on no CUDA device."""
import pytest
import torch

from paper_2603_03383_b200 import binding, build

BF16, I32, I64 = torch.bfloat16, torch.int32, torch.int64
B, T, HQ, HKV, D, PAGE, N_PAGES, LAYERS, V, WORDS = 2, 20, 4, 2, 64, 16, 9, 3, 100, 4
NOT_HERE = "not on the current CUDA device"


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.fixture(scope="module")
def tree():
    return binding.tree_build_static(3, binding.tree_gen_rank_prior(3, T), upload=False)


def i32(*n):
    return torch.zeros(n, dtype=I32)


def bf(*n):
    return torch.zeros(n, dtype=BF16)


def apart(t):
    """The same sizes and values, not contiguous."""
    return t.repeat_interleave(2, -1)[..., ::2]


def refused(f, args):
    with pytest.raises(binding.MtvError) as e:
        f(**args)
    assert e.value.code == -1
    return str(e.value)


def cache():
    k = bf(N_PAGES, HKV, PAGE, D)
    return dict(k_ptrs=torch.zeros(LAYERS, dtype=I64), v_ptrs=torch.zeros(LAYERS, dtype=I64), pool=binding.pool_layout(k), page_table=i32(B, 4),
                seq_lens=i32(B), status=i32(B))


def append_args():
    q, k = (LAYERS, B, T, HQ, D), (LAYERS, B, T, HKV, D)
    return dict(q_layers=bf(*q), q_out_layers=bf(*q), k_new_layers=bf(*k), v_new_layers=bf(*k), **cache())


def rows_args():
    q, k = (LAYERS, 7, HQ, D), (LAYERS, 7, HKV, D)
    return dict(q_layers=bf(*q), q_out_layers=bf(*q), k_new_layers=bf(*k), v_new_layers=bf(*k), row_starts=i32(B + 1), **cache())


def compact_args():
    return dict(n_layers=LAYERS, Hkv=HKV, D=D, new_lens=i32(B), accept_len=i32(B), acc_nodes=i32(B, 4), **cache())


def attend_args():
    k = bf(N_PAGES, HKV, PAGE, D)
    return dict(q=bf(B, T, HQ, D), k_pool=k, v_pool=k.clone(), page_table=i32(B, 4), seq_lens=i32(B), out=bf(B, T, HQ, D),
                ws=torch.zeros(64, dtype=torch.uint8), status=i32(B))


def wrong(name, t):
    """Versions of an argument that a kernel would misread."""
    out = [t.to(I64 if t.dtype is not I64 else I32), t.to(torch.float16)]
    if t.dim():
        out += [t[..., :-1].contiguous()]
        if t.shape[-1] > 1:
            out += [apart(t), t[..., :1].expand(t.shape)]
    return out


@pytest.mark.parametrize("make,wrapper,of_tree", [(append_args, "tree_kv_append_rope_paged", True), (rows_args, "kv_append_rope_paged", False),
                                                  (compact_args, "kv_compact_accepted_paged", True)])
def test_appends_and_compaction(tree, make, wrapper, of_tree):
    def call(**a):
        getattr(binding, wrapper)(*((tree,) if of_tree else ()), **a)
    assert NOT_HERE in refused(call, make())
    assert NOT_HERE in refused(call, dict(make(), status=None))
    for name, good in make().items():
        if not isinstance(good, torch.Tensor):
            continue
        for bad in wrong(name, good):
            if name == "q_layers" and bad.dtype is BF16 and bad.shape[-1] < D:      # (then it is the keys that do not fit)
                continue
            if name == "page_table" and bad.is_contiguous() and bad.dtype is I32:
                continue                                    # (a table of fewer pages is a table)
            assert name in refused(call, dict(make(), **{name: bad})), (name, bad.dtype, bad.shape)
        if name != "status":
            with pytest.raises((binding.MtvError, AttributeError)):
                call(**dict(make(), **{name: None}))


def test_nodes_and_sequences_that_do_not_fit(tree):
    def call(**a):
        binding.tree_kv_append_rope_paged(tree, **a)
    a = append_args()
    short = {n: a[n][:, :, :T - 1].contiguous() for n in ("q_layers", "q_out_layers", "k_new_layers", "v_new_layers")}
    assert "q_layers" in refused(call, dict(a, **short))
    assert "page_table" in refused(call, dict(a, page_table=i32(B - 1, 4))) and "page_table" in refused(call, dict(a, page_table=i32(4)))
    assert NOT_HERE in refused(call, dict(a, page_table=i32(B + 3, 4), seq_lens=i32(B + 3), status=i32(B + 1)))     # buffers of a larger batch
    assert "row_starts" in refused(binding.kv_append_rope_paged, dict(rows_args(), row_starts=i32(B)))
    assert NOT_HERE in refused(binding.kv_append_rope_paged, {n: x[:, :0] if n[1:2] == "_" and "layers" in n else x for n, x in rows_args().items()})


def test_attention(tree):
    def call(**a):
        binding.tree_verify_attention_paged(tree, **a)
    assert NOT_HERE in refused(call, attend_args())
    for name, good in attend_args().items():
        for bad in wrong(name, good):
            if name == "ws" and bad.is_contiguous() or name == "page_table" and bad.is_contiguous() and bad.dtype is I32:
                continue                                    # (the library looks at its size)
            if name == "q" and bad.dtype is BF16 and bad.shape[-1] < D:
                continue
            assert any(n in refused(call, dict(attend_args(), **{name: bad})) for n in ([name, "v_pool"] if name == "k_pool" else [name])), (name, bad.dtype)
    a = attend_args()
    assert "q" in refused(call, dict(a, q=bf(B, T - 1, HQ, D), out=bf(B, T - 1, HQ, D)))
    assert "out" in refused(call, dict(a, out=bf(B * T, HQ, 1, D))) and "out" in refused(call, dict(a, out=bf(B, T, HQ // 2, 2 * D)))
    assert "v_pool" in refused(call, dict(a, v_pool=bf(N_PAGES - 1, HKV, PAGE, D)))
    assert "v_pool" in refused(call, dict(a, v_pool=bf(N_PAGES, PAGE, HKV, D).transpose(1, 2)))
    assert "k_pool" in refused(call, dict(a, k_pool=bf(N_PAGES, HKV, PAGE, 2 * D), v_pool=bf(N_PAGES, HKV, PAGE, 2 * D)))


def rules_args():
    return dict(counts=i32(B, V), seen=i32(B, WORDS), repetition=torch.ones(B), presence=torch.zeros(B), frequency=torch.zeros(B), bias_ids=i32(B, 5),
                bias=torch.zeros(B, 5), mask=i32(6, WORDS), mask_of=i32(B, T))


def test_rules():
    assert binding.logit_rules().n_bias == 0 and binding.logit_rules(**rules_args()).n_masks == 6
    for name, good in rules_args().items():
        bads = [good.double(), good.to(I64)] + ([apart(good)] if good.shape[-1] > 1 else []) + [good[None]]
        for bad in bads:
            assert name in refused(binding.logit_rules, {name: bad} if name not in ("bias", "bias_ids") else dict(rules_args(), **{name: bad}))
    for name, bad in (("seen", i32(B, WORDS - 1)), ("mask", i32(6, WORDS - 1)), ("bias", torch.zeros(B, 4))):
        assert "logit_rules" in refused(binding.logit_rules, dict(rules_args(), **{name: bad}))
    assert "bias" in refused(binding.logit_rules, dict(bias_ids=i32(B, 5)))


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_constrained(tree, dtype):
    x, keys, tok = torch.zeros(B, T, V, dtype=dtype), torch.zeros(B * T, dtype=I64), i32(B, T)

    def write(rules, x=x, out=x, tok=tok):
        return refused(binding.logits_constrain, dict(tree=tree, logits=x, out=out, rules=rules, tree_tok=tok))

    def top(rules, x=x, keys=keys, tok=tok):
        return refused(binding.constrained_argmax_keys, dict(tree=tree, logits=x, keys=keys, rules=rules, tree_tok=tok))
    fine = binding.logit_rules(**rules_args())
    for f in (write, top):
        for rules in (fine, binding.logit_rules(), binding.LogitRules()):
            assert NOT_HERE in f(rules) and NOT_HERE in f(rules, tok=None)
        for bad in (tok.to(I64), tok[:1], apart(tok), tok.float()):
            assert "tree_tok" in f(fine, tok=bad)
        for kw in (dict(counts=i32(B, V + 1), seen=i32(B, WORDS)), dict(seen=i32(B, WORDS + 1)), dict(mask=i32(6, WORDS - 1)), dict(mask_of=i32(B, T - 1)),
                   dict(counts=i32(B - 1, V)), dict(repetition=torch.ones(B - 1)), dict(bias_ids=i32(1, 5), bias=torch.zeros(1, 5))):
            assert "rules" in f(binding.logit_rules(**kw)), list(kw)
        assert NOT_HERE in f(binding.logit_rules(counts=i32(B + 2, V), seen=i32(B + 2, WORDS), presence=torch.zeros(B + 1)))
        assert "logits" in f(fine, x=torch.zeros(B, T + 1, V, dtype=dtype), **({"out": torch.zeros(B, T + 1, V, dtype=dtype)} if f is write else {}))
    for bad in (keys[:-1], keys.int(), keys.repeat_interleave(2)[::2], keys.double()):
        assert "keys" in top(fine, keys=bad)
    assert NOT_HERE in top(fine, keys=torch.zeros(B * T + 9, dtype=I64))
    for bad in (x.half(), x[:1], x.transpose(1, 2), torch.zeros(B, T, V + 1, dtype=dtype)):
        assert "logits_constrain" in write(fine, out=bad)


def test_counts():
    def call(**kw):
        a = dict(tokens=i32(B, 6), counts=i32(B, V), seen=i32(B, WORDS), lens=i32(B))
        return refused(binding.token_counts_add, dict(a, **kw))
    assert NOT_HERE in call() and NOT_HERE in call(lens=None) and NOT_HERE in call(tokens=i32(B, 0))
    for name, bads in (("tokens", [i32(B, 6).to(I64), apart(i32(B, 6)), i32(6)]), ("lens", [i32(B - 1), i32(B).to(I64)]),
                       ("counts", [i32(B - 1, V), i32(B, V).to(I64), i32(V)]), ("seen", [i32(B, WORDS - 1), i32(B, WORDS).to(I64)])):
        for bad in bads:
            assert name in call(**{name: bad}), (name, bad.shape)


def test_the_look_at_tensors_itself():
    look = binding._look
    with pytest.raises(TypeError):
        look("f", ("a",), i32(1), 1)
    with pytest.raises(RuntimeError):            # no storage to take an address of
        look("f", ("a",), torch.nn.parameter.UninitializedBuffer(dtype=I32), 1, 0)
    for bad in (7, "x", None, torch.zeros(2, 2).to_sparse().to(I32), torch.zeros(2, dtype=I32, device="meta")):
        with pytest.raises(binding.MtvError) as e:
            look("f", ("a", "b"), i32(2), 1, 2, bad, 1, 1)
        assert "f: b" in str(e.value)


@pytest.mark.gpu
def test_one_tensor_on_the_host(tree):
    """Among tensors of the device, any one that is not there; it is refused before anything is launched."""
    on = lambda a: {k: x.to("cuda") if isinstance(x, torch.Tensor) else x for k, x in a.items()}  # noqa: E731
    for f, make, lead in ((binding.tree_kv_append_rope_paged, append_args, (tree,)), (binding.kv_append_rope_paged, rows_args, ()),
                          (binding.kv_compact_accepted_paged, compact_args, (tree,)), (binding.tree_verify_attention_paged, attend_args, (tree,))):
        for name, x in make().items():
            if isinstance(x, torch.Tensor):
                with pytest.raises(binding.MtvError) as e:
                    f(*lead, **dict(on(make()), **{name: x}))
                assert e.value.code == -1 and f.__name__ in str(e.value)
    assert "several devices" in refused(binding.logit_rules, dict(on(rules_args()), seen=i32(B, WORDS)))
    x = torch.zeros(B, T, V, device="cuda")
    assert "rules" in refused(binding.logits_constrain, dict(tree=tree, logits=x, out=x, rules=binding.logit_rules(**rules_args())))
    assert "out" in refused(binding.logits_constrain, dict(tree=tree, logits=x, out=x.cpu(), rules=binding.logit_rules()))
