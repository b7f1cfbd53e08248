"""Constrained logits and their argmax, to the bit against the formula in fp32 one operation at a time, and within its roundings of the
formula in 64 bits."""
import pytest
import torch

from paper_2603_03383_b200 import binding
from tests import _rules
from tests._cases import make_tree

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
INF, NAN = float("inf"), float("nan")


def paths_of(tb):
    mask = torch.as_tensor(tb["mask"]).bool()
    return [[j for j in range(tb["T"]) if mask[i, j]] for i in range(tb["T"])]


def on_device(r):
    d = {k: None if v is None else v.to(DEV) for k, v in r.items() if k != "allowed"}
    return binding.logit_rules(**d)


def rows(x, offset, gap):
    """A copy of x [B][T][V] on the device whose rows begin at element `offset` of the buffer and are V + gap apart; what lies between holds 7."""
    B, T, V = x.shape
    buf = torch.full((offset + B * T * (V + gap),), 7.0, dtype=x.dtype, device=DEV)
    view = buf[offset:].view(B, T, V + gap)[:, :, :V]
    view.copy_(x)
    return buf, view


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == BF16 else torch.int32)


def case(K, T, B, V, dtype, hist, n_bias, n_masks, penalties=True, seed=3):
    g = torch.Generator().manual_seed(seed)
    tb, tree = make_tree("cartesian", K, (1,) * K) if T == K + 1 else make_tree("rank_prior", K, T=T)
    assert tree.T == T
    x = (2 * torch.randn(B, T, V, generator=g)).to(dtype)
    r = _rules.rules(g, B, T, V, hist, n_bias, n_masks, penalties)
    tok = torch.randint(0, min(V, 50), (B, T), generator=g).to(torch.int32)       # often the same token twice on a path
    tok[0, 0] = V - 1
    return tb, tree, x, r, tok, paths_of(tb)


CASES = [
    # K, T, B, V, dtype, hist, n_bias, n_masks, offset, gap
    (1, 1, 1, 1, BF16, 1, 1, 1, 0, 0),
    (1, 1, 3, 31, torch.float32, 5, 2, 2, 1, 0),
    (3, 29, 2, 1000, BF16, 60, 7, 3, 0, 0),
    (3, 29, 2, 1025, BF16, 60, 7, 3, 3, 5),                 # rows at every alignment
    (3, 29, 2, 1027, torch.float32, 2000, 30, 3, 1, 2),
    (4, 64, 1, 4099, BF16, 30, 0, 0, 0, 0),
    (4, 64, 3, 2048, torch.float32, 0, 300, 5, 0, 8),
    (5, 128, 2, 5003, BF16, 9000, 11, 9, 0, 8),             # nearly every token of a unit counted
    (2, 6, 40, 2049, BF16, 100, 3, 4, 8, 0),
    (8, 9, 2, 33333, BF16, 500, 4096, 2, 0, 0),
    (2, 4, 1, 700, BF16, 50, 4096, 2, 0, 0),                # every token biased, several times
    (1, 1, 1, 150000, torch.float32, 500, 40, 2, 0, 0),
]


@pytest.mark.parametrize("K,T,B,V,dtype,hist,n_bias,n_masks,offset,gap", CASES)
@pytest.mark.parametrize("in_place", [False, True])
def test_written_logits(K, T, B, V, dtype, hist, n_bias, n_masks, offset, gap, in_place):
    tb, tree, x, r, tok, paths = case(K, T, B, V, dtype, hist, n_bias, n_masks)
    _, view = rows(x, offset, gap)
    buf, out = (_, view) if in_place else rows(torch.zeros_like(x), offset + 1, gap + 3)
    binding.logits_constrain(tree, view, out, on_device(r), tok.to(DEV))
    want, _ = _rules.constrained(x, r, tok, paths, torch.float32)
    same = torch.equal(bits(out.cpu() + 0.0), bits(want.to(dtype) + 0.0))
    assert same
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert (buf[outside] == 7.0).all()
    exact, err = _rules.constrained(x, r, tok, paths, torch.float64)
    got = out.cpu().double()
    assert torch.equal(got == -INF, exact == -INF)
    half = torch.finfo(dtype).eps / 2 if dtype == BF16 else 0.0
    live = exact > -INF
    assert ((got - exact).abs() <= half * (exact.abs() + err) + err)[live].all()
    assert binding.mtv_device_error(tree) == 0


@pytest.mark.parametrize("K,T,B,V,dtype,hist,n_bias,n_masks,offset,gap", CASES)
def test_argmax_keys(K, T, B, V, dtype, hist, n_bias, n_masks, offset, gap):
    tb, tree, x, r, tok, paths = case(K, T, B, V, dtype, hist, n_bias, n_masks)
    _, view = rows(x, offset, gap)
    keys = torch.full((B * tree.T,), 77, dtype=torch.int64, device=DEV)
    binding.constrained_argmax_keys(tree, view, keys, on_device(r), tok.to(DEV))
    want, _ = _rules.constrained(x, r, tok, paths, torch.float32)
    key, at, top = _rules.keys_of(want)
    nothing = top == -INF
    assert torch.equal(keys.cpu(), torch.where(nothing, 0, key))
    if n_masks:
        assert nothing[0] or B * T == 1          # (a single row has the last row's mask)
    # the chosen token is the best one, up to the roundings, in 64 bits too
    exact, err = (y.view(-1, V) for y in _rules.constrained(x, r, tok, paths, torch.float64))
    for i in (~nothing).nonzero()[:, 0].tolist():
        assert exact[i, at[i]] + err[i, at[i]] >= (exact[i] - err[i]).max()


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("V", [40, 2100])
def test_parts_left_out(dtype, V):
    tb, tree, x, r, tok, paths = case(3, 20, 2, V, dtype, 50, 5, 3)
    for left_out in (["counts", "seen"], ["repetition"], ["presence", "frequency"], ["bias_ids", "bias"], ["mask", "mask_of"], list(r)):
        for t in (tok, None):
            some = {k: None if k in left_out else v for k, v in r.items()}
            want, _ = _rules.constrained(x, some, t, paths, torch.float32)
            out = torch.empty_like(x, device=DEV)
            keys = torch.empty(x.shape[0] * x.shape[1], dtype=torch.int64, device=DEV)
            t = None if t is None else t.to(DEV)
            binding.logits_constrain(tree, x.to(DEV), out, on_device(some), t)
            binding.constrained_argmax_keys(tree, x.to(DEV), keys, on_device(some), t)
            assert torch.equal(bits(out.cpu() + 0.0), bits(want.to(dtype) + 0.0)), left_out
            key, _, top = _rules.keys_of(want)
            assert torch.equal(keys.cpu(), torch.where(top == -INF, 0, key)), left_out


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_nan_and_infinities(dtype):
    V = 1100
    tb, tree = make_tree("rank_prior", 2, T=8)
    g = torch.Generator().manual_seed(9)
    x = torch.randn(1, 8, V, generator=g).to(dtype)
    x[0, 0, 3] = NAN                                    # never chosen
    x[0, 1, 5], x[0, 1, 900] = INF, INF                 # the lowest token of two
    x[0, 2] = -INF                                      # allowed, but all -inf: the lowest token
    x[0, 3] = -INF
    x[0, 3, 1050] = NAN
    x[0, 4] = NAN                                       # nothing left
    x[0, 5, ::2] = INF                                  # infinities and NaN in masked places
    x[0, 5, 11] = NAN
    x[0, 6, 7], x[0, 6, 8] = -0.0, 0.0                  # both zeros are one value
    x[0, 6, 9:], x[0, 6, :7] = -1, -1
    x[0, 7] = torch.finfo(dtype).min                    # the type's lowest value is a value
    r = dict.fromkeys(["counts", "seen", "repetition", "presence", "frequency", "bias_ids", "bias", "mask", "mask_of", "allowed"])
    allowed = torch.zeros(2, V, dtype=torch.bool)
    allowed[0, 1::2] = True
    allowed[0, 11] = False
    allowed[1, 20:] = True
    r.update(allowed=allowed, mask=_rules.packed(allowed), mask_of=torch.tensor([[-1, -1, -1, 1, -1, 0, -1, 1]], dtype=torch.int32))
    keys = torch.empty(8, dtype=torch.int64, device=DEV)
    binding.constrained_argmax_keys(tree, x.to(DEV), keys, on_device(r))
    want, _ = _rules.constrained(x, r, None, paths_of(tb), torch.float32)
    key, at, top = _rules.keys_of(want)
    key[3] = (0x007fffff << 32) + (0xffffffff - 20)     # (the image of -inf; the lowest token that is allowed)
    key[4] = 0
    assert torch.equal(keys.cpu(), key)
    out = torch.empty_like(x, device=DEV)
    binding.logits_constrain(tree, x.to(DEV), out, on_device(r))
    out = out.cpu()
    assert torch.equal(out.isnan(), want.isnan())
    assert torch.equal(out.nan_to_num(5), want.to(dtype).nan_to_num(5))


def test_a_mask_that_does_not_exist():
    tb, tree, x, r, tok, paths = case(3, 20, 2, 300, BF16, 50, 5, 3)
    r["mask_of"][1, 4] = 3
    keys = torch.empty(2 * 20, dtype=torch.int64, device=DEV)
    binding.constrained_argmax_keys(tree, x.to(DEV), keys, on_device(r), tok.to(DEV))
    assert binding.mtv_device_error(tree) == -7
    r["mask_of"][1, 4] = -1
    want, _ = _rules.constrained(x, r, tok, paths, torch.float32)
    key, _, top = _rules.keys_of(want)
    assert torch.equal(keys.cpu(), torch.where(top == -INF, 0, key))


def test_rows_far_apart():
    """Row offsets beyond 2^31 elements."""
    V, stride = 1500, (1 << 30) + 1
    tb, tree, x, r, tok, paths = case(2, 4, 1, V, BF16, 50, 5, 2)
    T = tree.T
    buf = torch.empty((T - 1) * stride + V, dtype=BF16, device=DEV)
    view = buf.as_strided((1, T, V), (T * stride, stride, 1))
    view.copy_(x)
    keys = torch.empty(T, dtype=torch.int64, device=DEV)
    binding.constrained_argmax_keys(tree, view, keys, on_device(r), tok.to(DEV))
    binding.logits_constrain(tree, view, view, on_device(r), tok.to(DEV))
    want, _ = _rules.constrained(x, r, tok, paths, torch.float32)
    key, _, top = _rules.keys_of(want)
    assert torch.equal(keys.cpu(), torch.where(top == -INF, 0, key))
    assert torch.equal(bits(view.cpu() + 0.0), bits(want.to(BF16) + 0.0))


def test_captured_and_replayed():
    tb, tree, x, r, tok, paths = case(3, 29, 2, 3000, BF16, 60, 7, 3)
    view, t, rules = x.to(DEV), tok.to(DEV), on_device(r)
    keys = torch.empty(2 * tree.T, dtype=torch.int64, device=DEV)
    binding.constrained_argmax_keys(tree, view, keys, rules, t)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        binding.constrained_argmax_keys(tree, view, keys, rules, t)
    for seed in (4, 5):
        y = torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)).to(BF16)
        view.copy_(y)
        keys.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = _rules.constrained(y, r, tok, paths, torch.float32)
        key, _, top = _rules.keys_of(want)
        assert torch.equal(keys.cpu(), torch.where(top == -INF, 0, key))


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("B,V,n", [(1, 1, 1), (3, 33, 7), (2, 1000, 700)])
def test_counts(B, V, n, prompt):
    g = torch.Generator().manual_seed(n)
    tokens = torch.randint(-2, V + 2, (B, n), generator=g).to(torch.int32)
    lens = torch.randint(-1, n + 3, (B,), generator=g).to(torch.int32)
    counts = torch.zeros(B, V, dtype=torch.int32, device=DEV)
    seen = torch.zeros(B, -(-V // 32), dtype=torch.int32, device=DEV)
    want = torch.zeros(B, V, dtype=torch.int64)
    for ls in (None, lens, lens):
        binding.token_counts_add(tokens.to(DEV), counts, seen, None if ls is None else ls.to(DEV), prompt)
        for b in range(B):
            for v in tokens[b, :n if ls is None else max(0, min(n, int(ls[b])))].tolist():
                if 0 <= v < V:
                    want[b, v] = _rules.PROMPT if prompt else want[b, v] + 1
    assert torch.equal(counts.cpu().long(), want)
    assert torch.equal(seen.cpu(), _rules.packed(want != 0))
    binding.token_counts_add(tokens[:, :0].to(DEV), counts, seen)          # nothing to add
    assert torch.equal(counts.cpu().long(), want)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("V", [900, 5003])
def test_counts_whose_seen_bit_is_not_set(dtype, V):
    """A token whose bit in `seen` is 0 counts as never seen whatever its count says, biased or not, on the path or not."""
    tb, tree, x, r, tok, paths = case(3, 29, 2, V, dtype, 400, 200, 3)
    g = torch.Generator().manual_seed(1)
    cleared = torch.rand(2, V, generator=g) < 0.5
    cleared[1] = True                               # a sequence that begins anew by clearing its words
    cleared[:, tok[0, 1]] = True
    r["seen"] = _rules.packed((r["counts"] != 0) & ~cleared)
    plain = dict(r, counts=torch.where(cleared, 0, r["counts"]))
    assert (cleared & (r["counts"] != 0)).gather(1, r["bias_ids"].long().clamp(0, V - 1)).any()
    want, _ = _rules.constrained(x, plain, tok, paths, torch.float32)
    out, keys = torch.empty_like(x, device=DEV), torch.empty(2 * tree.T, dtype=torch.int64, device=DEV)
    binding.logits_constrain(tree, x.to(DEV), out, on_device(r), tok.to(DEV))
    binding.constrained_argmax_keys(tree, x.to(DEV), keys, on_device(r), tok.to(DEV))
    assert torch.equal(bits(out.cpu() + 0.0), bits(want.to(dtype) + 0.0))
    key, _, top = _rules.keys_of(want)
    assert torch.equal(keys.cpu(), torch.where(top == -INF, 0, key))


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_an_infinite_frequency_penalty(dtype):
    """It takes what was generated, on the path too, out of the choice, and nothing else: not what is only in the prompt, nor what is only biased."""
    tb, tree, x, r, tok, paths = case(3, 29, 2, 1100, dtype, 300, 100, 0)
    r["frequency"][:] = 0.0
    want, _ = _rules.constrained(x, r, tok, paths, torch.float32)
    generated = ((r["counts"].long() & 0x7fffffff) > 0)[:, None].repeat(1, tree.T, 1)
    for b in range(2):
        for i, p in enumerate(paths):
            generated[b, i, tok[b, p].long()] = True
    want = torch.where(generated, -INF, want)
    r["frequency"][:] = INF
    out, keys = torch.empty_like(x, device=DEV), torch.empty(2 * tree.T, dtype=torch.int64, device=DEV)
    binding.logits_constrain(tree, x.to(DEV), out, on_device(r), tok.to(DEV))
    binding.constrained_argmax_keys(tree, x.to(DEV), keys, on_device(r), tok.to(DEV))
    assert torch.equal(bits(out.cpu() + 0.0), bits(want.to(dtype) + 0.0))
    assert torch.equal(keys.cpu(), _rules.keys_of(want)[0])


@pytest.mark.parametrize("V", [300, 40000])
def test_one_token_named_by_a_whole_bias_list(V):
    """4096 entries of one token (a list padded with a valid id): their sum in the list's order, and no slower than a list of many tokens
    by more than its loads.  Adding 4096 values one by one is a chain of some 100 thousand cycles, 60 us; a millisecond bounds a call."""
    tb, tree, x, r, tok, paths = case(2, 6, 3, V, BF16, 50, 4096, 0)
    r["bias"] *= 2.0 ** -6
    r["bias_ids"][0] = 7
    r["bias_ids"][1, ::2] = V - 1
    r["bias_ids"][2, 64:] = 0
    xd, rd, td = x.to(DEV), on_device(r), tok.to(DEV)
    out, keys = torch.empty_like(xd), torch.empty(3 * tree.T, dtype=torch.int64, device=DEV)
    want, _ = _rules.constrained(x, r, tok, paths, torch.float32)
    for _ in range(2):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        binding.logits_constrain(tree, xd, out, rd, td)
        binding.constrained_argmax_keys(tree, xd, keys, rd, td)
        stop.record()
    assert torch.equal(bits(out.cpu() + 0.0), bits(want.to(BF16) + 0.0))
    assert torch.equal(keys.cpu(), _rules.keys_of(want)[0])
    assert start.elapsed_time(stop) < 2.0
