"""The calls on paged caches and constrained logits as a serving program runs them: prompts that share a prefix, then steps of append, attention,
constrained acceptance, compaction and counting, eagerly and as one replayed graph; against the same calls on a contiguous cache, the oracle's
attention and the formula of the constrained argmax."""
import pytest
import torch

from oracle import reference as ref
from paper_2603_03383_b200 import binding
from tests import _rules
from tests._cases import make_tree
from tests._paged import contiguous, pools, table

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
B, HQ, HKV, D, PAGE, LAYERS, V = 3, 8, 2, 64, 16, 2, 1500
SHARED, PROMPTS = 48, [5, 0, 40]                 # the prefix that all have, and what follows it


def i32(x):
    return torch.as_tensor(x).to(torch.int32).to(DEV)


class Server:
    """Buffers of a batch, and one step over them: nothing is allocated and the host reads nothing."""
    def __init__(self, K, T, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.tb, self.tree = make_tree("rank_prior", K, (), T)
        self.K, self.T = K, self.tree.T
        t, n_pages = table(self.g, B, 160, PAGE, SHARED)
        self.t = t.to(DEV)
        self.k, self.v = (pools(self.g, LAYERS, n_pages, HKV, PAGE, D, False, DEV) for _ in range(2))
        self.kp, self.vp = binding.cache_pointer_array(self.k, DEV), binding.cache_pointer_array(self.v, DEV)
        self.pool = binding.pool_layout(self.k[0])
        self.lens = i32([SHARED] * B)
        self.status = i32([0] * B)
        zeros = lambda *n: torch.zeros(*n, dtype=torch.int32, device=DEV)  # noqa: E731
        self.counts, self.seen = zeros(B, V), zeros(B, -(-V // 32))
        self.q, self.out = (torch.zeros(LAYERS, B, self.T, HQ, D, dtype=BF16, device=DEV) for _ in range(2))
        self.kn, self.vn = (torch.zeros(LAYERS, B, self.T, HKV, D, dtype=BF16, device=DEV) for _ in range(2))
        self.logits = torch.zeros(B, self.T, V, dtype=BF16, device=DEV)
        self.tok = zeros(B, self.T)
        self.keys = torch.zeros(B * self.T, dtype=torch.int64, device=DEV)
        self.acc = dict(accept_len=zeros(B), best_path=zeros(B), acc_nodes=zeros(B, K + 1), acc_tok=zeros(B, K + 1), next_root=zeros(B))
        self.ws = torch.zeros(binding.paged_workspace_bytes(self.tree, B, HQ, HKV, D, SHARED), dtype=torch.uint8, device=DEV)
        r = _rules.rules(self.g, B, self.T, V, 0, 6, 4)
        r["mask_of"][1:] = -1                   # two sequences without a grammar, so that something is accepted
        self.plain_rules = r
        self.rules = binding.logit_rules(counts=self.counts, seen=self.seen, **{k: r[k].to(DEV) for k in (
            "repetition", "presence", "frequency", "bias_ids", "bias", "mask", "mask_of")})

    def prompts(self):
        n = sum(PROMPTS)
        starts = [0]
        for p in PROMPTS:
            starts.append(starts[-1] + p)
        q, k, v = (torch.randn(LAYERS, n, h, D, generator=self.g).to(BF16).to(DEV) for h in (HQ, HKV, HKV))
        binding.kv_append_rope_paged(q, q, k, v, self.kp, self.vp, self.pool, self.t, self.lens, i32(starts), status=self.status)
        self.lens += i32(PROMPTS)
        said = torch.full((B, max(PROMPTS)), -1, dtype=torch.int32)
        for b, p in enumerate(PROMPTS):
            said[b, :p] = torch.randint(0, V, (p,), generator=self.g)
        binding.token_counts_add(said.to(DEV), self.counts, self.seen, i32(PROMPTS), prompt=True)

    def inputs(self):
        for x in (self.q, self.kn, self.vn):
            x.copy_(torch.randn(x.shape, generator=self.g).to(BF16))
        self.logits.copy_((2 * torch.randn(self.logits.shape, generator=self.g)).to(BF16))
        self.tok.copy_(torch.stack([torch.randperm(V, generator=self.g)[:self.T] for _ in range(B)]))
        self.tok[:, 0].copy_(torch.where(self.acc["next_root"] >= 0, self.acc["next_root"], 0))
        children = [j for j in range(self.T) if self.tb["depth"][j] == 1]
        for b in range(B):                      # a walk down the tree that the logits favour
            node = 0
            for _ in range(b + 1):
                below = [j for j in range(self.T) if self.tb["parent"][j] == node]
                if not below:
                    break
                nxt = below[int(torch.randint(0, len(below), (1,), generator=self.g))]
                self.logits[b, node, self.tok[b, nxt]] = 40.0
                node = nxt
        assert children

    def step(self):
        tree = self.tree
        binding.tree_kv_append_rope_paged(tree, self.q, self.q, self.kn, self.vn, self.kp, self.vp, self.pool, self.t, self.lens, status=self.status)
        for l in range(LAYERS):
            binding.tree_verify_attention_paged(tree, self.q[l], self.k[l], self.v[l], self.t, self.lens, self.out[l], self.ws, shared_len=SHARED)
        binding.constrained_argmax_keys(tree, self.logits, self.keys, self.rules, self.tok)
        binding.tree_accept_keys(tree, B, self.keys, self.tok, **self.acc)
        binding.kv_compact_accepted_paged(tree, self.kp, self.vp, LAYERS, HKV, D, self.pool, self.t, self.lens, self.lens, self.acc["accept_len"],
                                          self.acc["acc_nodes"], self.status)
        binding.token_counts_add(self.acc["acc_tok"], self.counts, self.seen)


def check(s, before):
    """One step that s has made, against the state `before` it."""
    torch.cuda.synchronize()
    k0, v0, lens, counts, seen, q0 = before
    T, K = s.T, s.K
    t = s.t.cpu()
    acc = {k: x.cpu() for k, x in s.acc.items()}
    # ---- the constrained argmax and the acceptance
    r = dict(s.plain_rules, counts=counts, seen=seen)
    mask = torch.tensor(s.tb["mask"], dtype=torch.bool)
    paths = [[j for j in range(T) if mask[i, j]] for i in range(T)]
    x, _ = _rules.constrained(s.logits.cpu(), r, s.tok.cpu(), paths, torch.float32)
    key, at, top = _rules.keys_of(x)
    nothing = top == -float("inf")
    assert torch.equal(s.keys.cpu(), torch.where(nothing, 0, key))
    want = ref.tree_accept(torch.where(nothing, -1, at).to(torch.int32).view(B, T), s.tok.cpu(), s.tb)
    for name, y in want.items():
        if name in acc:
            assert torch.equal(acc[name], y.to(torch.int32)), name
    # ---- the cache: the same calls on a contiguous one
    n = t.shape[1] * PAGE
    strides = (HKV * n * D, n * D, D)
    kc, vc = ([contiguous(x, t).to(DEV) for x in c] for c in (k0, v0))
    ld, status = i32(lens), i32([0] * B)
    kd, vd, qd = [x.to(DEV) for x in k0], [x.to(DEV) for x in v0], q0.to(DEV)
    binding.tree_kv_append_rope_paged(s.tree, qd, qd, s.kn, s.vn, binding.cache_pointer_array(kd, DEV), binding.cache_pointer_array(vd, DEV), s.pool, s.t, ld)
    assert torch.equal(qd, s.q)
    for l in range(LAYERS):
        q = q0[l].to(DEV)
        binding.tree_kv_append_rope(s.tree, q, s.kn[l], s.vn[l], kc[l], vc[l], ld, status=status)
        # Rotations of the two calls differ by less than 2^-19 (|a| + |b|) in front of their roundings (2^-20 each at most), then by a step of
        # bf16, 2^-7 of the value, where one lies on the other side of a tie.  |a| + |b| is below 16 here.
        kp_now, vp_now = contiguous(kd[l].cpu(), t), contiguous(vd[l].cpu(), t)
        for x, y in ((q.cpu(), qd[l].cpu()), (kc[l].cpu(), kp_now)):
            assert ((x.double() - y.double()).abs() <= 2.0 ** -7 * x.double().abs() + 2.0 ** -15).all()
        assert torch.equal(vc[l].cpu(), vp_now)
        kc[l] = kp_now.to(DEV)
        want = ref.tree_attention(qd[l].cpu(), kp_now, vp_now, lens, s.tb["mask"])
        absolute = ref.tree_attention(qd[l].cpu(), kp_now, vp_now.abs(), lens, s.tb["mask"])
        # roundings of the result and of the weights, as derived for the attention's own tests
        assert ((s.out[l].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + (1.02 * 2.0 ** -8 + 1e-4) * absolute + 1e-30).all()
    binding.kv_compact_accepted(s.tree, binding.cache_pointer_array(kc, DEV), binding.cache_pointer_array(vc, DEV), LAYERS, B, HKV, D, strides, n, ld,
                                s.acc["accept_len"], s.acc["acc_nodes"], status=status)
    torch.cuda.synchronize()
    assert torch.equal(ld, s.lens) and status.tolist() == [0] * B == s.status.tolist()
    for l in range(LAYERS):
        assert torch.equal(contiguous(s.k[l].cpu(), t), kc[l].cpu()) and torch.equal(contiguous(s.v[l].cpu(), t), vc[l].cpu())
    # ---- the counts
    new = counts.long()
    for b in range(B):
        for v in acc["acc_tok"][b].tolist():
            if v >= 0:
                new[b, v] += 1
    assert torch.equal(s.counts.cpu().long(), new) and torch.equal(s.seen.cpu(), _rules.packed(new != 0))
    assert binding.mtv_device_error(s.tree) == 0
    return acc["accept_len"].tolist()


def state(s):
    return ([x.cpu() for x in s.k], [x.cpu() for x in s.v], s.lens.cpu(), s.counts.cpu(), s.seen.cpu(), s.q.cpu())


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("K,T", [(3, 20), (4, 64)])
def test_steps(K, T, graph):
    s = Server(K, T, 17)
    s.prompts()
    torch.cuda.synchronize()
    assert s.lens.tolist() == [SHARED + p for p in PROMPTS] and s.status.tolist() == [0] * B
    accepted = []
    captured = None
    for step in range(4):
        s.inputs()
        before = state(s)
        if graph and step == 1:
            stream, captured = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(captured, stream=stream):
                s.step()
        if captured:
            captured.replay()
        else:
            s.step()
        accepted.append(check(s, before))
    assert any(n > 0 for a in accepted for n in a)


def test_single_tokens():
    """Plain decoding: a tree of its root alone, append, attention, constrained argmax, counts."""
    s = Server(3, 20, 23)
    s.prompts()
    tree = binding.tree_build_static(1, [])
    ws = torch.zeros(binding.paged_workspace_bytes(tree, B, HQ, HKV, D, SHARED), dtype=torch.uint8, device=DEV)
    tok = i32([[1], [2], [3]])
    for step in range(3):
        q, kn, vn = (torch.randn(1, B, 1, h, D, generator=s.g).to(BF16) for h in (HQ, HKV, HKV))
        logits = (2 * torch.randn(B, 1, V, generator=s.g)).to(BF16)
        counts, seen, lens = s.counts.cpu(), s.seen.cpu(), s.lens.cpu()
        qd, out, keys = q.to(DEV), torch.zeros(B, 1, HQ, D, dtype=BF16, device=DEV), torch.zeros(B, dtype=torch.int64, device=DEV)
        rows = lambda x: x.to(DEV).view(1, B, -1, D)  # noqa: E731  (one row per sequence: a ragged batch of ones)
        binding.kv_append_rope_paged(rows(q), qd.view(1, B, HQ, D), rows(kn), rows(vn), s.kp, s.vp, s.pool, s.t, s.lens, i32(range(B + 1)), status=s.status)
        binding.tree_verify_attention_paged(tree, qd[0], s.k[0], s.v[0], s.t, s.lens, out, ws, shared_len=SHARED, status=s.status)
        rules = binding.logit_rules(counts=s.counts, seen=s.seen, repetition=i32([1] * B).float() * 1.2, frequency=i32([1] * B).float())
        binding.constrained_argmax_keys(tree, logits.to(DEV), keys, rules, tok)
        binding.token_counts_add(tok, s.counts, s.seen)
        torch.cuda.synchronize()
        assert s.status.tolist() == [0] * B
        t = s.t.cpu()
        kc, vc = contiguous(s.k[0].cpu(), t), contiguous(s.v[0].cpu(), t)
        q_ref, k_ref = ref.rope(q[0], kn[0], lens.tolist(), [0])
        assert (qd[0].cpu().double() - q_ref).abs().max().item() <= 2.0 ** -7 * q_ref.abs().max().item()
        want = ref.tree_attention(qd[0].cpu(), kc, vc, lens, [[1]])
        absolute = ref.tree_attention(qd[0].cpu(), kc, vc.abs(), lens, [[1]])
        assert ((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + (1.02 * 2.0 ** -8 + 1e-4) * absolute + 1e-30).all()
        r = dict.fromkeys(s.plain_rules)
        r.update(counts=counts, seen=seen, repetition=torch.full((B,), 1.0) * 1.2, frequency=torch.ones(B))
        x, _ = _rules.constrained(logits, r, tok.cpu(), [[0]], torch.float32)
        assert torch.equal(keys.cpu(), _rules.keys_of(x)[0])
        s.lens += 1
        tok = i32((0xffffffff - (keys.cpu() & 0xffffffff)).view(B, 1))
