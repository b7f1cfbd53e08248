"""The calls on a cache in 8 bits as a serving program runs them: prompts that share a prefix, then steps of append, attention, acceptance and
compaction over all layers, eagerly and as one replayed graph, and plain decoding; every step against the formulas on the codes that it found."""
import pytest
import torch

from oracle import reference as ref
from paper_2603_03383_b200 import binding
from tests import _fp8
from tests._cases import make_tree
from tests._paged import table
from tests.test_gpu_paged_fp8_cache import byte_pools, i32, layout, ptrs, rotated, stored

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
B, HQ, HKV, PAGE, LAYERS, V = 3, 8, 2, 16, 3, 1500
SHARED, PROMPTS = 48, [5, 0, 40]                 # the prefix that all have, and what follows it


class Server:
    """Buffers of a batch, and one step over them: nothing is allocated and the host reads nothing."""
    def __init__(self, K, T, D, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.tb, self.tree = make_tree("rank_prior", K, (), T) if T > 1 else (dict(mask=[[1]], depth=[0], parent=[-1], T=1), binding.tree_build_static(1, []))
        self.K, self.T, self.D = self.tree.K, self.tree.T, D
        t, n_pages = table(self.g, B, 200, PAGE, SHARED)
        self.t = t.to(DEV)
        self.k, self.v = ([x & 0xf7 for x in byte_pools(self.g, LAYERS, n_pages, HKV, PAGE, D)] for _ in range(2))      # (no NaN)
        self.at, self.pool = ptrs(self.k, self.v), layout(self.k[0])
        self.ks, self.vs = (_fp8.scales(self.g, LAYERS, HKV).to(DEV) for _ in range(2))
        self.lens, self.status = i32([0] * B), i32([5] * B)
        zeros = lambda *n: torch.zeros(*n, dtype=torch.int32, device=DEV)  # noqa: E731
        self.q, self.out = (torch.zeros(LAYERS, B, self.T, HQ, D, dtype=BF16, device=DEV) for _ in range(2))
        self.kn, self.vn = (torch.zeros(LAYERS, B, self.T, HKV, D, dtype=BF16, device=DEV) for _ in range(2))
        self.logits, self.tok = torch.zeros(B, self.T, V, dtype=BF16, device=DEV), zeros(B, self.T)
        self.keys = torch.zeros(B * self.T, dtype=torch.int64, device=DEV)
        self.scan = torch.zeros(binding.mtv_workspace_bytes(self.tree, B, 64, V, HQ, HKV, D, 64), dtype=torch.uint8, device=DEV)
        self.acc = dict(accept_len=zeros(B), best_path=zeros(B), acc_nodes=zeros(B, self.K + 1), acc_tok=zeros(B, self.K + 1), next_root=zeros(B))
        self.ws = torch.zeros(binding.paged_workspace_bytes(self.tree, B, HQ, HKV, D, SHARED), dtype=torch.uint8, device=DEV)

    def append(self, counts, q, k, v):
        starts = [0]
        for n in counts:
            starts.append(starts[-1] + n)
        binding.kv_append_rope_paged_fp8(q, q, k, v, *self.at, self.pool, self.t, self.lens, i32(starts), self.ks, self.vs, status=self.status)
        return starts

    def prompts(self):
        # the prefix: one sequence writes it, all name its pages; then the ragged rest
        for counts in ([SHARED, 0, 0], PROMPTS):
            n = sum(counts)
            q, k, v = (torch.randn(LAYERS, n, h, self.D, generator=self.g).to(BF16).to(DEV) for h in (HQ, HKV, HKV))
            self.append(counts, q, k, v)
            self.lens += i32(counts if counts is PROMPTS else [SHARED] * B)

    def inputs(self):
        for x in (self.q, self.kn, self.vn):
            x.copy_(torch.randn(x.shape, generator=self.g).to(BF16))
        self.logits.copy_((2 * torch.randn(self.logits.shape, generator=self.g)).to(BF16))
        self.tok.copy_(torch.stack([torch.randperm(V, generator=self.g)[:self.T] for _ in range(B)]))
        for b in range(B):                      # a walk down the tree that the logits favour
            node = 0
            for _ in range(b + 1):
                below = [j for j in range(self.T) if self.tb["parent"][j] == node]
                if not below:
                    break
                nxt = below[int(torch.randint(0, len(below), (1,), generator=self.g))]
                self.logits[b, node, self.tok[b, nxt]] = 40.0
                node = nxt

    def step(self):
        tree = self.tree
        binding.tree_kv_append_rope_paged_fp8(tree, self.q, self.q, self.kn, self.vn, *self.at, self.pool, self.t, self.lens, self.ks, self.vs, status=self.status)
        for l in range(LAYERS):
            binding.tree_verify_attention_paged_fp8(tree, self.q[l], self.k[l].view(_fp8.FP8), self.v[l].view(_fp8.FP8), self.t, self.lens, self.out[l], self.ws,
                                                    self.ks[l], self.vs[l], shared_len=SHARED)
        binding.node_argmax_keys(tree, self.logits, self.keys, self.scan)
        binding.tree_accept_keys(tree, B, self.keys, self.tok, **self.acc)
        binding.kv_compact_accepted_paged_fp8(tree, *self.at, LAYERS, HKV, self.D, self.pool, self.t, self.lens, self.lens, self.acc["accept_len"],
                                              self.acc["acc_nodes"], self.status)


def check(s, k0, v0, lens, q0):
    """One step that s has made, against the state in front of it."""
    torch.cuda.synchronize()
    t, T = s.t.cpu(), s.T
    acc = {k: x.cpu() for k, x in s.acc.items()}
    assert s.status.tolist() == [0] * B and binding.mtv_device_error(s.tree) == 0
    am = s.logits.cpu().float().argmax(-1).to(torch.int32)
    for name, y in ref.tree_accept(am, s.tok.cpu(), s.tb).items():
        if name in acc:
            assert torch.equal(acc[name], y.to(torch.int32)), name
    assert s.lens.tolist() == [L + n + 1 for L, n in zip(lens, acc["accept_len"].tolist())]
    for l in range(LAYERS):
        q_ref, k_ref = ref.rope(q0[l], s.kn[l].cpu(), lens, s.tb["depth"])
        assert rotated(s.q[l].cpu(), q_ref, q0[l])
        # the codes as the append left them: the rows of nodes that were moved over are read from where they went
        k1, v1 = s.k[l].cpu(), s.v[l].cpu()
        for b, L in enumerate(lens):
            place = lambda i: (int(t[b, (L + i) // PAGE]), slice(None), (L + i) % PAGE)  # noqa: E731
            n = int(acc["accept_len"][b])
            moved = {int(acc["acc_nodes"][b, j]): j for j in range(1, n + 1)}
            for i in range(T):
                now = moved.get(i, i)
                if now == i and 1 <= i <= n and i not in moved:
                    continue                                   # written over by an accepted row
                for x0, x1, want, scale, of in ((k0, k1, k_ref[b, i], s.ks, s.kn[l, b, i].cpu()), (v0, v1, s.vn[l, b, i].cpu().double(), s.vs, None)):
                    got = x1[place(now)]
                    assert stored(got, want, scale[l].cpu(), of)
            for x0, x1 in ((k0[l], k1), (v0[l], v1)):
                for i in range(T):
                    x0[place(i)] = x1[place(i)]
        assert torch.equal(k0[l], k1) and torch.equal(v0[l], v1)          # nothing else was written
    return acc["accept_len"].tolist()


def attention_of(s, k, v, lens, l):
    return _fp8.attention(s.q[l].cpu(), k, v, s.ks[l].cpu(), s.vs[l].cpu(), s.t.cpu(), lens, s.tb["mask"])


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("K,T,D", [(3, 20, 64), (4, 64, 128)])
def test_steps(K, T, D, graph):
    s = Server(K, T, D, 17)
    s.prompts()
    torch.cuda.synchronize()
    assert s.lens.tolist() == [SHARED + p for p in PROMPTS] and s.status.tolist() == [0] * B
    accepted, captured = [], None
    for step in range(4):
        s.inputs()
        k0, v0, lens, q0 = [x.cpu() for x in s.k], [x.cpu() for x in s.v], s.lens.tolist(), s.q.cpu()
        if graph and step == 1:
            stream, captured = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(captured, stream=stream):
                s.step()
        if captured:
            captured.replay()
        else:
            s.step()
        # what the attention found: the same append into the state in front of the step
        kd, vd, qd = [x.to(DEV) for x in k0], [x.to(DEV) for x in v0], q0.to(DEV)
        binding.tree_kv_append_rope_paged_fp8(s.tree, qd, qd, s.kn, s.vn, *ptrs(kd, vd), s.pool, s.t, i32(lens), s.ks, s.vs)
        torch.cuda.synchronize()
        assert torch.equal(qd, s.q)
        for l in range(LAYERS):
            want, absolute = attention_of(s, kd[l], vd[l], lens, l)
            # roundings of the result, of the weights and of their exponentials, as derived for the attention's own tests
            assert ((s.out[l].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (2.0 ** -11 + 2 * 7.5e-5 + 1e-4) * absolute + 1e-30).all()
        accepted.append(check(s, k0, v0, lens, q0))
    assert any(n > 0 for a in accepted for n in a)


@pytest.mark.parametrize("D", [64, 128])
def test_single_tokens_and_reading_back(D):
    """Plain decoding: a ragged batch of ones, attention of a tree of its root alone; then the whole cache is read back and attended to in bf16."""
    s = Server(1, 1, D, 23)
    s.prompts()
    for step in range(3):
        q, k, v = (torch.randn(LAYERS, B, h, D, generator=s.g).to(BF16).to(DEV) for h in (HQ, HKV, HKV))
        lens = s.lens.tolist()
        s.append([1] * B, q, k, v)
        s.q.copy_(q.view(s.q.shape))
        for l in range(LAYERS):
            binding.tree_verify_attention_paged_fp8(s.tree, s.q[l], s.k[l].view(_fp8.FP8), s.v[l].view(_fp8.FP8), s.t, s.lens, s.out[l], s.ws, s.ks[l], s.vs[l],
                                                    shared_len=SHARED, status=s.status)
        torch.cuda.synchronize()
        assert s.status.tolist() == [0] * B
        for l in range(LAYERS):
            want, absolute = attention_of(s, s.k[l], s.v[l], lens, l)
            assert ((s.out[l].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (2.0 ** -11 + 2 * 7.5e-5 + 1e-4) * absolute + 1e-30).all()
        s.lens += 1
    n = s.lens.tolist()
    starts = [0, n[0], n[0] + n[1], sum(n)]
    k, v = (torch.zeros(LAYERS, sum(n), HKV, D, dtype=BF16, device=DEV) for _ in range(2))
    binding.kv_read_paged_fp8(*s.at, s.pool, s.t, i32(starts), s.ks, s.vs, k, v, status=s.status)
    assert s.status.tolist() == [0] * B
    for l in range(LAYERS):
        for b in range(B):
            # the last token's attention once more, from the rows that were read: a bf16 rounding of every key and value
            rows = slice(starts[b], starts[b + 1])
            kb, vb = (x[l, rows].cpu().double().transpose(0, 1).repeat_interleave(HQ // HKV, 0) for x in (k, v))
            y = s.q[l, b, 0].cpu().double()
            w = torch.softmax(torch.einsum("hd,hnd->hn", y, kb) * D ** -0.5, -1)
            want, absolute = torch.einsum("hn,hnd->hd", w, vb), torch.einsum("hn,hnd->hd", w, vb.abs())
            # keys off by 2^-9 each: scores by 2^-9 of sum |q k| / sqrt(D), weights by twice as much in numerator and sum; values by 2^-9
            slack = 2 * 2.0 ** -9 * (y.abs()[:, None] * kb.abs()).sum(-1).amax(-1) * D ** -0.5
            assert ((s.out[l, b, 0].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -9 + 1e-3 + 1.1 * slack[:, None]) * absolute).all()
