"""Operators of a verification step over a paged K/V cache, as a list of cases that can be timed.

A case names an operator and its sizes:

  append   tree_kv_append_rope_paged: rotated K rows and V rows of the tree's nodes into the pages, all layers in one call
  rows     kv_append_rope_paged: the same for ragged runs of tokens (prompts in chunks, single tokens)
  attend   tree_verify_attention_paged: tree nodes (or single tokens: a tree of its root alone) over a cache whose first
           `shared` keys are the same for the whole batch
  compact  kv_compact_accepted_paged: the accepted nodes' rows move to the front, all layers
  logits   logits_constrain: penalties, biases and grammar masks, logits written
  accept   constrained_argmax_keys and tree_accept_keys: the same fused with the argmax, and the acceptance that reads it

Queries, keys, values ~ N(0, 1); pages in random order; lengths in [lo, hi]; logits ~ N(0, 2) with a greedy walk planted
down the tree; histories with a few frequent tokens and many rare ones.
"""
import heapq
import math
import random

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16
THETA = 10000.0


def _case(name, op, B=1, K=4, T=64, Hq=32, Hkv=8, D=128, page=64, shared=0, lo=0, hi=0, layers=1, V=0, dtype="bf16", hist=0, bias=0, masks=0):
    """lo, hi: keys of each sequence before this step, behind the shared ones (rows: tokens that are appended to each);
    hist: tokens of a sequence so far; bias: entries of a sequence's bias list; masks: grammar masks, 0 for none."""
    c = dict(op=op, B=B, K=K, T=T, Hq=Hq, Hkv=Hkv, D=D, page=page, shared=shared, lo=lo, hi=hi, layers=layers, V=V, dtype=dtype, hist=hist, bias=bias, masks=masks)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One verification step of a batch of four: the tree's rows for all 32 layers of a 7B-class model.
        _case("append batch of four", "append", B=4, lo=500, hi=2000, layers=32),
        # A prefill chunk of five ragged prompts, groups of seven query heads, small pages; one layer, as a backbone calls it.
        _case("append prompts", "rows", B=5, Hq=28, Hkv=4, page=16, lo=1, hi=1201),
        # The smallest step: one short sequence, latency counts.
        _case("attend tiny", "attend", K=3, T=29, Hq=8, Hkv=2, D=64, page=16, lo=128, hi=128),
        # Plain decoding of a serving batch behind one long system prompt: bound by the sequences' own keys.
        _case("attend single tokens", "attend", B=64, K=1, T=1, shared=8192, lo=100, hi=1000),
        # A ragged batch, groups of seven query heads, small pages, a shared prefix that no tile divides.
        _case("attend ragged", "attend", B=7, T=29, Hq=28, Hkv=4, page=16, shared=1008, lo=1, hi=5001),
        # The widest tree at head size 64.
        _case("attend head size 64", "attend", B=3, K=5, T=128, Hq=16, Hkv=2, D=64, page=32, shared=4096, lo=97, hi=1003),
        # Eight requests over one 16k document: a dense contraction.
        _case("attend document", "attend", B=8, shared=16384, lo=64, hi=2048),
        # The end of a step: a serving batch, all layers; and one sequence, latency.
        _case("compact batch", "compact", B=16, lo=1024, hi=4096, layers=32),
        _case("compact one", "compact", Hq=28, Hkv=4, page=16, lo=700, hi=700, layers=28),
        # Sampling outside: penalties written back for five sequences' trees, a vocabulary that no tile divides.
        _case("logits written", "logits", B=5, V=50003, hist=1500, bias=20, masks=8),
        # Greedy acceptance under a grammar: one small tree; a serving batch.
        _case("accept tiny", "accept", K=3, T=29, V=1024, hist=100, bias=3, masks=4),
        _case("accept batch", "accept", B=8, V=131072, hist=4000, bias=50, masks=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "rows", "attend", "attend", "attend", "compact", "logits", "accept"])
    K = rng.choice([2, 3, 4, 4, 5])
    T = 1 if rng.random() < 0.25 else _log_int(rng, 2, 128)
    D = 64 if rng.random() < 0.25 else 128
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    heads = dict(K=K, T=T, Hq=Hkv * G, Hkv=Hkv, D=D, page=page)
    if op in ("append", "rows", "compact"):
        B = _log_int(rng, 1, 64)
        layers = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, 4096)
        room = int(4e9 / (8 * B * Hkv * D * layers))            # a pool of at most 2 GB for K, and as much for V
        hi = max(1, min(hi, room // 2))
        if op == "rows":
            hi = max(1, min(hi, int(1e9 / (4 * B * layers * D * Hkv * (G + 2)))))
        lo = rng.choice([hi, max(1, hi // 3), 1])
        return _case("", op, B=B, lo=lo, hi=hi, layers=layers, **heads)
    if op == "attend":
        B = _log_int(rng, 1, 64)
        shared = 0 if rng.random() < 0.25 else _log_int(rng, 16, 16384) // page * page
        hi = _log_int(rng, 1, 4096)
        most = min(1.5e11 / (4 * B * T * Hkv * G * D), 2e9 / (4 * B * Hkv * max(G * T, D)))     # flops; the plain form's scores and keys
        shared = int(min(shared, max(16, most))) // page * page
        hi = int(max(1, min(hi, max(1, most - shared))))
        return _case("", op, B=B, shared=shared, lo=rng.choice([hi, max(1, hi // 10)]), hi=hi, **heads)
    V = _log_int(rng, 1000, 131072)
    B = max(1, min(_log_int(rng, 1, 64), int(7e7 / (T * V))))
    return _case("", op, B=B, K=K, T=T, V=V, dtype=rng.choice(["bf16", "bf16", "fp32"]), hist=_log_int(rng, 1, 8000),
                 bias=rng.choice([0, 0, _log_int(rng, 1, 300)]), masks=rng.choice([0, _log_int(rng, 1, 64)]))


# ------------------------------------------------------------------------------------------------ the tree
def _tree(K, T):
    """The T most likely nodes where the r-th candidate of a depth has weight 1 / (r + 1): rank tuples in the order (depth, ranks),
    with parent, depth and the paths from the root."""
    heap, nodes = [(-1.0, 0, ())], []
    while heap and len(nodes) < T:
        s, d, ranks = heapq.heappop(heap)
        nodes.append(ranks)
        if d < K:
            for r in range(10):
                heapq.heappush(heap, (s / (r + 1), d + 1, ranks + (r,)))
    nodes.sort(key=lambda n: (len(n), n))
    at = {n: i for i, n in enumerate(nodes)}
    parent = [at[n[:-1]] if n else -1 for n in nodes]
    paths = []
    for i, n in enumerate(nodes):
        p = [i]
        while parent[p[-1]] >= 0:
            p.append(parent[p[-1]])
        paths.append(p[::-1])
    leaves = [p for i, p in enumerate(paths) if i not in parent]
    return nodes, parent, paths, leaves


def _padded(rows, width):
    return torch.tensor([r + [-1] * (width - len(r)) for r in rows], device=DEV)


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape, scale=1.0, dtype=BF16):
    t = torch.empty(shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    for s in range(0, flat.numel(), 1 << 30):
        flat[s:s + (1 << 30)].normal_(0.0, scale, generator=g)
    return t


def _ints(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV, dtype=torch.int32)


def _pages(g, s, c, lens, room):
    """Pools of all layers and a table: the shared pages first, the same in every row, then each sequence's own."""
    B, page = c["B"], c["page"]
    n_shared = c["shared"] // page
    own_pages = -(-room // page)
    n_pages = n_shared + B * own_pages + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    s["table"] = torch.cat([order[:n_shared].expand(B, n_shared), order[n_shared:n_shared + B * own_pages].view(B, own_pages)], dim=1).contiguous()
    s["k"], s["v"] = (_normal(g, c["layers"], n_pages, c["Hkv"], page, c["D"]) for _ in range(2))
    s["lens"], s["status"] = lens, torch.zeros(B, dtype=torch.int32, device=DEV)


def _text(c, g, s, py, paths, parent):
    """Logits, drafted tokens, what the sequences said so far, penalties, biases and masks."""
    B, T, V = c["B"], len(paths), c["V"]
    s["tree_tok"] = torch.stack([torch.randperm(V, generator=g, device=DEV)[:T] for _ in range(B)]).to(torch.int32)
    x = _normal(g, B, T, V, scale=2.0, dtype=BF16 if c["dtype"] == "bf16" else torch.float32)
    tok, at = s["tree_tok"].tolist(), []
    for b in range(B):
        node = 0
        while True:
            ch = [j for j in range(T) if parent[j] == node]
            if not ch or py.random() > (0.3, 0.6, 0.9)[b % 3]:
                break
            nxt = py.choice(ch)
            at.append((b, node, tok[b][nxt]))
            node = nxt
    if at:
        b, i, t = torch.tensor(at, device=DEV).T
        x[b, i, t] = 24.0
    s["logits"] = x
    # tokens so far: bit 31 marks the prompt's, the lower bits count the generated ones; a few tokens are frequent
    counts = torch.zeros(B, V, dtype=torch.int64, device=DEV)
    said = (V * torch.rand(B, c["hist"], generator=g, device=DEV) ** 3).long().clamp(max=V - 1)
    n_prompt = c["hist"] // 2
    counts.scatter_add_(1, said[:, n_prompt:], torch.ones_like(said[:, n_prompt:]))
    prompt = torch.zeros(B, V, dtype=torch.bool, device=DEV)
    prompt.scatter_(1, said[:, :n_prompt], True)
    s["counts"] = (counts - (prompt.long() << 31)).to(torch.int32)
    words = -(-V // 32)
    bit = (1 << torch.arange(32, device=DEV)).view(1, 1, 32)

    def packed(m):
        m = torch.nn.functional.pad(m, (0, words * 32 - V)).view(m.shape[0], words, 32)
        w = (m.long() * bit).sum(-1)
        return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
    s["seen"] = packed(s["counts"] != 0)
    s["repetition"] = 1.0 + 0.3 * torch.rand(B, generator=g, device=DEV)
    s["presence"] = 0.5 * torch.rand(B, generator=g, device=DEV)
    s["frequency"] = 0.3 * torch.rand(B, generator=g, device=DEV)
    s["bias_ids"] = s["bias"] = s["mask"] = s["mask_of"] = None
    if c["bias"]:
        s["bias_ids"] = torch.where(torch.rand(B, c["bias"], generator=g, device=DEV) < 0.9, _ints(g, 0, V - 1, B, c["bias"]), -1).to(torch.int32)
        s["bias"] = 4.0 * torch.randn(B, c["bias"], generator=g, device=DEV)
    if c["masks"]:
        # grammars allow from a handful of tokens to nearly all; a third of the nodes is free
        share = 10.0 ** (-3.0 * torch.rand(c["masks"], 1, generator=g, device=DEV))
        allowed = torch.rand(c["masks"], V, generator=g, device=DEV) < share
        s["mask"] = packed(allowed)
        s["mask_of"] = _ints(g, -(c["masks"] // 2) - 1, c["masks"] - 1, B, T).clamp(min=-1)


def prepare(case, seed):
    c = case
    g, py = torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)
    nodes, parent, paths, leaves = _tree(c["K"], c["T"])
    op, B, T, K, D = c["op"], c["B"], len(nodes), c["K"], c["D"]
    s = dict(case=c, op=op, T=T, scale=D ** -0.5)
    s["depth"] = torch.tensor([len(n) for n in nodes], device=DEV)
    s["paths"] = _padded(paths, K + 1)
    s["leaves"] = _padded(leaves, K + 1)
    anc = [[0] * T for _ in range(T)]
    for i, p in enumerate(paths):
        for j in p:
            anc[i][j] = 1
    s["anc"] = torch.tensor(anc, dtype=torch.bool, device=DEV)
    if op in ("append", "rows", "attend", "compact"):
        lens = c["shared"] + _ints(g, c["lo"], c["hi"], B)
        room = c["hi"] + T
        if op == "rows":
            counts = [c["lo"] + (c["hi"] - c["lo"]) * b // max(1, B - 1) for b in range(B)]      # the same total for every seed
            py.shuffle(counts)
            lens = _ints(g, 0, 3 * c["page"], B)
            N = sum(counts)
            s["starts"] = torch.tensor([0] + counts, dtype=torch.int32, device=DEV).cumsum(0).to(torch.int32)
            room = c["hi"] + 3 * c["page"]
        _pages(g, s, c, lens, room)
    if op in ("append", "rows"):
        rows = (c["layers"], B, T) if op == "append" else (c["layers"], N)
        s["q"] = _normal(g, *rows, c["Hq"], D)
        s["k_new"], s["v_new"] = (_normal(g, *rows, c["Hkv"], D) for _ in range(2))
        s["q_out"] = torch.zeros_like(s["q"])
    elif op == "attend":
        s["q"] = _normal(g, B, T, c["Hq"], D)
        s["out"] = torch.zeros_like(s["q"])
    elif op == "compact":
        # accepted paths whose rows lie behind the rows they move to, so that a second pass finds the same rows
        nodes_of, n_of = [], []
        for _ in range(B):
            p = py.choice(leaves)
            n = py.randint(0, len(p) - 1)
            while any(j != p[j] and p[j] <= n for j in range(1, n + 1)):
                n -= 1
            nodes_of.append(p[:n + 1])
            n_of.append(n)
        s["acc_nodes"] = _padded(nodes_of, K + 1).to(torch.int32)
        s["accept_len"] = torch.tensor(n_of, dtype=torch.int32, device=DEV)
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    else:
        _text(c, g, s, py, paths, parent)
        if op == "logits":
            s["out"] = torch.zeros_like(s["logits"])
        else:
            i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
            s["keys"] = torch.zeros(B * T, dtype=torch.int64, device=DEV)
            s["accepted"] = dict(accept_len=i32(B), best_path=i32(B), acc_nodes=i32(B, K + 1), acc_tok=i32(B, K + 1), next_root=i32(B))
    if own:
        from paper_2603_03383_b200 import binding
        s["b"] = binding
        s["tree"] = binding.tree_build_static(K, [list(n) for n in nodes[1:]])
        if "k" in s:
            s["pool"] = binding.pool_layout(s["k"][0])
            s["k_ptrs"], s["v_ptrs"] = (binding.cache_pointer_array(list(s[x]), DEV) for x in "kv")
        if op == "attend":
            n = binding.paged_workspace_bytes(s["tree"], B, c["Hq"], c["Hkv"], D, c["shared"])
            s["ws"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
        if op in ("logits", "accept"):
            s["rules"] = binding.logit_rules(counts=s["counts"], seen=s["seen"], repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                                             bias_ids=s["bias_ids"], bias=s["bias"], mask=s["mask"], mask_of=s["mask_of"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _slots(s, slot):
    """Page and row in it of each sequence's slots [B][n]."""
    page = s["case"]["page"]
    return s["table"].gather(1, slot // page).long(), slot % page


def _rotated(x, pos, D):
    """x [layers, ..., heads, D] at positions pos [...]: angles in 64 bits, the rotation in 32, rounded once."""
    ang = pos.double()[..., None] * THETA ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    cs, sn = ang.cos().float()[..., None, :], ang.sin().float()[..., None, :]
    a, b = x.float().split(D // 2, dim=-1)
    return torch.cat([a * cs - b * sn, b * cs + a * sn], dim=-1).to(BF16)


def _plain_append(s):
    c = s["case"]
    if s["op"] == "append":
        L = s["lens"].long()[:, None]
        pos, slot = L + s["depth"], L + torch.arange(s["T"], device=DEV)
        pg, row = _slots(s, slot)
    else:
        r = torch.arange(s["q"].shape[1], device=DEV)
        b = torch.searchsorted(s["starts"][1:].contiguous(), r.to(torch.int32), right=True)
        slot = pos = s["lens"].long()[b] + r - s["starts"].long()[b]
        pg, row = s["table"][b, slot // c["page"]].long(), slot % c["page"]
    s["q_out"].copy_(_rotated(s["q"], pos, c["D"]))
    s["k"].transpose(2, 3)[:, pg, row] = _rotated(s["k_new"], pos, c["D"])
    s["v"].transpose(2, 3)[:, pg, row] = s["v_new"]


def _plain_attention(s):
    c, T = s["case"], s["T"]
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    n = -(-(c["shared"] + c["hi"] + T) // page)
    L = s["lens"].long()[:, None, None]
    j = torch.arange(n * page, device=DEV)
    node = (j - L).clamp(0, T - 1)                                             # [B, 1, keys]
    see = (j < L) | ((j >= L) & (j < L + T) & s["anc"][torch.arange(T, device=DEV)[:, None], node])   # [B, T, keys]
    pages = s["table"][:, :n].long()

    def gathered(pool):
        x = pool[0][pages].float().transpose(1, 2).reshape(B, Hkv, n * page, D)
        return x.mul_((j < L + T)[:, :, :, None])
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    x = (q @ gathered(s["k"]).transpose(2, 3)).view(B, Hkv, Hq // Hkv, T, n * page).mul_(s["scale"])
    x.masked_fill_(~see[:, None, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    w = x.sum(-1, keepdim=True)
    o = (x.view(B, Hkv, -1, n * page) @ gathered(s["v"])).view(B, Hkv, Hq // Hkv, T, D) / w
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D))


def _plain_compact(s):
    L = s["lens"].long()[:, None]
    j = torch.arange(s["acc_nodes"].shape[1], device=DEV)
    on = j <= s["accept_len"][:, None]
    src, sr = _slots(s, L + torch.where(on, s["acc_nodes"].long(), 0))
    dst, dr = _slots(s, L + torch.where(on, j, 0))
    for x in (s["k"], s["v"]):
        y = x.transpose(2, 3)
        y[:, dst, dr] = y[:, src, sr]
    s["new_lens"].copy_(s["lens"] + s["accept_len"] + 1)


def _bits(words, V):
    at = torch.arange(V, device=DEV)
    return (words[:, at // 32] >> (at % 32).to(torch.int32)) & 1 != 0


def _plain_constrained(s):
    """The constrained logits [B][T][V] in 32 bits."""
    c, T = s["case"], s["T"]
    B, V = c["B"], c["V"]
    x = s["logits"].float()
    path = s["paths"].expand(B, T, -1)
    tok = s["tree_tok"].long().gather(1, path.clamp(min=0).reshape(B, -1)).view_as(path)
    n = (s["counts"] & 0x7fffffff)[:, None, :].repeat(1, T, 1)
    n.scatter_add_(2, tok, (path >= 0).to(torch.int32))
    seen = (n > 0) | (s["counts"] < 0)[:, None, :]
    r, p, f = (s[k].view(B, 1, 1) for k in ("repetition", "presence", "frequency"))
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - f * n.float()
    x = torch.where(n > 0, x - p, x)
    if s["bias"] is not None:
        add = torch.zeros(B, V + 1, dtype=torch.float32, device=DEV)
        add.scatter_add_(1, torch.where(s["bias_ids"] >= 0, s["bias_ids"], V).long(), s["bias"])
        x = x + add[:, None, :V]
    if s["mask"] is not None:
        free = torch.cat([_bits(s["mask"], V), torch.ones(1, V, dtype=torch.bool, device=DEV)])
        x = torch.where(free[s["mask_of"].long()], x, -math.inf)     # -1: the last row, which allows everything
    return x


def _first_max(x):
    """The lowest index of each row's maximum, -1 where everything is masked."""
    top = x.amax(-1, keepdim=True)
    at = torch.where(x == top, torch.arange(x.shape[-1], device=DEV), x.shape[-1]).amin(-1)
    return torch.where(top[..., 0] == -math.inf, -1, at), top[..., 0]


def _accepted(s, am):
    """The longest path whose tokens are the ones chosen at their parents (ties: the first path)."""
    tok, ri = s["tree_tok"].long(), s["leaves"]
    B, (P, K1) = tok.shape[0], ri.shape
    at = ri.clamp(min=0).view(-1)
    path_tok, chosen = tok[:, at].view(B, P, K1), am[:, at].view(B, P, K1)
    ok = (path_tok[:, :, 1:] == chosen[:, :, :-1]) & (ri[:, 1:] >= 0)
    n = ok.long().cumprod(-1).sum(-1)
    best = torch.where(n == n.amax(1, keepdim=True), torch.arange(P, device=DEV), P).amin(1)
    n = n.gather(1, best[:, None])
    nodes = torch.where(torch.arange(K1, device=DEV) <= n, ri[best], -1)
    acc_tok = torch.where(nodes >= 0, tok.gather(1, nodes.clamp(min=0)), -1)
    nxt = am.gather(1, nodes.gather(1, n))[:, 0]
    return dict(accept_len=n[:, 0].int(), best_path=best.int(), acc_nodes=nodes.int(), acc_tok=acc_tok.int(), next_root=nxt.int())


def _plain_accept(s):
    am, top = _first_max(_plain_constrained(s))
    bits = (top + 0.0).view(torch.int32).long() & 0xffffffff          # + 0: one zero
    image = torch.where(bits >= 1 << 31, bits ^ 0xffffffff, bits | (1 << 31))
    image = torch.where(image >= 1 << 31, image - (1 << 32), image)   # as the high word of a signed key
    key = torch.where(am < 0, 0, (image << 32) + (0xffffffff - am))
    s["keys"].copy_(key.view(-1))
    for k, v in _accepted(s, am).items():
        s["accepted"][k].copy_(v)


def _outputs(s):
    op = s["op"]
    if op in ("append", "rows"):
        return [s["q_out"], s["k"], s["v"]]
    if op == "compact":
        return [s["k"], s["v"], s["new_lens"]]
    if op == "accept":
        return [s["keys"], s["accepted"]]
    return [s["out"]]


def run(state):
    s = state
    op = s["op"]
    if not own:
        {"append": _plain_append, "rows": _plain_append, "attend": _plain_attention, "compact": _plain_compact, "accept": _plain_accept,
         "logits": lambda s: s["out"].copy_(_plain_constrained(s))}[op](s)
        return _outputs(s)
    b, tree = s["b"], s["tree"]
    if op == "append":
        b.tree_kv_append_rope_paged(tree, s["q"], s["q_out"], s["k_new"], s["v_new"], s["k_ptrs"], s["v_ptrs"], s["pool"], s["table"], s["lens"], status=s["status"])
    elif op == "rows":
        b.kv_append_rope_paged(s["q"], s["q_out"], s["k_new"], s["v_new"], s["k_ptrs"], s["v_ptrs"], s["pool"], s["table"], s["lens"], s["starts"], status=s["status"])
    elif op == "attend":
        b.tree_verify_attention_paged(tree, s["q"], s["k"][0], s["v"][0], s["table"], s["lens"], s["out"], s["ws"], shared_len=s["case"]["shared"], status=s["status"])
    elif op == "compact":
        c = s["case"]
        b.kv_compact_accepted_paged(tree, s["k_ptrs"], s["v_ptrs"], c["layers"], c["Hkv"], c["D"], s["pool"], s["table"], s["lens"], s["new_lens"],
                                    s["accept_len"], s["acc_nodes"], status=s["status"])
    elif op == "logits":
        b.logits_constrain(tree, s["logits"], s["out"], s["rules"], s["tree_tok"])
    else:
        a = s["accepted"]
        b.constrained_argmax_keys(tree, s["logits"], s["keys"], s["rules"], s["tree_tok"])
        b.tree_accept_keys(tree, s["case"]["B"], s["keys"], s["tree_tok"], a["accept_len"], a["best_path"], a["acc_nodes"], a["acc_tok"], a["next_root"])
    return _outputs(s)


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    c = case
    B, T, D, Hq, Hkv, V = c["B"], len(_tree(c["K"], c["T"])[0]), c["D"], c["Hq"], c["Hkv"], c["V"]
    mean = (c["lo"] + c["hi"]) / 2
    if c["op"] in ("append", "rows"):
        each = [c["lo"] + (c["hi"] - c["lo"]) * b // max(1, B - 1) for b in range(B)]
        rows = (B * T if c["op"] == "append" else sum(each)) * c["layers"]
        return {"bytes": rows * D * (4.0 * Hq + 8.0 * Hkv), "flops": rows * D * 3.0 * (Hq + Hkv)}
    if c["op"] == "attend":
        return {"bytes": 4.0 * D * Hkv * (c["shared"] + B * (mean + T)) + 4.0 * B * T * Hq * D, "flops": 4.0 * B * T * Hq * D * (c["shared"] + mean + T)}
    if c["op"] == "compact":
        return {"bytes": 8.0 * c["layers"] * B * Hkv * D * 0.5 * min(c["K"], T - 1) + 12.0 * B, "flops": 0.0}
    size = 2.0 if c["dtype"] == "bf16" else 4.0
    once = B * T * V * size * (2 if c["op"] == "logits" else 1)
    bits = (B + min(c["masks"], B * T)) * V / 8.0
    return {"bytes": once + bits + 4.0 * B * c["hist"], "flops": 2.0 * B * T * V}


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_rows(s, x):
    """x [layers, rows, heads, D] rotated pair by pair as complex numbers, and where each row's K goes: (page, row in it)."""
    c, D = s["case"], s["case"]["D"]
    lens, table = s["lens"].tolist(), s["table"].tolist()
    pos, at = [], []
    if s["op"] == "append":
        depth = s["depth"].tolist()
        for b, L in enumerate(lens):
            for i in range(s["T"]):
                pos.append(L + depth[i])
                at.append((table[b][(L + i) // c["page"]], (L + i) % c["page"]))
    else:
        starts = s["starts"].tolist()
        for b, L in enumerate(lens):
            for i in range(starts[b + 1] - starts[b]):
                pos.append(L + i)
                at.append((table[b][(L + i) // c["page"]], (L + i) % c["page"]))
    freq = torch.tensor([THETA ** (-2.0 * d / D) for d in range(D // 2)], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones_like(freq)[None], torch.tensor(pos, dtype=torch.float64, device=DEV)[:, None] * freq)
    x = x.reshape(c["layers"], len(pos), -1, D).double()
    z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn[None, :, None]
    return torch.cat([z.real, z.imag], dim=-1), torch.tensor(at, device=DEV)


def _exact_attention(s):
    c, T = s["case"], s["T"]
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    lens, out = s["lens"].tolist(), torch.empty(B, T, Hq, D, dtype=torch.float64, device=DEV)
    for b in range(B):
        n = lens[b] + T
        slot = torch.arange(n, device=DEV)
        pg, row = s["table"][b].long()[slot // page], slot % page
        hide = torch.zeros(T, n, dtype=torch.bool, device=DEV)
        hide[:, lens[b]:] = ~s["anc"]
        for h in range(Hkv):
            k, v = s["k"][0][pg, h, row].double(), s["v"][0][pg, h, row].double()
            for x in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                z = (s["q"][b, :, x].double() @ k.T) / math.sqrt(D)
                out[b, :, x] = torch.softmax(z.masked_fill(hide, -math.inf), dim=-1) @ v
    return out


def _exact_constrained(s):
    c, T = s["case"], s["T"]
    B, V = c["B"], c["V"]
    out = torch.empty(B, T, V, dtype=torch.float64, device=DEV)
    counts, paths = s["counts"].long(), s["paths"].tolist()
    for b in range(B):
        r, p, f = (float(s[k][b]) for k in ("repetition", "presence", "frequency"))
        add = torch.zeros(V, dtype=torch.float64, device=DEV)
        if s["bias"] is not None:
            for t, x in zip(s["bias_ids"][b].tolist(), s["bias"][b].tolist()):
                if t >= 0:
                    add[t] += x
        for i in range(T):
            n = counts[b] % (1 << 31)
            for t in s["tree_tok"][b][[k for k in paths[i] if k >= 0]].tolist():
                n[t] += 1
            x = s["logits"][b, i].double()
            known = (n > 0) | (counts[b] < 0)
            x[known & (x > 0)] /= r
            low = known & (s["logits"][b, i] <= 0)
            x[low] *= r
            x = x - f * n - p * (n > 0) + add
            if s["mask"] is not None and int(s["mask_of"][b, i]) >= 0:
                w = s["mask"][int(s["mask_of"][b, i])].long() % (1 << 32)
                allowed = ((w[:, None] >> torch.arange(32, device=DEV)) % 2).view(-1)[:V] == 1
                x[~allowed] = -math.inf
            out[b, i] = x
    return out


def _exact_accept(s):
    x = _exact_constrained(s)
    am = torch.where((x == -math.inf).all(-1), -1, x.argmax(-1)).tolist()
    tok, leaves = s["tree_tok"].tolist(), s["leaves"].tolist()
    got = dict(accept_len=[], best_path=[], acc_nodes=[], acc_tok=[], next_root=[])
    for b in range(len(tok)):
        best = (0, 0)
        for p, path in enumerate(leaves):
            n = 0
            while n + 1 < len(path) and path[n + 1] >= 0 and tok[b][path[n + 1]] == am[b][path[n]]:
                n += 1
            if n > best[0]:
                best = (n, p)
        n, p = best
        nodes = leaves[p][:n + 1]
        got["accept_len"].append(n)
        got["best_path"].append(p)
        got["acc_nodes"].append(nodes + [-1] * (len(leaves[p]) - n - 1))
        got["acc_tok"].append([tok[b][k] for k in nodes] + [-1] * (len(leaves[p]) - n - 1))
        got["next_root"].append(am[b][nodes[-1]])
    return {k: torch.tensor(v, dtype=torch.int32, device=DEV) for k, v in got.items()}


def exact(case, seed):
    op = case["op"]
    if op == "compact":
        return None                     # copies and whole numbers
    s = prepare(case, seed)
    if op in ("append", "rows"):
        if s["k"].numel() > 1 << 29:
            return None
        q, at = _exact_rows(s, s["q"])
        k, _ = _exact_rows(s, s["k_new"])
        pool = s["k"].double()
        pool.transpose(2, 3)[:, at[:, 0], at[:, 1]] = k
        return [q.view(s["q"].shape), pool, None]
    if op == "attend":
        return [_exact_attention(s)]
    if op == "logits":
        return [_exact_constrained(s)]
    return [None, _exact_accept(s)]
