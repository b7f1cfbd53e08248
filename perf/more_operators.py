"""Operators of a verification step over a paged K/V cache of 8 bits, as a list of cases that can be timed.

The cache holds e4m3 codes with one scale per layer and KV head.  A case names an operator and its sizes:

  append   tree_kv_append_rope_paged_fp8: rotated K rows and V rows of the tree's nodes quantised into the pages, all layers in one call
  rows     kv_append_rope_paged_fp8: the same for ragged runs of tokens (prompts in chunks, single tokens)
  read     kv_read_paged_fp8: ragged runs of slots back as bf16 rows
  compact  kv_compact_accepted_paged_fp8: the accepted nodes' rows move to the front, all layers
  attend   tree_verify_attention_paged_fp8: tree nodes (or single tokens: a tree of its root alone) over a cache whose first
           `shared` keys are the same for the whole batch

Queries, keys, values ~ N(0, 1), scales that lay a head's largest values near the end of e4m3's range; pages in random order; lengths in [lo, hi].
"""
import heapq
import math
import random

import torch

own = False

DEV = "cuda"
BF16, FP8 = torch.bfloat16, torch.float8_e4m3fn
FP8_MAX = 448.0
THETA = 10000.0


def _case(name, op, B=1, K=4, T=64, Hq=32, Hkv=8, D=128, page=64, shared=0, lo=0, hi=0, layers=1):
    """lo, hi: keys of each sequence before this step, behind the shared ones (rows: tokens that are appended to each; read: slots that are
    read of each)."""
    c = dict(op=op, B=B, K=K, T=T, Hq=Hq, Hkv=Hkv, D=D, page=page, shared=shared, lo=lo, hi=hi, layers=layers)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One verification step of a batch of four: the tree's rows for all 32 layers of a 7B-class model.
        _case("append batch of four", "append", B=4, lo=500, hi=2000, layers=32),
        # The smallest step: one short sequence of a small model, latency counts.
        _case("append tiny", "append", K=3, T=29, Hq=8, Hkv=2, D=64, page=16, lo=128, hi=128, layers=2),
        # A prefill chunk of five ragged prompts, groups of seven query heads, small pages; one layer, as a backbone calls it.
        _case("append prompts", "rows", B=5, Hq=28, Hkv=4, page=16, lo=1, hi=1201),
        # Cached prefixes of a prefill batch, for a backbone whose own attention wants bf16 rows; one layer.
        _case("read prefixes", "read", B=4, lo=501, hi=8000),
        # A prompt's whole cache, handed over to another engine.
        _case("read all layers", "read", Hq=28, Hkv=4, page=16, lo=2050, hi=2050, layers=28),
        # The end of a step: a serving batch, all layers; and one sequence, latency.
        _case("compact batch", "compact", B=16, lo=1024, hi=4096, layers=32),
        _case("compact one", "compact", Hq=28, Hkv=4, page=16, lo=700, hi=700, layers=28),
        # The smallest step: one short sequence, latency counts.
        _case("attend tiny", "attend", K=3, T=29, Hq=8, Hkv=2, D=64, page=16, lo=128, hi=128),
        # Plain decoding of a serving batch: bound by the sequences' own keys.
        _case("attend single tokens", "attend", B=64, K=1, T=1, lo=500, hi=4000),
        # A ragged batch, groups of seven query heads, small pages, a shared prefix that no tile divides.
        _case("attend ragged", "attend", B=7, T=29, Hq=28, Hkv=4, page=16, shared=1008, lo=1, hi=5001),
        # One tree over a long context.
        _case("attend long", "attend", B=1, lo=60001, hi=60001),
        # Eight requests over one 16k document: a dense contraction.
        _case("attend document", "attend", B=8, shared=16384, lo=64, hi=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "rows", "read", "compact", "attend", "attend", "attend", "attend"])
    K = rng.choice([2, 3, 4, 4, 5])
    T = 1 if rng.random() < 0.25 else _log_int(rng, 2, 128)
    D = 64 if rng.random() < 0.25 else 128
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    heads = dict(K=K, T=T, Hq=Hkv * G, Hkv=Hkv, D=D, page=page)
    if op != "attend":
        B = _log_int(rng, 1, 64)
        layers = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, 4096)
        room = int(2e9 / (4 * B * Hkv * D * layers))            # a pool of at most 1 GB for K, and as much for V
        hi = max(1, min(hi, room // 2))
        if op in ("rows", "read"):
            hi = max(1, min(hi, int(4e8 / (B * layers * D * (4 * Hkv * G + 6 * Hkv if op == "rows" else 6 * Hkv)))))
        lo = rng.choice([hi, max(1, hi // 3), 1])
        return _case("", op, B=B, lo=lo, hi=hi, layers=layers, **heads)
    B = _log_int(rng, 1, 64)
    shared = 0 if rng.random() < 0.25 else _log_int(rng, 16, 16384) // page * page
    hi = _log_int(rng, 1, 60000 // B + 1000)
    most = min(1.4e11 / (4 * B * T * Hkv * G * D), 2e9 / (4 * B * Hkv * max(G * T, D)))     # flops; the plain form's scores and keys
    shared = int(min(shared, max(16, most))) // page * page
    hi = int(max(1, min(hi, max(1, most - shared))))
    return _case("", op, B=B, shared=shared, lo=rng.choice([hi, max(1, hi // 10)]), hi=hi, **heads)


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
    return nodes, paths, leaves


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape, dtype=BF16):
    t = torch.empty(shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    for s in range(0, flat.numel(), 1 << 30):
        flat[s:s + (1 << 30)].normal_(0.0, 1.0, generator=g)
    return t


def _ints(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV, dtype=torch.int32)


def _codes(g, scale, n_pages, Hkv, page, D):
    """A pool of all layers [layers][n_pages][Hkv][page][D], as the bytes of its codes."""
    pool = torch.empty(scale.shape[0], n_pages, Hkv, page, D, dtype=torch.uint8, device=DEV)
    for layer, s in zip(pool, scale):
        x = _normal(g, n_pages, Hkv, page, D) / s.view(1, Hkv, 1, 1).to(BF16)
        layer.copy_(x.clamp_(-FP8_MAX, FP8_MAX).to(FP8).view(torch.uint8))
    return pool


def prepare(case, seed):
    c = case
    g, py = torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)
    nodes, paths, leaves = _tree(c["K"], c["T"])
    op, B, T, K, D, Hkv, page, layers = c["op"], c["B"], len(nodes), c["K"], c["D"], c["Hkv"], c["page"], c["layers"]
    s = dict(case=c, op=op, T=T, scale=D ** -0.5)
    s["depth"] = torch.tensor([len(n) for n in nodes], device=DEV)
    anc = [[0] * T for _ in range(T)]
    for i, p in enumerate(paths):
        for j in p:
            anc[i][j] = 1
    s["anc"] = torch.tensor(anc, dtype=torch.bool, device=DEV)
    lens, room = c["shared"] + _ints(g, c["lo"], c["hi"], B), c["hi"] + T
    if op in ("rows", "read"):
        counts = [c["lo"] + (c["hi"] - c["lo"]) * b // max(1, B - 1) for b in range(B)]      # the same total for every seed
        py.shuffle(counts)
        lens = _ints(g, 0, 3 * page, B)           # read: the first slot of each run
        s["starts"] = torch.tensor([0] + counts, dtype=torch.int32, device=DEV).cumsum(0).to(torch.int32)
        room, N = c["hi"] + 3 * page, sum(counts)
    s["lens"], s["status"] = lens, torch.zeros(B, dtype=torch.int32, device=DEV)
    # pages: the shared ones first, the same in every row, then each sequence's own
    n_shared, own_pages = c["shared"] // page, -(-room // page)
    n_pages = n_shared + B * own_pages + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    s["table"] = torch.cat([order[:n_shared].expand(B, n_shared), order[n_shared:n_shared + B * own_pages].view(B, own_pages)], dim=1).contiguous()
    # a head's largest values are 3.5 to 7 in size
    s["k_scale"], s["v_scale"] = ((3.5 + 3.5 * torch.rand(layers, Hkv, generator=g, device=DEV)) / FP8_MAX for _ in range(2))
    s["k"], s["v"] = (_codes(g, s[x], n_pages, Hkv, page, D) for x in ("k_scale", "v_scale"))
    if op in ("append", "rows"):
        rows = (layers, B, T) if op == "append" else (layers, N)
        s["q"] = _normal(g, *rows, c["Hq"], D)
        s["k_new"], s["v_new"] = (_normal(g, *rows, Hkv, D) for _ in range(2))
        s["q_out"] = torch.zeros_like(s["q"])
    elif op == "read":
        s["k_out"], s["v_out"] = (torch.zeros(layers, N, Hkv, D, dtype=BF16, device=DEV) for _ in range(2))
    elif op == "attend":
        s["q"] = _normal(g, B, T, c["Hq"], D)
        s["out"] = torch.zeros_like(s["q"])
    else:
        # accepted paths whose rows lie behind the rows they move to, so that a second pass finds the same rows
        nodes_of, n_of = [], []
        for _ in range(B):
            p = py.choice(leaves)
            n = py.randint(0, len(p) - 1)
            while any(j != p[j] and p[j] <= n for j in range(1, n + 1)):
                n -= 1
            nodes_of.append(p[:n + 1] + [-1] * (K - n))
            n_of.append(n)
        s["acc_nodes"] = torch.tensor(nodes_of, dtype=torch.int32, device=DEV)
        s["accept_len"] = torch.tensor(n_of, dtype=torch.int32, device=DEV)
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    if own:
        from paper_2603_03383_b200 import binding
        s["b"] = binding
        s["tree"] = binding.tree_build_static(K, [list(n) for n in nodes[1:]])
        s["pool"] = binding.pool_layout(s["k"][0].view(FP8))
        s["k_ptrs"], s["v_ptrs"] = (binding.cache_pointer_array(list(s[x]), DEV) for x in "kv")
        if op == "attend":
            n = binding.paged_workspace_bytes(s["tree"], B, c["Hq"], Hkv, D, c["shared"])
            s["ws"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _slots(s, slot):
    """Page and row in it of each sequence's slots [B][n]."""
    page = s["case"]["page"]
    return s["table"].gather(1, slot // page).long(), slot % page


def _run_slots(s):
    """Sequence, and slot, of every row of the ragged runs."""
    r = torch.arange(_n_rows(s["case"]), device=DEV)
    b = torch.searchsorted(s["starts"][1:].contiguous(), r.to(torch.int32), right=True)
    return b, s["lens"].long()[b] + r - s["starts"].long()[b]


def _n_rows(c):
    return sum(c["lo"] + (c["hi"] - c["lo"]) * b // max(1, c["B"] - 1) for b in range(c["B"]))


def _rotated(x, pos, D):
    """x [layers, ..., heads, D] at positions pos [...]: angles in 64 bits, the rotation in 32."""
    ang = pos.double()[..., None] * THETA ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    cs, sn = ang.cos().float()[..., None, :], ang.sin().float()[..., None, :]
    a, b = x.float().split(D // 2, dim=-1)
    return torch.cat([a * cs - b * sn, b * cs + a * sn], dim=-1)


def _quantised(x, scale):
    """x [layers, ..., Hkv, D] in 32 bits -> codes, as bytes."""
    shape = [scale.shape[0]] + [1] * (x.dim() - 3) + [scale.shape[1], 1]
    return (x / scale.view(shape)).clamp(-FP8_MAX, FP8_MAX).to(FP8).view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    if s["op"] == "append":
        L = s["lens"].long()[:, None]
        pos, slot = L + s["depth"], L + torch.arange(s["T"], device=DEV)
        pg, row = _slots(s, slot)
    else:
        b, pos = _run_slots(s)
        pg, row = s["table"][b, pos // c["page"]].long(), pos % c["page"]
    s["q_out"].copy_(_rotated(s["q"], pos, c["D"]).to(BF16))
    s["k"].transpose(2, 3)[:, pg, row] = _quantised(_rotated(s["k_new"], pos, c["D"]), s["k_scale"])
    s["v"].transpose(2, 3)[:, pg, row] = _quantised(s["v_new"].float(), s["v_scale"])


def _plain_read(s):
    b, slot = _run_slots(s)
    pg, row = s["table"][b, slot // s["case"]["page"]].long(), slot % s["case"]["page"]
    for x in "kv":
        s[x + "_out"].copy_(s[x].transpose(2, 3)[:, pg, row].view(FP8).float() * s[x + "_scale"][:, None, :, None])


def _plain_attention(s):
    c, T = s["case"], s["T"]
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    n = -(-(c["shared"] + c["hi"] + T) // page)
    L = s["lens"].long()[:, None, None]
    j = torch.arange(n * page, device=DEV)
    node = (j - L).clamp(0, T - 1)                                             # [B, 1, keys]
    see = (j < L) | ((j >= L) & (j < L + T) & s["anc"][torch.arange(T, device=DEV)[:, None], node])   # [B, T, keys]
    pages = s["table"][:, :n].long()

    def gathered(x):
        y = s[x][0][pages].view(FP8).float().transpose(1, 2).reshape(B, Hkv, n * page, D)
        return y.mul_((j < L + T)[:, :, :, None]).mul_(s[x + "_scale"][0].view(1, Hkv, 1, 1))
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    x = (q @ gathered("k").transpose(2, 3)).view(B, Hkv, Hq // Hkv, T, n * page).mul_(s["scale"])
    x.masked_fill_(~see[:, None, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    w = x.sum(-1, keepdim=True)
    o = (x.view(B, Hkv, -1, n * page) @ gathered("v")).view(B, Hkv, Hq // Hkv, T, D) / w
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


def _outputs(s):
    op = s["op"]
    if op in ("append", "rows"):
        return [s["q_out"], s["k"].view(FP8), s["v"].view(FP8)]
    if op == "read":
        return [s["k_out"], s["v_out"]]
    if op == "compact":
        return [s["k"].view(FP8), s["v"].view(FP8), s["new_lens"]]
    return [s["out"]]


def run(state):
    s = state
    op = s["op"]
    if not own:
        {"append": _plain_append, "rows": _plain_append, "read": _plain_read, "attend": _plain_attention, "compact": _plain_compact}[op](s)
        return _outputs(s)
    b, tree, c = s["b"], s["tree"], s["case"]
    cache = (s["k_ptrs"], s["v_ptrs"])
    if op == "append":
        b.tree_kv_append_rope_paged_fp8(tree, s["q"], s["q_out"], s["k_new"], s["v_new"], *cache, s["pool"], s["table"], s["lens"],
                                        s["k_scale"], s["v_scale"], status=s["status"])
    elif op == "rows":
        b.kv_append_rope_paged_fp8(s["q"], s["q_out"], s["k_new"], s["v_new"], *cache, s["pool"], s["table"], s["lens"], s["starts"],
                                   s["k_scale"], s["v_scale"], status=s["status"])
    elif op == "read":
        b.kv_read_paged_fp8(*cache, s["pool"], s["table"], s["starts"], s["k_scale"], s["v_scale"], s["k_out"], s["v_out"], first=s["lens"],
                            status=s["status"])
    elif op == "compact":
        b.kv_compact_accepted_paged_fp8(tree, *cache, c["layers"], c["Hkv"], c["D"], s["pool"], s["table"], s["lens"], s["new_lens"],
                                        s["accept_len"], s["acc_nodes"], status=s["status"])
    else:
        b.tree_verify_attention_paged_fp8(tree, s["q"], s["k"][0].view(FP8), s["v"][0].view(FP8), s["table"], s["lens"], s["out"], s["ws"],
                                          s["k_scale"][0], s["v_scale"][0], shared_len=c["shared"], status=s["status"])
    return _outputs(s)


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    c = case
    B, T, D, Hq, Hkv = c["B"], len(_tree(c["K"], c["T"])[0]), c["D"], c["Hq"], c["Hkv"]
    mean = (c["lo"] + c["hi"]) / 2
    if c["op"] in ("append", "rows"):
        rows = (B * T if c["op"] == "append" else _n_rows(c)) * c["layers"]
        return {"bytes": rows * D * (4.0 * Hq + 6.0 * Hkv), "flops": rows * D * 3.0 * (Hq + Hkv)}
    if c["op"] == "read":
        return {"bytes": 6.0 * _n_rows(c) * c["layers"] * Hkv * D, "flops": 2.0 * _n_rows(c) * c["layers"] * Hkv * D}
    if c["op"] == "attend":
        return {"bytes": 2.0 * D * Hkv * (c["shared"] + B * (mean + T)) + 4.0 * B * T * Hq * D, "flops": 4.0 * B * T * Hq * D * (c["shared"] + mean + T)}
    return {"bytes": 4.0 * c["layers"] * B * Hkv * D * 0.5 * min(c["K"], T - 1) + 12.0 * B, "flops": 0.0}


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_places(s):
    """Positions of the call's rows and where each row's K lies: (page, row in it)."""
    c, lens, table = s["case"], s["lens"].tolist(), s["table"].tolist()
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
    return torch.tensor(pos, dtype=torch.float64, device=DEV), torch.tensor(at, device=DEV)


def _exact_turned(s, x, pos):
    """x [layers, rows, heads, D] rotated pair by pair as complex numbers."""
    c, D = s["case"], s["case"]["D"]
    freq = torch.tensor([THETA ** (-2.0 * d / D) for d in range(D // 2)], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones_like(freq)[None], pos[:, None] * freq)
    x = x.reshape(c["layers"], len(pos), -1, D).double()
    z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn[None, :, None]
    return torch.cat([z.real, z.imag], dim=-1)


def _values(codes):
    """The numbers that e4m3 codes stand for, from their bits."""
    table = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if (e, m) == (15, 7) else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        table.append(-v if c >> 7 else v)
    return torch.tensor(table, dtype=torch.float64, device=DEV)[codes.long()]


def _exact_append(s):
    pos, at = _exact_places(s)
    out = [_exact_turned(s, s["q"], pos).view(s["q"].shape)]
    for x, y in (("k", _exact_turned(s, s["k_new"], pos)), ("v", s["v_new"].reshape(s["case"]["layers"], len(pos), -1, s["case"]["D"]).double())):
        pool = _values(s[x])
        pool.transpose(2, 3)[:, at[:, 0], at[:, 1]] = (y / s[x + "_scale"].double()[:, None, :, None]).clamp(-FP8_MAX, FP8_MAX)
        out.append(pool)
    return out


def _exact_read(s):
    _, at = _exact_places(s)
    return [_values(s[x].transpose(2, 3)[:, at[:, 0], at[:, 1]]) * s[x + "_scale"].double()[:, None, :, None] for x in "kv"]


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
            k, v = (_values(s[x][0][pg, h, row]) * float(s[x + "_scale"][0, h]) for x in "kv")
            for x in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                z = (s["q"][b, :, x].double() @ k.T) / math.sqrt(D)
                out[b, :, x] = torch.softmax(z.masked_fill(hide, -math.inf), dim=-1) @ v
    return out


def _exact_compact(s):
    """Row by row; every row is read from the pool as it was."""
    page, lens, table, nodes = s["case"]["page"], s["lens"].tolist(), s["table"].tolist(), s["acc_nodes"].tolist()
    out = []
    for x in "kv":
        pool = _values(s[x])
        before = pool.clone()
        for b, n in enumerate(s["accept_len"].tolist()):
            for j in range(1, n + 1):
                (sp, sr), (dp, dr) = ((table[b][i // page], i % page) for i in (lens[b] + nodes[b][j], lens[b] + j))
                pool[:, dp, :, dr] = before[:, sp, :, sr]
        out.append(pool)
    return out + [s["lens"] + s["accept_len"] + 1]


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if s["k"].numel() > 1 << 29:
        return None
    if op == "compact":
        return _exact_compact(s)
    if op in ("append", "rows"):
        return _exact_append(s)
    if op == "read":
        return _exact_read(s)
    return [_exact_attention(s)]
