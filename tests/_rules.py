"""Penalties, biases and masks in plain form: in fp32 one operation at a time (what the library promises to the bit), and in 64 bits."""
import torch

PROMPT = -(1 << 31)


def packed(allowed):
    """bool [n][V] -> int32 words [n][ceil(V / 32)]."""
    n, V = allowed.shape
    words = -(-V // 32)
    m = torch.nn.functional.pad(allowed, (0, words * 32 - V)).view(n, words, 32).long()
    w = (m << torch.arange(32)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def rules(g, B, T, V, hist=0, n_bias=0, n_masks=0, penalties=True):
    """Random rules as a dict of CPU tensors (None: left out), `allowed` bool [n_masks][V] beside the packed words."""
    r = dict.fromkeys(["counts", "seen", "repetition", "presence", "frequency", "bias_ids", "bias", "mask", "mask_of", "allowed"])
    if hist:
        said = (V * torch.rand(B, hist, generator=g) ** 2).long().clamp(max=V - 1)
        c = torch.zeros(B, V, dtype=torch.int64).scatter_add_(1, said[:, hist // 2:], torch.ones(B, hist - hist // 2, dtype=torch.int64))
        prompt = torch.zeros(B, V, dtype=torch.bool).scatter_(1, said[:, :hist // 2], True)
        r["counts"] = (c - (prompt.long() << 31)).to(torch.int32)
        r["seen"] = packed(r["counts"] != 0)
    if penalties:
        r["repetition"] = 0.8 + torch.rand(B, generator=g)
        r["presence"], r["frequency"] = torch.randn(B, generator=g), torch.randn(B, generator=g)
    if n_bias:
        r["bias_ids"] = torch.randint(-3, V + 3, (B, n_bias), generator=g).to(torch.int32)
        r["bias_ids"][:, n_bias // 2:] = r["bias_ids"][:, :n_bias - n_bias // 2].clone()     # most named twice
        r["bias"] = 4 * torch.randn(B, n_bias, generator=g)
    if n_masks:
        r["allowed"] = torch.rand(n_masks, V, generator=g) < 10.0 ** (-3 * torch.rand(n_masks, 1, generator=g))
        r["allowed"][0] = False                     # a mask that leaves nothing
        if n_masks > 1:
            r["allowed"][1] = torch.arange(V) == V - 1
        r["mask"] = packed(r["allowed"])
        r["mask_of"] = torch.randint(-1, n_masks, (B, T), generator=g).to(torch.int32)
        r["mask_of"][0, 0] = 0
        r["mask_of"][-1, -1] = min(1, n_masks - 1)
    return r


def constrained(x, r, tree_tok, paths, dtype):
    """x [B][T][V] -> (the constrained logits in dtype, a bound on what fp32 may differ by from exact arithmetic): every operation is
    rounded once, by at most 2^-24 of its result."""
    B, T, V = x.shape
    x = x.to(dtype)
    err = torch.zeros_like(x, dtype=torch.float64)
    half = 2.0 ** -24

    def rounded(y, carried):
        return carried + half * y.double().abs().nan_to_num(0, 0, 0)

    n = torch.zeros(B, T, V, dtype=torch.int64)
    prompt = torch.zeros(B, 1, V, dtype=torch.bool)
    if r["counts"] is not None:
        n += (r["counts"].long() & 0x7fffffff)[:, None]
        prompt = (r["counts"] < 0)[:, None]
    if tree_tok is not None:
        for b in range(B):
            for i, p in enumerate(paths):
                for j in p:
                    if 0 <= tree_tok[b, j] < V:
                        n[b, i, tree_tok[b, j]] += 1
    seen = prompt | (n > 0)

    def per_row(k, default):
        return torch.full((B, 1, 1), default, dtype=dtype) if r[k] is None else r[k].view(B, 1, 1).to(dtype)
    rep, pre, fre = per_row("repetition", 1.0), per_row("presence", 0.0), per_row("frequency", 0.0)
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    err = rounded(x, err)
    d = fre * n.to(dtype)
    x = x - d
    err = rounded(x, rounded(d, err))
    x = torch.where(n > 0, x - pre, x)
    err = rounded(x, err)
    if r["bias"] is not None:
        for b in range(B):
            add, size = torch.zeros(V, dtype=dtype), torch.zeros(V, dtype=torch.float64)
            for v, w in zip(r["bias_ids"][b].tolist(), r["bias"][b]):
                if 0 <= v < V:
                    add[v] += w.to(dtype)
                    size[v] += 2 * half * add[v].abs().double()
            x[b] = x[b] + add
            err[b] = rounded(x[b], err[b] + size)
    if r["mask"] is not None:
        free = torch.cat([r["allowed"], torch.ones(1, V, dtype=torch.bool)])
        x = torch.where(free[r["mask_of"].long().clamp(min=-1)], x, -float("inf"))
    return x, 4 * err            # the repetition scales what is carried (by less than two), the sums add up


def keys_of(x):
    """int64 keys [B * T] of fp32 values: the image of the largest value above, the lowest token's complement below; 0 for a row that
    has none (NaN counts for nothing; `x` has -inf in masked places, which a key may name only where `allowed` says so)."""
    x = x.reshape(-1, x.shape[-1])
    real = torch.where(x.isnan(), -float("inf"), x)
    top = real.amax(-1, keepdim=True)
    at = torch.where(x == top, torch.arange(x.shape[-1]), x.shape[-1]).amin(-1)
    bits = (top[:, 0] + 0.0).view(torch.int32).long() & 0xffffffff
    image = torch.where(bits >= 1 << 31, bits ^ 0xffffffff, bits | (1 << 31))
    image = torch.where(image >= 1 << 31, image - (1 << 32), image)
    return (image << 32) + (0xffffffff - at), at, top[:, 0]
