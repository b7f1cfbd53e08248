"""Helpers of the tests of the 8-bit cache: pools of codes, and the values that they stand for."""
import torch

FP8 = torch.float8_e4m3fn
MAX = 448.0


def scales(g, *shape):
    """Scales that lay the largest of some thousand normal values near the end of the range."""
    return 0.008 + 0.012 * torch.rand(*shape, generator=g)


def code(x, scale):
    """x fp64, scale to its right sizes -> the codes of x / scale, from 64 bits (torch rounds once more, from fp32: values next to the middle of two
    codes may go either way)."""
    return (x.double() / scale.double()).clamp(-MAX, MAX).float().to(FP8)


def pools(g, n, n_pages, Hkv, page, D, tokens_outside=False, device="cpu"):
    """n pools of codes [n_pages][Hkv][page][D] of values of some units; tokens_outside: a page holds [page][Hkv][D]."""
    def one():
        shape = (n_pages, page, Hkv, D) if tokens_outside else (n_pages, Hkv, page, D)
        x = (100.0 * torch.randn(shape, generator=g)).clamp(-MAX, MAX).to(FP8).to(device)
        return x.transpose(1, 2) if tokens_outside else x
    return [one() for _ in range(n)]


def values(pool, scale):
    """What a pool [n_pages][Hkv][page][D] of codes (or their bytes) stands for, fp64; scale [Hkv]."""
    return pool.cpu().view(FP8).float().double() * scale.cpu().double()[None, :, None, None]


def put(pool, at, x):
    """pool[at] = x, x a number: codes are not written to by every torch operation."""
    pool.view(torch.uint8)[at] = torch.tensor(x).to(FP8).view(torch.uint8)


def attention(q, kp, vp, ks, vs, t, lens, mask, scale=None):
    """The formula in 64 bits, and the same on |v|: [B][T][Hq][D] each."""
    B, T, Hq, D = q.shape
    Hkv, page = kp.shape[1], kp.shape[2]
    k, v = values(kp, ks), values(vp, vs)
    hidden = ~torch.tensor(mask, dtype=torch.bool)
    out, absolute = torch.empty(2, B, T, Hq, D, dtype=torch.float64)
    for b, L in enumerate(lens):
        n = L + T
        pages = t[b, :-(-n // page)].long()
        kb, vb = (x[pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :n] for x in (k, v))
        y = q[b].double().view(T, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3)                        # [Hkv][G][T][D]
        z = (y @ kb[:, None].transpose(-1, -2)) * (scale or D ** -0.5)
        z[..., L:].masked_fill_(hidden, -torch.inf)
        w = torch.softmax(z, -1)
        for to, x in ((out, vb), (absolute, vb.abs())):
            to[b] = (w @ x[:, None]).permute(2, 0, 1, 3).reshape(T, Hq, D)
    return out, absolute
