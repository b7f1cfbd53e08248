"""Helpers of the tests of the paged calls: random pages, and the contiguous cache that a page table stands for."""
import torch

BF16 = torch.bfloat16


def pools(g, n, n_pages, Hkv, page, D, tokens_outside=False, device="cpu"):
    """n pools as tensors [n_pages][Hkv][page][D]; tokens_outside: a page holds [page][Hkv][D]."""
    def one():
        if tokens_outside:
            return torch.randn(n_pages, page, Hkv, D, generator=g).to(BF16).to(device).transpose(1, 2)
        return torch.randn(n_pages, Hkv, page, D, generator=g).to(BF16).to(device)
    return [one() for _ in range(n)]


def table(g, B, rows, page, shared=0, spare=2):
    """(page table [B][max_pages], n_pages): room for `rows` slots behind the shared ones, pages in random order, a few of nobody."""
    n_shared, own = shared // page, -(-rows // page)
    n_pages = n_shared + B * own + spare
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    t = torch.cat([order[:n_shared].expand(B, n_shared), order[n_shared:n_shared + B * own].view(B, own)], dim=1)
    return t.contiguous(), n_pages


def contiguous(pool, t):
    """pool [n_pages][Hkv][page][D], table [B][max_pages] -> [B][Hkv][max_pages * page][D] (a copy)."""
    x = pool[t.long()]                                   # [B][pages][Hkv][page][D]
    B, n, Hkv, page, D = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * page, D).contiguous()
