"""What the tests of the serving operators share: packed rows, pages, caches."""

import numpy as np
import torch

from long_helpers import f64, normal
from paper_2609_12330_amd import ef_attention as ef


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts_of(counts, first=0):
    return [first + sum(counts[:i]) for i in range(len(counts) + 1)]


def quantised(x):
    """(codes, scales) of rows x by the definition: the smallest power of two, 2^-100 at least,
    that brings the largest magnitude to 448 at most. x is on the CPU."""
    x = x.float()
    top = x.abs().amax(-1)
    s = torch.full_like(top, 2.0 ** -100)
    while True:
        low = top > 448 * s.double()
        if not low.any():
            break
        s = torch.where(low, 2 * s, s)
    return (x / s[..., None]).to(torch.float8_e4m3fn), s


def make_table(seed, page, capacities, spare=3):
    """(pages, table [B, width]) with every sequence's pages somewhere among them; entries behind
    a sequence's last page name none."""
    need = [-(-n // page) for n in capacities]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = np.full((len(need), max(need + [1])), 10 ** 6, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = [order.pop() for _ in range(n)]
    return pages, table


class Pages:
    """A cache with random rows where sequences have keys, NaN everywhere else, and its values in
    64 bits."""

    def __init__(self, seed, H, page, D, lengths, e4m3):
        self.pages, self.table = make_table(seed, page, lengths)
        shape = (self.pages, H, page, D)
        self.values, held = [], []
        live = np.zeros((self.pages, page), bool)
        for b, n in enumerate(lengths):
            for p in range(n):
                if 0 <= self.table[b, p // page] < self.pages:
                    live[self.table[b, p // page], p % page] = True
        live = torch.from_numpy(live)[:, None].expand(self.pages, H, page)
        for i in range(2):
            x = normal(seed + 1 + i, *shape)
            if e4m3:
                codes, scales = quantised(x)
                codes.view(torch.uint8)[~live] = 0x7f
                scales = torch.where(live, scales, torch.nan)
                held.append((codes.cuda(), scales.cuda()))
                self.values.append(f64(codes.float()) * f64(scales)[..., None])
            else:
                x = torch.where(live[..., None], x, torch.nan)
                held.append((x.cuda(), None))
                self.values.append(f64(x))
        self.cache = ef.PagedCache(held[0][0], held[1][0], held[0][1], held[1][1])
        self.dev_table = torch.from_numpy(self.table).cuda()
