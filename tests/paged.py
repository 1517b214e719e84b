"""Rows of several sequences in pages for the tests, and what the calls on them have to give, in float64 on the CPU.

Whatever is nobody's row holds NaN: the pool is filled with it and only the rows that a sequence has are written."""
import math
import random

import torch

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Batch:
    def __init__(self, **kw):
        self.rows, self.new = [70, 0, 33], [5, 1, 3]
        self.heads, self.repeat, self.d, self.page_rows, self.layers, self.layer = 2, 7, 128, 16, 2, 1
        self.dtype, self.seed, self.one_each, self.order, self.holes, self.spare, self.spread = "bf16", 1, False, "lphrc", [], 2, 1.0
        self.behind = 0  # tokens behind the last sequence's
        for name, value in kw.items():
            assert hasattr(self, name), name
            setattr(self, name, value)
        self.B, self.T = len(self.new), sum(self.new) + self.behind
        self.starts_list = [sum(self.new[:i]) for i in range(self.B + 1)]
        g = torch.Generator().manual_seed(self.seed)
        rng = random.Random(self.seed)
        P, t = self.page_rows, DTYPE[self.dtype]
        used = [(r + n + P - 1) // P for r, n in zip(self.rows, self.new)]
        self.n_pages = sum(used) + self.spare
        order = list(range(self.n_pages))
        rng.shuffle(order)
        self.width = max(used) + 1
        self.table_list, at = [], 0
        for n in used:
            self.table_list.append(order[at:at + n] + [self.n_pages + 7, -1][:1] * (self.width - n))
            at += n
        self.k64, self.v64 = [], []  # [layers][heads][rows][d] a sequence, as the dtype holds them
        sizes = {"l": self.layers, "p": self.n_pages, "h": self.heads, "r": P, "c": self.d}
        shape = [sizes[x] for x in self.order]
        back = ["lphrc".index(x) for x in self.order]
        inverse = [back.index(i) for i in range(5)]
        self.k, self.v = (torch.full(shape, math.nan, dtype=t).permute(inverse) for _ in range(2))
        for s, (r, n) in enumerate(zip(self.rows, self.new)):
            pair = []
            for pool in (self.k, self.v):
                x = (torch.randn((self.layers, self.heads, r + n, self.d), generator=g) * self.spread).to(t)
                for i in range(r + n):
                    pool[:, self.table_list[s][i // P], :, i % P] = x[:, :, i]
                pair.append(x.double())
            self.k64.append(pair[0])
            self.v64.append(pair[1])
        for s, page in self.holes:
            self.table_list[s][page] = -1
        self.q = torch.randn((self.heads * self.repeat, self.T, self.d), generator=g).to(t)

    def device_pool(self, x):
        """The same tensor on the device, with the strides that its order gives."""
        back = ["lphrc".index(c) for c in self.order]
        inverse = [back.index(i) for i in range(5)]
        return x.permute(back).contiguous().cuda().permute(inverse)

    def pages(self, oqm):
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        return oqm.Pages.create(self.device_pool(self.k), self.device_pool(self.v), ints(self.table_list).reshape(self.B, self.width), ints(self.rows),
                                None if self.one_each else ints(self.starts_list))

    def there(self, s):
        """Which rows of sequence s have a page."""
        return torch.tensor([self.table_list[s][i // self.page_rows] in range(self.n_pages) for i in range(self.rows[s] + self.new[s])], dtype=torch.bool)

    def attention(self, masks, causal, scale, softcap, prior=None, one_part=False):
        """out, lse and how far each may be off.  masks: a set of seen new tokens for each token, or None; prior: (out, lse) in float64.

        A score is off by at most scale * sum_c |q_c k_c| * 2^-16 (float32 sums of up to 256 products) and with a cap, whose slope is at most one, by softcap *
        2^-20 more; that changes a probability by a factor of e^(2 off).  Probabilities enter the products as two 16-bit parts, 2^-16 of each, or as one, half a
        step of the type; sums of n terms in float32 add n * 2^-24, and exponentials 2^-20."""
        t = DTYPE[self.dtype]
        half = torch.finfo(t).eps / 2
        Hq = self.heads * self.repeat
        out = torch.zeros((Hq, self.T, self.d), dtype=torch.float64)
        lse = torch.full((Hq, self.T), -math.inf, dtype=torch.float64)
        bound, lse_bound = torch.zeros_like(out), torch.zeros_like(lse)
        for s in range(self.B):
            n, r = self.new[s], self.rows[s]
            if n == 0:
                continue
            at, there = self.starts_list[s], self.there(s)
            see = torch.zeros((n, r + n), dtype=torch.bool)
            see[:, :r] = True
            for j in range(n):
                for i in (masks[at + j] if masks is not None else range(j + 1) if causal else range(n)):
                    if i < n:
                        see[j, r + i] = True
            see &= there
            for h in range(Hq):
                k, v = self.k64[s][self.layer, h // self.repeat], self.v64[s][self.layer, h // self.repeat]
                q = self.q[h, at:at + n].double()
                w = q @ k.T * scale
                off = (abs(scale) * (q.abs() @ k.abs().T) * 2.0 ** -16).masked_fill(~see, 0).amax(1)
                if softcap:
                    w = softcap * torch.tanh(w / softcap)
                    off = off + softcap * 2.0 ** -20
                w = w.masked_fill(~see, -math.inf)
                v = v.clone()
                v[~see.any(0)] = 0
                if prior is not None:
                    w = torch.cat([w, prior[1][h, at:at + n][:, None]], 1)
                    off = torch.maximum(off, prior[1][h, at:at + n].abs().nan_to_num(posinf=0, neginf=0) * 2.0 ** -22)
                total = torch.logsumexp(w, 1)
                p = torch.exp(w - torch.where(total == -math.inf, 0.0, total)[:, None])
                o, size = p[:, :r + n] @ v, p[:, :r + n] @ v.abs()
                if prior is not None:
                    before = torch.where(prior[1][h, at:at + n][:, None] == -math.inf, 0.0, prior[0][h, at:at + n])
                    o, size = o + p[:, r + n:] * before, size + p[:, r + n:] * before.abs()
                rest = (half if one_part else 2.0 ** -16 if self.dtype != "f32" else 0) + (r + n) * 2.0 ** -24 + 2.0 ** -20
                out[h, at:at + n], lse[h, at:at + n] = o, total
                bound[h, at:at + n] = (2 * off + rest)[:, None] * size + half * o.abs() + torch.finfo(t).tiny
                lse_bound[h, at:at + n] = off + (r + n) * 2.0 ** -24 + 2.0 ** -20 * (1 + total.abs().nan_to_num(posinf=0, neginf=0))
        return out, lse, bound, lse_bound


def ancestors(parents, new):
    """The set of seen tokens of each token, numbers within its sequence."""
    out, at = [], 0
    for n in new:
        for j in range(n):
            p = parents[at + j]
            out.append([j] if p < 0 or p >= j else out[at + p] + [j])
        at += n
    return out


def to_words(masks, words):
    rows = []
    for seen in masks:
        w = [0] * words
        for j in set(seen):
            if j < 64 * words:
                w[j // 64] |= 1 << (j % 64)
        rows.append([x - (1 << 64) if x >= 1 << 63 else x for x in w])
    return torch.tensor(rows, dtype=torch.int64).reshape(len(masks), words)


def tree(new, seed):
    rng = random.Random(seed)
    return [-1 if j == 0 else max(0, j - rng.choice([1, 1, 2, 3, 7])) for n in new for j in range(n)]
