"""A video stream kept, shortened, forked and asked: the calls of a decoder's layers around the memory, on random weights.

    python examples/answer_from_memory.py [--layers 28] [--frames 64] [--question 32] [--answer 16]

For every frame the new keys are turned to their positions and stored with their values; then every fourth frame is dropped
(tom_oqm_keep_groups), the last few are copied into a second memory (tom_oqm_copy_groups), and a question is asked of the first:
its tokens are normed and turned into the rows where the attention reads them (tom_oqm_rotate), the frames are scored and
selected, and question and answer attend over system tokens, selected groups as they are stored and their own rows
(tom_oqm_attend).  At the end the last token is attended once more over the reconstructed active buffer, as a check.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2510_18269_amd import oqm  # noqa: E402


class Layers:
    """Random projections of a decoder with normed heads, and its rotary embedding."""
    def __init__(self, n_layers, q_heads, kv_heads, head_dim, hidden, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.n, self.q_heads, self.kv_heads, self.d, self.hidden = n_layers, q_heads, kv_heads, head_dim, hidden
        heads = q_heads + 2 * kv_heads
        draw = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.qkv = [(draw(hidden, heads * head_dim) * hidden ** -0.5).bfloat16() for _ in range(n_layers)]
        self.out = [(draw(q_heads * head_dim, hidden) * (q_heads * head_dim) ** -0.5).bfloat16() for _ in range(n_layers)]
        self.norm = [[(1 + 0.1 * draw(head_dim)).bfloat16() for _ in range(2)] for _ in range(n_layers)]
        self.rotary = oqm.Rotary.create(head_dim, base=1000000.0, scaling=oqm.TOM_ROTARY_BY_PARTS, factor=4.0, original_length=32768)

    def project(self, layer, x):
        """Queries, keys and values [tokens][heads][d], views of one product."""
        y = (x @ self.qkv[layer]).view(x.shape[0], -1, self.d)
        return y.split((self.q_heads, self.kv_heads, self.kv_heads), 1)


class Session:
    """A stream's memory, its system tokens, and the rows of what has been asked and answered."""
    def __init__(self, layers: Layers, group_tokens, capacity, longest):
        m = layers
        self.m, self.G = m, group_tokens
        self.memory = oqm.Memory.allocate(oqm.make_config(m.n, m.kv_heads, m.q_heads, m.d, group_tokens, 64, capacity))
        rows = lambda n: torch.zeros((m.n, m.kv_heads, n, m.d), dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.system = [rows(14), rows(14)]
        self.recent = [rows(longest), rows(longest)]
        self.used, self.position = 0, 0

    def watch(self, x):
        """One frame [G][hidden]: its keys are normed and turned, stored with the values; scored by the keys before the turn."""
        m, at = self.m, self.position + torch.arange(self.G, device="cuda")
        for layer in range(m.n):
            _, k, v = m.project(layer, x)
            turned = torch.empty_like(k)
            oqm.tom_oqm_rotate(m.rotary, at, k=k, k_out=turned, k_norm=m.norm[layer][1])
            tile = lambda t: t.transpose(0, 1).contiguous()[None, None]  # noqa: E731
            oqm.tom_oqm_quantize_append(self.memory.handle, layer, 1, 1, tile(turned), tile(v), tile(k), commit=layer == m.n - 1)
        self.position += self.G

    def shorten(self, keep):
        oqm.tom_oqm_keep_groups(self.memory.handle, keep, keep.numel())

    def fork(self, groups, capacity):
        other = Session(self.m, self.G, capacity, self.recent[0].shape[2])
        oqm.tom_oqm_copy_groups(other.memory.handle, self.memory.handle, groups, groups.numel())
        other.position = self.position
        return other

    def retrieve(self, x, k):
        """The frames of each layer that fit the question's queries: indices on the device."""
        m, T = self.m, self.memory.n_groups
        q = torch.stack([m.project(layer, x)[0].transpose(0, 1) for layer in range(m.n)]).contiguous()
        scores = torch.empty((m.n, T), device="cuda")
        ws = torch.empty(oqm.tom_oqm_score_workspace_bytes(self.memory.handle, m.n, x.shape[0]), dtype=torch.uint8, device="cuda")
        oqm.tom_oqm_score_groups(self.memory.handle, 0, m.n, q, x.shape[0], scores, T, workspace=ws)
        self.idx = torch.empty((m.n, k), dtype=torch.int32, device="cuda")
        self.k_eff = oqm.tom_oqm_topk(scores, T, m.n, T, k, self.idx)
        rows = 14 + k * self.G + self.recent[0].shape[2]
        need = max(oqm.tom_oqm_attend_workspace_bytes(self.memory.handle, t, rows) for t in (1, x.shape[0]))
        self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step(self, x):
        """New tokens [t][hidden] through all layers; returns what the last layer gives."""
        m, t, first = self.m, x.shape[0], self.used
        at = self.position + torch.arange(t, device="cuda")
        for layer in range(m.n):
            q, k, v = m.project(layer, x)
            turned, out = torch.empty_like(q), torch.empty_like(q)
            rows = [r[layer, :, first:first + t].transpose(0, 1) for r in self.recent]
            oqm.tom_oqm_rotate(m.rotary, at, q=q, q_out=turned, k=k, k_out=rows[0], v=v, v_out=rows[1], q_norm=m.norm[layer][0],
                               k_norm=m.norm[layer][1])
            oqm.tom_oqm_attend(self.memory.handle, layer, turned.transpose(0, 1), out.transpose(0, 1), self.idx[layer], self.k_eff,
                               self.system[0][layer], self.system[1][layer], self.recent[0][layer, :, :first + t],
                               self.recent[1][layer, :, :first + t], workspace=self.workspace)
            self.last = (layer, turned, out)
            x = x + out.reshape(t, -1) @ m.out[layer]
            x = x * torch.rsqrt((x.float() ** 2).mean(-1, keepdim=True) + 1e-6).bfloat16()
        self.used += t
        self.position += t
        return x

    def check(self):
        """The last layer's attention of the last step again, over the reconstructed active buffer instead of the codes; how far
        the two are apart, as a share of the largest value."""
        layer, q, out = self.last
        m = self.m
        shape = (1, m.kv_heads, 14 + self.k_eff * self.G, m.d)
        k, v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        oqm.tom_oqm_assemble_active(self.memory.handle, layer, 1, self.idx[layer:layer + 1], self.k_eff, self.k_eff, 14,
                                    self.system[0][layer:layer + 1], self.system[1][layer:layer + 1], k, v)
        again = torch.empty_like(out)
        oqm.tom_oqm_attend(self.memory.handle, layer, q.transpose(0, 1), again.transpose(0, 1), front_k=k[0], front_v=v[0],
                           recent_k=self.recent[0][layer, :, :self.used], recent_v=self.recent[1][layer, :, :self.used],
                           workspace=self.workspace)
        return float((again.float() - out.float()).abs().max() / again.float().abs().max())


def main(n_layers=28, frames=64, question=32, answer=16, group_tokens=196, q_heads=28, kv_heads=4, head_dim=128, hidden=3584, top_k=16):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tokens = lambda n: torch.randn((n, hidden), generator=g, device="cuda").bfloat16()  # noqa: E731
    s = Session(Layers(n_layers, q_heads, kv_heads, head_dim, hidden), group_tokens, frames, question + answer)
    for _ in range(frames):
        s.watch(tokens(group_tokens))
    keep = torch.tensor([i for i in range(frames) if i % 4 != 3], dtype=torch.int32, device="cuda")
    s.shorten(keep)
    last = torch.arange(max(0, s.memory.n_groups - 8), s.memory.n_groups, dtype=torch.int32, device="cuda")
    branch = s.fork(last, frames)

    asked = tokens(question)
    times, ends = [], []
    for session, k in ((s, min(top_k, s.memory.n_groups)), (branch, branch.memory.n_groups)):
        session.retrieve(asked, k)
        x = session.step(asked)[-1:]
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(answer):
            x = session.step(x)
        torch.cuda.synchronize()
        times.append((time.perf_counter() - t) / answer * 1e3)
        ends.append(x)
    off = [session.check() for session in (s, branch)]
    result = dict(kept=s.memory.n_groups, forked=branch.memory.n_groups, ms_per_token=times, apart=off, finite=all(bool(x.isfinite().all()) for x in ends))
    for session in (s, branch):
        session.memory.close()
    return result


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, default in (("layers", 28), ("frames", 64), ("question", 32), ("answer", 16)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    r = main(a.layers, a.frames, a.question, a.answer)
    print("%d groups kept, %d in the fork; a token through %d layers %.2f ms, in the fork %.2f ms; codes and reconstructed buffer apart by %.2g and %.2g "
          "of the largest value" % (r["kept"], r["forked"], a.layers, *r["ms_per_token"], *r["apart"]))
