"""Performance cases of answers that are drafted: several conversations at once, their recent rows in pages of one pool, and drafted
tokens that form a tree.

Four kinds of pass:

  tree    the parents of drafted tokens made into masks of ancestors and positions, once for all layers of a step
  append  new queries and keys normed and turned to their positions, the keys and values written to the rows behind their sequences
  attend  new tokens over the paged rows of their sequences, a tree's tokens over their ancestors among the new rows only, joined
          with a part that another attention has given for the same tokens (over the stored frames)
  keep    the rows of the accepted tokens move together behind their sequences, in all layers, and the others are dropped

Sizes are those of the repository's workloads (28 layers, 4 KV heads of 128 channels, 28 query heads; the tiny stream of 64
channels its tests use) and generic ragged ones.
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# rows: how many each sequence has, between rows_from and rows_to; new: tokens of each, between new_from and new_to; by `shape`
_BATCH = {"sequences": 1, "rows_from": 0, "rows_to": 0, "new_from": 1, "new_to": 1, "shape": 1}
_TREE = {"kind": "tree", **_BATCH, "deep": False}
_APPEND = {"kind": "append", **_BATCH, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "rotary_dim": 128, "layout": "half", "norm": False,
           "dtype": "bf16", "base": 1000000.0, "first": 0, "page_rows": 64, "layers": 2, "one_each": False}
_ATTEND = {"kind": "attend", **_BATCH, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "dtype": "bf16", "page_rows": 64, "layers": 1,
           "one_each": False, "tree": False, "causal": True, "softcap": 0.0, "prior": False, "holes": 0}
_KEEP = {"kind": "keep", **_BATCH, "kv_heads": 4, "head_dim": 128, "dtype": "bf16", "page_rows": 64, "layers": 28, "kept": 4}


def listed():
    return [
        # a small draft of one conversation; latency
        {**_TREE, "name": "tree_one", "new_from": 13, "new_to": 13},
        # a serving step: 96 conversations with drafts of up to 200 tokens, ragged
        {**_TREE, "name": "tree_many", "sequences": 96, "new_from": 5, "new_to": 200, "shape": 7},
        # one generated token of the 28-head model, norms and all, into its page; latency
        {**_APPEND, "name": "append_token", "norm": True, "rows_from": 12700, "rows_to": 12700, "first": 12700, "one_each": True},
        # the drafts of 24 conversations, pages of 50 rows, half of each head turned, interleaved
        {**_APPEND, "name": "append_drafts", "sequences": 24, "rows_from": 100, "rows_to": 20000, "new_from": 3, "new_to": 64, "shape": 3, "rotary_dim": 64,
         "layout": "pairs", "dtype": "f16", "page_rows": 50, "first": 705600},
        # prompts of seven conversations at once
        {**_APPEND, "name": "append_prompts", "sequences": 7, "rows_from": 0, "rows_to": 3000, "new_from": 700, "new_to": 5000, "shape": 5, "page_rows": 256},
        # the tiny float32 stream of the tests: launches, hardly any data
        {**_ATTEND, "name": "pages_tiny", "sequences": 2, "kv_heads": 2, "q_heads": 2, "head_dim": 64, "dtype": "f32", "page_rows": 16, "rows_from": 3,
         "rows_to": 70, "new_from": 2, "new_to": 5, "tree": True},
        # one generated token of one conversation over what a question retrieved and the answer so far
        {**_ATTEND, "name": "pages_token", "layers": 2, "rows_from": 12600, "rows_to": 12600, "one_each": True},
        # one generated token each of 48 conversations of very different lengths
        {**_ATTEND, "name": "pages_batch", "sequences": 48, "rows_from": 40, "rows_to": 30000, "shape": 11, "one_each": True},
        # drafted trees of four conversations, their stored frames already attended to
        {**_ATTEND, "name": "pages_drafts", "sequences": 4, "rows_from": 2000, "rows_to": 13000, "new_from": 33, "new_to": 64, "shape": 2, "tree": True,
         "prior": True},
        # prompts of three conversations over what they have, scores capped, binary16, pages of a frame
        {**_ATTEND, "name": "pages_prompts", "sequences": 3, "rows_from": 500, "rows_to": 6000, "new_from": 900, "new_to": 3000, "shape": 9, "dtype": "f16",
         "softcap": 30.0, "page_rows": 196},
        # one conversation's accepted tokens, all layers; latency
        {**_KEEP, "name": "keep_one", "rows_from": 12600, "rows_to": 12600, "new_from": 13, "new_to": 13},
        # a serving step: 64 conversations, drafts of up to 64 tokens
        {**_KEEP, "name": "keep_many", "sequences": 64, "rows_from": 40, "rows_to": 1200, "new_from": 20, "new_to": 64, "shape": 4, "kept": 12, "page_rows": 50},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree", "append", "attend", "attend", "attend", "attend", "keep"])
    shape = rng.randint(1, 1 << 30)
    pages = rng.choice([1, 7, 16, 16, 50, 64, 64, 128, 196, 256])
    if kind == "tree":
        n = _log(rng, 1, 200)
        return {**_TREE, "shape": shape, "sequences": _log(rng, 1, 96), "new_from": rng.randint(1, n), "new_to": n, "deep": rng.random() < 0.3}
    if kind == "append":
        c = {**_APPEND, "shape": shape, "page_rows": pages}
        c["head_dim"] = rng.choice([64, 80, 96, 128, 128, 256])
        c["rotary_dim"] = rng.choice([c["head_dim"], c["head_dim"], c["head_dim"] // 2, 2 * rng.randint(1, c["head_dim"] // 2)])
        c["layout"] = rng.choice(["half", "pairs"])
        c["kv_heads"] = rng.choice([1, 2, 4, 8])
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 7])
        c["norm"] = rng.random() < 0.5
        c["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["base"] = rng.choice([10000.0, 500000.0, 1000000.0])
        c["first"] = rng.choice([0, rng.randint(0, 5000), rng.randint(0, 1000000)])
        c["sequences"] = _log(rng, 1, 60)
        c["one_each"] = rng.random() < 0.3
        if not c["one_each"]:
            c["new_to"] = _log(rng, 1, 4000 // c["sequences"])
            c["new_from"] = rng.randint(0, c["new_to"])
        c["rows_to"] = _log(rng, 1, 40000 // c["sequences"])
        c["rows_from"] = rng.randint(0, c["rows_to"])
        return c
    if kind == "attend":
        c = {**_ATTEND, "shape": shape, "page_rows": pages, "layers": rng.choice([1, 2, 3])}
        c["head_dim"] = rng.choice([64, 80, 96, 128, 128, 128, 256])
        c["kv_heads"] = rng.choice([1, 2, 4, 4, 8])
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 7, 8])
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
        c["sequences"] = _log(rng, 1, 64)
        which = rng.choice(["one", "tree", "tree", "prompt"])
        if which == "one":
            c["one_each"] = True
            c["rows_to"] = _log(rng, 1, 60000 // c["sequences"] + 100)
        elif which == "tree":
            c["tree"] = True
            c["new_to"] = _log(rng, 1, 400 // c["sequences"] + 10)
            c["rows_to"] = _log(rng, 1, 40000 // c["sequences"] + 100)
        else:
            c["sequences"] = min(c["sequences"], rng.randint(1, 8))
            c["new_to"] = _log(rng, 2, 1500 // c["sequences"])
            c["rows_to"] = _log(rng, 1, 6000 // c["sequences"])
            c["causal"] = rng.random() < 0.8
        c["new_from"] = c["new_to"] if which == "one" else rng.randint(0 if c["sequences"] > 1 else 1, c["new_to"])
        c["rows_from"] = rng.randint(0, c["rows_to"])
        c["softcap"] = rng.choice([0.0, 0.0, 20.0, 50.0])
        c["prior"] = rng.random() < 0.4
        c["holes"] = rng.choice([0, 0, 0, 2])
        return c
    c = {**_KEEP, "shape": shape, "page_rows": pages}
    c["layers"] = rng.choice([1, 2, 4, 28])
    c["kv_heads"] = rng.choice([1, 2, 4, 8])
    c["head_dim"] = rng.choice([64, 80, 128, 256])
    c["dtype"] = rng.choice(["bf16", "f16", "f32"])
    c["sequences"] = _log(rng, 1, 64)
    c["new_to"] = _log(rng, 1, 64)
    c["new_from"] = rng.randint(0, c["new_to"])
    c["kept"] = rng.randint(1, c["new_to"])
    most = max(1, 300_000_000 // (c["layers"] * c["kv_heads"] * c["head_dim"] * c["sequences"]) - c["new_to"] - pages)
    c["rows_to"] = _log(rng, 1, min(3000, most))
    c["rows_from"] = rng.randint(0, c["rows_to"])
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _sizes(c):
    """Rows and new tokens of each sequence, by the case alone."""
    rng = random.Random(c["shape"])
    rows = [rng.randint(c["rows_from"], c["rows_to"]) for _ in range(c["sequences"])]
    new = [1 if c.get("one_each") else rng.randint(c["new_from"], c["new_to"]) for _ in range(c["sequences"])]
    if sum(new) == 0:
        new[0] = 1
    return rows, new


def _parents(c, new, seed):
    """Parents within each sequence: mostly recent tokens, so that trees have branches and some depth."""
    rng = random.Random(seed * 7919 + 5)
    out = []
    for n in new:
        for j in range(n):
            if c.get("deep"):
                out.append(j - 1)
            else:
                out.append(-1 if j == 0 else max(0, j - rng.choice([1, 1, 2, 3, 5, 8, 13])))
    return out


def _ancestors(parents, new):
    """Of each token the numbers within its sequence that it sees."""
    out, at = [], 0
    for n in new:
        for j in range(n):
            p = parents[at + j]
            out.append([j] if p < 0 else out[at + p] + [j])
        at += n
    return out


def _words(new):
    return (max(new) + 63) // 64


def _starts(new):
    s = [0]
    for n in new:
        s.append(s[-1] + n)
    return s


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _pool(c, seed, rows, new):
    """Pages of one pool in a random order, [layers][pages][heads][page_rows][channels], and the sequences' tables."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    P = c["page_rows"]
    used = [(r + n + P - 1) // P for r, n in zip(rows, new)]
    pages, width = sum(used) + 3, max(max(used), 1) + 1
    shape = (c["layers"], pages, c["kv_heads"], P, c["head_dim"])
    k, v = (torch.empty(shape, dtype=_TORCH[c["dtype"]], device="cuda") for _ in range(2))
    for x in (k, v):
        for layer in range(c["layers"]):
            x[layer] = torch.randn(shape[1:], generator=g, device="cuda")
    rng = random.Random(seed * 31 + 2)
    order = list(range(pages))
    rng.shuffle(order)
    table = [[-1] * width for _ in used]
    at = 0
    for s, n in enumerate(used):
        table[s][:n] = order[at:at + n]
        at += n
        # pages that a conversation has let go, all of them in front of its new tokens
        for _ in range(c.get("holes", 0) if n > 2 and rows[s] >= P else 0):
            table[s][rng.randint(0, rows[s] // P - 1)] = -1
    return k, v, _ints(table)


def _radians(c):
    n = c["rotary_dim"]
    return c["base"] ** (-torch.arange(0, n, 2, dtype=torch.float64) / n)


def prepare(case, seed):
    c = dict(case)
    rows, new = _sizes(c)
    T, B = sum(new), len(new)
    s = {"c": c, "rows": rows, "new": new}
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 11)
    s["row_counts"], s["starts"] = _ints(rows), None if c.get("one_each") else _ints(_starts(new))
    if c["kind"] == "tree":
        s["parents"] = _ints(_parents(c, new, seed))
        rng = random.Random(seed + 1)
        s["first"] = _ints([rng.randint(0, 1000000) for _ in range(B)], torch.int64)
        s["mask"] = torch.empty((T, _words(new)), dtype=torch.int64, device="cuda")
        s["positions"] = torch.empty(T, dtype=torch.int64, device="cuda")
        return s
    s["k"], s["v"], s["table"] = _pool(c, seed, rows, new)
    if own:
        from paper_2510_18269_amd import oqm
        s["pages"] = oqm.Pages.create(s["k"], s["v"], s["table"], s["row_counts"], s["starts"])
    t, d, H, Hq = _TORCH[c["dtype"]], c["head_dim"], c["kv_heads"], c.get("q_heads", 0)
    if c["kind"] == "append":
        # what one projection gives: the query, key and value heads of a token beside each other
        x = torch.randn((T, Hq + 2 * H, d), generator=g, device="cuda").to(t)
        s["q"], s["new_k"], s["new_v"] = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
        s["q_out"] = torch.empty((T, Hq, d), dtype=t, device="cuda")
        s["q_norm"] = s["k_norm"] = None
        if c["norm"]:
            s["q_norm"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
            s["k_norm"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
        s["positions"] = _ints([c["first"] + j for n in new for j in range(n)], torch.int64)
        s["radians"] = _radians(c).cuda()
        if own:
            s["rotary"] = oqm.Rotary.create(c["rotary_dim"], layout=oqm.TOM_ROTARY_HALF if c["layout"] == "half" else oqm.TOM_ROTARY_PAIRS, base=c["base"])
        return s
    if c["kind"] == "attend":
        s["layer"] = c["layers"] - 1
        # queries as the turned rows lie: a token's heads beside each other
        s["q"] = torch.randn((T, Hq, d), generator=g, device="cuda").to(t).transpose(0, 1)
        s["out"] = torch.empty((T, Hq, d), dtype=t, device="cuda").transpose(0, 1)
        s["lse"] = torch.empty((Hq, T), dtype=torch.float32, device="cuda")
        s["mask"] = None
        if c["tree"]:
            words = [[0] * _words(new) for _ in range(T)]
            for i, seen in enumerate(_ancestors(_parents(c, new, seed), new)):
                for j in seen:
                    words[i][j // 64] |= 1 << (j % 64)
            s["mask"] = _ints([[w - (1 << 64) if w >> 63 else w for w in row] for row in words], torch.int64)
        s["prior_out"] = s["prior_lse"] = None
        if c["prior"]:
            # a part over some thousand stored tokens: averages, and the logarithm of a sum of as many exponentials
            s["prior_out"] = (0.05 * torch.randn((T, Hq, d), generator=g, device="cuda")).to(t).transpose(0, 1)
            s["prior_lse"] = 8.5 + 0.5 * torch.randn((Hq, T), generator=g, device="cuda")
        if own:
            size = oqm.tom_oqm_attend_pages_workspace_bytes(s["pages"], T, Hq)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        return s
    rng = random.Random(seed * 13 + 3)
    idx, counts = [], []
    for n in new:
        m = min(n, rng.randint(1, c["kept"]))
        idx.append(sorted(rng.sample(range(n), m)) + [0] * (c["kept"] - m))
        counts.append(m)
    s["idx"], s["counts"] = _ints(idx), _ints(counts)
    s["kept_rows"] = torch.empty(B, dtype=torch.int32, device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def _turned(x, norm, cos, sin, c):
    """x [T][heads][d] in 32 bits: each head's norm, then its pairs turned by (cos, sin) [T][1][rotary_dim / 2]."""
    x = x.float()
    if norm is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * norm.float()
    n = c["rotary_dim"]
    if c["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., n:]], -1)


def _places(s):
    """Of each new token the page and the row in it."""
    P, dev = s["c"]["page_rows"], "cuda"
    n = torch.tensor(s["new"], device=dev)
    which = torch.repeat_interleave(torch.arange(len(s["new"]), device=dev), n)
    row = s["row_counts"][which] + torch.arange(len(which), device=dev) - (torch.cumsum(n, 0) - n)[which]
    return s["table"][which, row // P].long(), row % P


def _run_tree(s):
    # all sequences padded to the longest; ancestors by squaring the matrix of parents, with ones on its diagonal
    new, words = s["new"], s["mask"].shape[1]
    N, B, dev = words * 64, len(new), "cuda"
    n = torch.tensor(new, device=dev)
    which = torch.repeat_interleave(torch.arange(B, device=dev), n)
    j = torch.arange(len(which), device=dev) - (torch.cumsum(n, 0) - n)[which]
    p = s["parents"].long()
    seen = torch.zeros((B, N, N), device=dev)
    seen[which, j, j] = 1.0
    seen[which, j, torch.where(p >= 0, p, j)] = 1.0
    length = 1
    while length < max(new):
        seen = (torch.bmm(seen, seen) > 0).float()
        length *= 2
    mine = seen[which, j]
    bits = mine.to(torch.int64).reshape(len(which), words, 64) << torch.arange(64, device=dev)
    s["mask"].copy_(bits.sum(-1))
    s["positions"].copy_(s["first"][which] + mine.sum(-1).to(torch.int64) - 1)
    return [s["mask"], s["positions"]]


def _run_attend(s):
    c = s["c"]
    H, R, d, P, layer = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["page_rows"], s["layer"]
    at = 0
    for i, (rows, n) in enumerate(zip(s["rows"], s["new"])):
        if n == 0:
            continue
        total = rows + n
        pages = s["table"][i, :(total + P - 1) // P]
        there = (pages >= 0).repeat_interleave(P)[:total]
        k, v = (x[layer].index_select(0, pages.clamp(min=0).long()).transpose(0, 1).reshape(H, -1, d)[:, :total].float() for x in (s["k"], s["v"]))
        q = s["q"][:, at:at + n].float().reshape(H, R * n, d)
        scores = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5
        if c["softcap"]:
            scores = c["softcap"] * torch.tanh(scores / c["softcap"])
        t, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        if c["tree"]:
            sees = (s["mask"][at:at + n][:, torch.arange(n, device="cuda") // 64] >> (j % 64)) & 1 > 0
        else:
            sees = j <= t if c["causal"] else (j >= 0).expand(n, -1)
        sees = torch.cat([torch.ones((n, rows), dtype=torch.bool, device="cuda"), sees], 1) & there
        scores = scores.reshape(H, R, n, total).masked_fill(~sees, -math.inf)
        top = scores.amax(-1, keepdim=True)
        if c["prior"]:
            before = s["prior_lse"][:, at:at + n].reshape(H, R, n, 1)
            top = torch.maximum(top, before)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.exp(scores - top)
        sums = p.sum(-1, keepdim=True)
        out = torch.bmm(p.reshape(H, R * n, total), v).reshape(H, R, n, d)
        if c["prior"]:
            weight = torch.exp(before - top)
            sums = sums + weight
            out = out + weight * s["prior_out"][:, at:at + n].float().reshape(H, R, n, d)
        out = out / torch.where(sums > 0, sums, torch.ones_like(sums))
        s["out"][:, at:at + n] = out.reshape(H * R, n, d).to(s["out"].dtype)
        s["lse"][:, at:at + n] = (top + torch.log(sums)).reshape(H * R, n)
        at += n
    return [s["out"], s["lse"]]


def run(s):
    c = s["c"]
    if own:
        from paper_2510_18269_amd import oqm
    if c["kind"] == "tree":
        if not own:
            return _run_tree(s)
        oqm.tom_oqm_draft_tree(s["parents"], s["starts"], s["mask"], positions=s["positions"], first=s["first"])
        return [s["mask"], s["positions"]]
    if c["kind"] == "append":
        if own:
            oqm.tom_oqm_append_rows(s["pages"], 1, s["rotary"], s["positions"], s["new_k"], s["new_v"], q=s["q"], q_out=s["q_out"], q_norm=s["q_norm"],
                                    k_norm=s["k_norm"], norm_eps=1e-6)
        else:
            angle = s["positions"].double()[:, None] * s["radians"][None]
            cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
            s["q_out"].copy_(_turned(s["q"], s["q_norm"], cos, sin, c))
            page, row = _places(s)
            s["k"][1, page, :, row] = _turned(s["new_k"], s["k_norm"], cos, sin, c).to(s["k"].dtype)
            s["v"][1, page, :, row] = s["new_v"]
        return [s["q_out"], s["k"], s["v"]]
    if c["kind"] == "attend":
        if not own:
            return _run_attend(s)
        oqm.tom_oqm_attend_pages(s["pages"], s["layer"], s["q"], s["out"], mask=s["mask"], causal=c["causal"], scale=c["head_dim"] ** -0.5, softcap=c["softcap"],
                                 prior_out=s["prior_out"], prior_lse=s["prior_lse"], lse=s["lse"], workspace=s["workspace"])
        return [s["out"], s["lse"]]
    if own:
        oqm.tom_oqm_keep_rows(s["pages"], s["idx"], s["counts"], s["kept_rows"])
    else:
        P = c["page_rows"]
        i = torch.arange(c["kept"], device="cuda")[None]
        kept = i < s["counts"][:, None]
        which = torch.arange(len(s["new"]), device="cuda")[:, None].expand_as(kept)[kept]
        to, source = (s["row_counts"][:, None] + i)[kept], (s["row_counts"][:, None] + s["idx"])[kept]
        for x in (s["k"], s["v"]):
            moved = x[:, s["table"][which, source // P].long(), :, source % P]
            x[:, s["table"][which, to // P].long(), :, to % P] = moved
        s["kept_rows"].copy_(s["row_counts"] + s["counts"])
    return [s["k"], s["v"], s["kept_rows"]]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(c):
    rows, new = _sizes(c)
    T, B = sum(new), len(new)
    e = 4 if c.get("dtype") == "f32" else 2
    starts = 0 if c.get("one_each") else 4 * (B + 1)
    if c["kind"] == "tree":
        return {"bytes": T * (4 + 8 + 8 * _words(new)) + starts + 8 * B, "flops": 0}
    if c["kind"] == "append":
        heads, turned = c["q_heads"] + 2 * c["kv_heads"], (c["q_heads"] + c["kv_heads"]) * T
        return {"bytes": 2 * e * heads * T * c["head_dim"] + 8 * T + starts + 8 * B,
                "flops": turned * (3 * c["rotary_dim"] + (4 * c["head_dim"] if c["norm"] else 0))}
    if c["kind"] == "attend":
        d, P = c["head_dim"], c["page_rows"]
        cached = sum(r + n for r, n in zip(rows, new) if n)
        holes = sum(min(c["holes"], r // P) * P for r, n in zip(rows, new) if n and (r + n + P - 1) // P > 2)
        mine = T * c["q_heads"] * (2 * d * e + 4) + (T * c["q_heads"] * (d * e + 4) if c["prior"] else 0)
        seen = 0
        for r, n in zip(rows, new):
            seen += n * r + (n if c["tree"] else n * (n + 1) // 2 if c["causal"] else n * n)
        return {"bytes": max(0, cached - holes) * 2 * c["kv_heads"] * d * e + mine + (8 * T * _words(new) if c["tree"] else 0) + starts + 4 * B
                + 4 * sum((r + n + P - 1) // P for r, n in zip(rows, new)), "flops": 4 * c["q_heads"] * d * max(0, seen - holes)}
    # on average half of what may be kept is
    moved = sum((min(n, c["kept"]) + 1) // 2 for n in new)
    return {"bytes": 2 * 2 * c["layers"] * c["kv_heads"] * c["head_dim"] * e * moved + 4 * B * (c["kept"] + 3) + starts, "flops": 0}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def _row_at(s, x, i, r):
    """Row r of sequence i in the pool x, all layers and heads; None where its page is not there."""
    page = s["tables"][i][r // s["c"]["page_rows"]]
    return None if page < 0 else x[:, page, :, r % s["c"]["page_rows"]]


def exact(c, seed):
    s = prepare(c, seed)
    new, rows = s["new"], s["rows"]
    if c["kind"] == "tree":
        parents, words = _parents(c, new, seed), _words(new)
        first = s["first"].tolist()
        masks, positions, at = [], [], 0
        for i, n in enumerate(new):
            for j in range(n):
                row, depth, p = [0] * words, -1, j
                while p >= 0:
                    row[p // 64] |= 1 << (p % 64)
                    depth += 1
                    p = parents[at + p]
                masks.append([w - (1 << 64) if w >= 1 << 63 else w for w in row])
                positions.append(first[i] + depth)
            at += n
        return [torch.tensor(masks, dtype=torch.int64), torch.tensor(positions, dtype=torch.int64)]
    s["tables"] = s["table"].tolist()
    d = c["head_dim"]
    if c["kind"] == "append":
        n = c["rotary_dim"]
        half = torch.arange(n // 2, device="cuda")
        one, two = (half, half + n // 2) if c["layout"] == "half" else (2 * half, 2 * half + 1)
        turn = torch.polar(torch.ones((sum(new), n // 2), dtype=torch.float64, device="cuda"), s["positions"].double().outer(_radians(c).cuda()))
        made = []
        for x, w in ((s["q"], s["q_norm"]), (s["new_k"], s["k_norm"])):
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for h in range(x.shape[1]):
                z = x[:, h].double()
                if w is not None:
                    z = z / torch.sqrt(z.square().sum(-1, keepdim=True) / d + 1e-6) * w.double()
                r = torch.complex(z[:, one], z[:, two]) * turn
                z = z.clone()
                z[:, one], z[:, two] = r.real, r.imag
                y[:, h] = z
            made.append(y)
        k, v, at = s["k"].double(), s["v"].double(), 0
        for i, m in enumerate(new):
            for j in range(m):
                page, row = s["tables"][i][(rows[i] + j) // c["page_rows"]], (rows[i] + j) % c["page_rows"]
                k[1, page, :, row] = made[1][at]
                v[1, page, :, row] = s["new_v"][at].double()
                at += 1
        return [made[0], k, v]
    if c["kind"] == "keep":
        k, v = s["k"].clone(), s["v"].clone()
        idx, counts = s["idx"].tolist(), s["counts"].tolist()
        for i, m in enumerate(counts):
            for j in range(m):
                for x, y in ((s["k"], k), (s["v"], v)):
                    _row_at(s, y, i, rows[i] + j).copy_(_row_at(s, x, i, rows[i] + idx[i][j]))
        return [k.double(), v.double(), torch.tensor([r + m for r, m in zip(rows, counts)], dtype=torch.int32)]
    H, Hq, P, T = c["kv_heads"], c["q_heads"], c["page_rows"], sum(new)
    out = torch.zeros((Hq, T, d), dtype=torch.float64, device="cuda")
    lse = torch.full((Hq, T), -math.inf, dtype=torch.float64, device="cuda")
    seen_new = _ancestors(_parents(c, new, seed), new) if c["tree"] else None
    at = 0
    for i, n in enumerate(new):
        total = rows[i] + n
        r = torch.arange(total, device="cuda")
        page = s["table"][i].long()[r // P]
        held = torch.nonzero(page >= 0).flatten()
        see = torch.ones((n, total), dtype=torch.bool, device="cuda")
        for t in range(n):
            if c["tree"]:
                see[t, rows[i]:] = False
                see[t, rows[i] + torch.tensor(seen_new[at + t], device="cuda")] = True
            elif c["causal"]:
                see[t, rows[i] + t + 1:] = False
        see = see[:, held]
        for h in range(H if n else 0):
            k, v = (x[s["layer"], page[held], h, held % P].double() for x in (s["k"], s["v"]))
            step = max(1, 40_000_000 // max(1, total))
            for g in range(h * Hq // H, (h + 1) * Hq // H):
                for t in range(0, n, step):
                    mine = torch.arange(t, min(t + step, n), device="cuda")
                    w = s["q"][g, at + mine].double() @ k.T / math.sqrt(d)
                    if c["softcap"]:
                        w = torch.tanh(w / c["softcap"]) * c["softcap"]
                    w = torch.where(see[mine], w, -math.inf)
                    if c["prior"]:
                        w = torch.cat([w, s["prior_lse"][g, at + mine].double()[:, None]], 1)
                    total_lse = torch.logsumexp(w, 1)
                    lse[g, at + mine] = total_lse
                    w = torch.exp(w - torch.where(total_lse == -math.inf, 0.0, total_lse)[:, None])
                    if c["prior"]:
                        out[g, at + mine] = w[:, :-1] @ v + w[:, -1:] * s["prior_out"][g, at + mine].double()
                    else:
                        out[g, at + mine] = w @ v
        at += n
    return [out, lse]
