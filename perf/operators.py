"""Performance cases of what a model does with the memory once frames are stored: turn its queries and keys to
their positions, attend over stored groups without unpacking them first, and drop or copy groups as the stream goes on.

Four kinds of pass:

  turn    rotary positions (with a norm of every head first, where asked) of queries and keys, and the new key
          and value rows written where the attention reads them; or a whole active key buffer turned again
  attend  new tokens over rows in front (system tokens or an active buffer), the selected 4-bit or 2-bit groups as
          they are stored, and recent rows, in one softmax
  keep    the groups of an ascending list move to the front of the storage, the others are dropped
  copy    groups of one memory appended to another

Sizes are those of the repository's workloads (28 layers, 4 KV heads of 128 channels, 28 query heads, frames of 196
or 50 tokens; the tiny stream of 64 channels its tests use) and generic ragged ones.
"""
import math

import numpy as np
import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

_TURN = {"kind": "turn", "tokens": 1, "q_heads": 28, "kv_heads": 4, "head_dim": 128, "rotary_dim": 128, "layout": "half",
         "norm": False, "values": True, "dtype": "bf16", "scaling": "none", "factor": 1.0, "original": 32768, "base": 1000000.0,
         "first": 0, "rows_after": 0}
_ATTEND = {"kind": "attend", "layers": 1, "kv_heads": 4, "q_heads": 28, "head_dim": 128, "tokens": 196, "qgroup": 64,
           "axis": "head_dim", "bits": 4, "meta": "f32", "dtype": "bf16", "stored": 0, "k": 0, "every": False, "holes": 0,
           "t_q": 1, "front": 0, "recent": 0, "causal": True, "softcap": 0.0, "outlier": False}
_GROUPS = {"layers": 28, "kv_heads": 4, "head_dim": 128, "tokens": 196, "qgroup": 64, "bits": 4, "meta": "f32", "stored": 0,
           "n": 0, "into": 0}


def listed():
    return [
        # one generated token of the 28-head model: norm, turn, and its key and value into the cache; latency
        {**_TURN, "name": "turn_token", "norm": True, "first": 12700, "rows_after": 255},
        # a long question late in an hour of video, positions scaled by parts, half of each head turned, interleaved
        {**_TURN, "name": "turn_question", "tokens": 1333, "rotary_dim": 64, "layout": "pairs", "dtype": "f16", "scaling": "by_parts",
         "factor": 24.0, "first": 705600},
        # the keys of a whole active buffer (28 layers x 4 heads x 64 frames) turned to their new places
        {**_TURN, "name": "turn_active", "tokens": 12544, "q_heads": 0, "kv_heads": 112, "values": False, "first": 14},
        # the tiny float32 stream of the tests: launches, hardly any data
        {**_ATTEND, "name": "attend_tiny", "kv_heads": 2, "q_heads": 2, "head_dim": 64, "tokens": 16, "qgroup": 32, "dtype": "f32",
         "stored": 32, "k": 4, "front": 3, "recent": 5},
        # one generated token over what a question retrieved: 64 of 1024 frames, system tokens, question and answer so far
        {**_ATTEND, "name": "attend_token", "layers": 2, "stored": 256, "k": 64, "front": 14, "recent": 57},
        # the paper's own setting: 50 tokens a frame, quantized along the tokens, binary16, everything in the budget
        {**_ATTEND, "name": "attend_token_axis", "tokens": 50, "axis": "tokens", "dtype": "f16", "stored": 64, "k": 64, "every": True,
         "front": 14, "recent": 33},
        # one generated token over the active buffer that a retrieval left, 16-bit rows alone
        {**_ATTEND, "name": "attend_rows", "front": 12558, "recent": 40},
        # one generated token over the whole hour: 3600 frames, 705600 tokens
        {**_ATTEND, "name": "attend_hour", "stored": 3600, "k": 3600, "every": True, "front": 14, "recent": 64},
        # a question of 64 tokens over 128 frames with outlier keys and groups of 32
        {**_ATTEND, "name": "attend_question", "qgroup": 32, "stored": 256, "k": 128, "front": 14, "recent": 64, "t_q": 64, "outlier": True},
        # a long prompt over its own rows and 32 retrieved frames, scores capped
        {**_ATTEND, "name": "attend_prompt", "stored": 64, "k": 32, "front": 14, "recent": 1000, "t_q": 1000, "softcap": 30.0},
        # every fourth frame of a full memory leaves, all layers
        {**_GROUPS, "kind": "keep", "name": "keep_frames", "stored": 128, "n": 96},
        # a short conversation forks: a few frames of a small memory into another
        {**_GROUPS, "kind": "copy", "name": "copy_frames", "layers": 4, "tokens": 50, "stored": 64, "n": 9, "into": 5},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["turn", "attend", "attend", "attend", "keep", "copy"])
    if kind == "turn":
        c = dict(_TURN)
        c["head_dim"] = rng.choice([64, 80, 96, 128, 128, 256])
        c["rotary_dim"] = rng.choice([c["head_dim"], c["head_dim"], c["head_dim"] // 2, 2 * rng.randint(1, c["head_dim"] // 2)])
        c["layout"] = rng.choice(["half", "pairs"])
        c["kv_heads"] = rng.choice([1, 2, 4, 8])
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 7])
        c["tokens"] = _log(rng, 1, 6000)
        c["norm"], c["values"] = rng.random() < 0.5, rng.random() < 0.7
        c["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["scaling"] = rng.choice(["none", "linear", "base", "by_parts", "by_wavelength"])
        c["factor"] = 1.0 if c["scaling"] == "none" else rng.choice([2.0, 4.0, 8.5, 32.0])
        c["original"] = rng.choice([4096, 8192, 32768])
        c["base"] = rng.choice([10000.0, 500000.0, 1000000.0])
        c["first"] = rng.choice([0, rng.randint(0, 5000), rng.randint(0, 1000000)])
        c["rows_after"] = rng.choice([0, rng.randint(1, 300)])
        if c["scaling"] == "base" and c["rotary_dim"] < 4:
            c["rotary_dim"] = 4
        return c
    if kind == "attend":
        c = dict(_ATTEND)
        c["head_dim"] = rng.choice([64, 128, 128, 128, 256])
        c["kv_heads"] = rng.choice([1, 2, 4, 4, 8])
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 7, 8])
        c["tokens"] = rng.choice([196, 50, _log(rng, 1, 300), _log(rng, 1, 300)])
        c["qgroup"] = rng.choice([g for g in (8, 16, 32, 64, 64, 128) if g <= c["head_dim"]])
        c["axis"] = rng.choice(["head_dim", "head_dim", "tokens"])
        c["bits"], c["meta"] = rng.choice([4, 4, 4, 2]), rng.choice(["f32", "f32", "bf16"])
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
        c["t_q"] = rng.choice([1, 1, _log(rng, 1, 200)])
        most = 40000 if c["t_q"] == 1 else 600000 // c["t_q"] + 200
        c["k"] = max(0, min(_log(rng, 1, 800), most // c["tokens"]))
        c["every"] = rng.random() < 0.3
        c["stored"] = c["k"] if c["every"] else c["k"] + rng.randint(0, 40)
        c["holes"] = rng.choice([0, 0, 0, min(2, c["k"])]) if not c["every"] else 0
        c["front"] = rng.choice([0, 14, _log(rng, 1, 2000)])
        c["recent"] = rng.choice([c["t_q"], c["t_q"] + rng.randint(0, 300), rng.randint(1, 2 * c["t_q"])])
        c["causal"] = rng.random() < 0.8
        c["softcap"] = rng.choice([0.0, 0.0, 20.0, 50.0])
        c["outlier"] = rng.random() < 0.2
        c["layers"] = rng.choice([1, 2, 3])
        return c
    c = {**_GROUPS, "kind": kind}
    c["layers"] = rng.choice([1, 2, 4, 28])
    c["kv_heads"] = rng.choice([1, 2, 4])
    c["head_dim"] = rng.choice([64, 96, 128])
    c["tokens"] = rng.choice([50, 196, _log(rng, 1, 200)])
    c["qgroup"] = rng.choice([8, 16, 32])
    c["bits"], c["meta"] = rng.choice([4, 2]), rng.choice(["f32", "bf16"])
    frame = c["layers"] * 2 * c["kv_heads"] * c["tokens"] * c["head_dim"]
    c["stored"] = _log(rng, 2, max(3, min(2000, 300_000_000 // frame)))
    c["n"] = rng.randint(1, c["stored"])
    c["into"] = rng.randint(0, 20) if kind == "copy" else 0
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + salt)
    return g


def _quantize(x, c):
    """Codes and (scale, zero) pairs of x [T][H][G][d] as the memory stores them."""
    T, H, G, d = x.shape
    levels = 2 ** c["bits"] - 1
    if c.get("axis", "head_dim") == "head_dim":
        g = x.reshape(T, H, G, d // c["qgroup"], c["qgroup"])
        lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    else:
        g = x
        lo, hi = g.amin(2, keepdim=True), g.amax(2, keepdim=True)
    s = (hi - lo) / levels
    if c["meta"] == "bf16":
        s, lo = s.bfloat16().float(), lo.bfloat16().float()
    q = torch.where(s > 0, torch.round((g - lo) / s), torch.zeros_like(g)).clamp_(0, levels).to(torch.uint8).reshape(T, H, G, d)
    if c["bits"] == 4:
        codes = q[..., 0::2] | (q[..., 1::2] << 4)
    else:
        codes = q[..., 0::4] | (q[..., 1::4] << 2) | (q[..., 2::4] << 4) | (q[..., 3::4] << 6)
    pairs = torch.stack([s, lo], -1)
    pairs = pairs.reshape(T, H, -1, 2)
    return codes, pairs.bfloat16() if c["meta"] == "bf16" else pairs


def _storage(c, seed, groups, capacity, salt=0):
    """The three arrays of a memory with `groups` frames in it, shaped [L][2][T_cap][...] and [L][T_cap][H][d]."""
    g = _generator(seed, 17 + salt)
    L, H, G, d = c["layers"], c["kv_heads"], c["tokens"], c["head_dim"]
    m = d // c["qgroup"] * G if c.get("axis", "head_dim") == "head_dim" else d
    codes = torch.zeros((L, 2, capacity, H, G, d * c["bits"] // 8), dtype=torch.uint8, device="cuda")
    meta = torch.zeros((L, 2, capacity, H, m, 2), dtype=torch.bfloat16 if c["meta"] == "bf16" else torch.float32, device="cuda")
    keys = torch.zeros((L, capacity, H, d), dtype=torch.float32, device="cuda")
    step = max(1, 30_000_000 // (H * G * d))
    for layer in range(L):
        for kv in range(2):
            for t in range(0, groups, step):
                n = min(step, groups - t)
                x = torch.randn((n, H, G, d), generator=g, device="cuda") * (0.7 + 0.4 * ((layer + kv) % 3))
                if c.get("outlier") and kv == 0:
                    x[..., 3::32] *= 20.0
                codes[layer, kv, t:t + n], meta[layer, kv, t:t + n] = _quantize(x, c)
                if kv == 0:
                    keys[layer, t:t + n] = x.mean(2)
    return codes, meta, keys


def _memory(c, codes, meta, keys, groups):
    """The handle of a memory on these arrays, as a program keeps it for the life of a stream."""
    from paper_2510_18269_amd import oqm
    dtype = {"f32": oqm.TOM_F32, "bf16": oqm.TOM_BF16, "f16": oqm.TOM_F16}
    axis = oqm.TOM_QAXIS_TOKENS if c.get("axis") == "tokens" else oqm.TOM_QAXIS_HEAD_DIM
    io = dtype[c.get("dtype", "bf16")]
    cfg = oqm.make_config(c["layers"], c["kv_heads"], c.get("q_heads", c["kv_heads"]), c["head_dim"], c["tokens"], c["qgroup"],
                          codes.shape[2], qaxis=axis, bits=c["bits"], in_dtype=io, out_dtype=io, meta_dtype=dtype[c["meta"]])
    handle = oqm.tom_oqm_create(cfg)
    oqm.tom_oqm_bind(handle, codes, meta, keys)
    oqm.tom_oqm_set_num_groups(handle, groups)
    return oqm.Memory(cfg, handle, codes, meta, keys)


def _frequencies(c):
    """Radians a position turns each pair by, in 64 bits, and the factor on the turned channels."""
    n = c["rotary_dim"]
    i = torch.arange(0, n, 2, dtype=torch.float64)
    base, factor, original = c["base"], c["factor"], c["original"]
    if c["scaling"] == "base":
        base = base * factor ** (n / (n - 2))
    f = base ** (-i / n)
    if c["scaling"] == "linear":
        f = f / factor
    if c["scaling"] == "by_parts":
        # pairs that turn over 32 times within the original length stay, those under once are stretched
        turns = original * f / (2 * math.pi)
        place = lambda r: n * math.log(original / (r * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(place(32.0)), 0), min(math.ceil(place(1.0)), n - 1)
        stretched = ((torch.arange(n // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f * (1 - stretched) + f / factor * stretched
        assert turns.numel() == n // 2
        return f, 0.1 * math.log(factor) + 1.0
    if c["scaling"] == "by_wavelength":
        # wavelengths under original / 4 stay, those over original are stretched, between them a straight line
        kept = ((original * f / (2 * math.pi) - 1.0) / 3.0).clamp(0, 1)
        f = f * kept + f / factor * (1 - kept)
    return f, 1.0


def prepare(case, seed):
    c = dict(case)
    s = {"c": c}
    if c["kind"] == "turn":
        g = _generator(seed, 3)
        T, d, t = c["tokens"], c["head_dim"], _TORCH[c["dtype"]]
        n = c["q_heads"] + 2 * c["kv_heads"]
        if c["q_heads"]:
            # what one projection gives: the query, key and value heads of a token beside each other
            x = torch.randn((T, n, d), generator=g, device="cuda").to(t)
            s["q"], s["k"], s["v"] = x[:, :c["q_heads"]], x[:, c["q_heads"]:c["q_heads"] + c["kv_heads"]], x[:, c["q_heads"] + c["kv_heads"]:]
            s["q_out"] = torch.empty((T, c["q_heads"], d), dtype=t, device="cuda")
        else:
            s["q"] = s["q_out"] = s["v"] = None
            s["k"] = torch.randn((c["kv_heads"], T, d), generator=g, device="cuda").to(t).transpose(0, 1)  # an active buffer, by heads
        rows = T + c["rows_after"]
        s["k_out"] = torch.zeros((c["kv_heads"], rows, d), dtype=t, device="cuda")
        s["v_out"] = torch.zeros((c["kv_heads"], rows, d), dtype=t, device="cuda") if c["values"] else None
        s["q_norm"] = s["k_norm"] = None
        if c["norm"]:
            s["q_norm"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
            s["k_norm"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
        s["positions"] = c["first"] + torch.arange(T, device="cuda", dtype=torch.int64)
        f, s["factor"] = _frequencies(c)
        s["radians"] = f.cuda()
        if own:
            from paper_2510_18269_amd import oqm
            scaling = {"none": oqm.TOM_ROTARY_PLAIN, "linear": oqm.TOM_ROTARY_LINEAR, "base": oqm.TOM_ROTARY_BASE,
                       "by_parts": oqm.TOM_ROTARY_BY_PARTS, "by_wavelength": oqm.TOM_ROTARY_BY_WAVELENGTH}[c["scaling"]]
            s["rotary"] = oqm.Rotary.create(c["rotary_dim"], layout=oqm.TOM_ROTARY_HALF if c["layout"] == "half" else oqm.TOM_ROTARY_PAIRS,
                                            base=c["base"], scaling=scaling, factor=c["factor"], original_length=c["original"])
        return s
    if c["kind"] == "attend":
        codes, meta, keys = _storage(c, seed, c["stored"], max(1, c["stored"]))
        g = _generator(seed, 5)
        t, d, H = _TORCH[c["dtype"]], c["head_dim"], c["kv_heads"]
        s["codes"], s["meta"], s["keys"] = codes, meta, keys
        s["layer"] = c["layers"] - 1
        # queries as the turned rows lie: a token's heads beside each other
        s["q"] = torch.randn((c["t_q"], c["q_heads"], d), generator=g, device="cuda").to(t).transpose(0, 1)
        s["out"] = torch.empty((c["t_q"], c["q_heads"], d), dtype=t, device="cuda").transpose(0, 1)
        s["lse"] = torch.empty((c["q_heads"], c["t_q"]), dtype=torch.float32, device="cuda")
        for name in ("front", "recent"):
            rows = c[name] + (37 if name == "recent" else 0)  # the recent rows stand in a cache with room for more
            for kv in ("k", "v"):
                x = torch.randn((H, rows, d), generator=g, device="cuda").to(t)
                s["%s_%s" % (name, kv)] = x[:, :c[name]] if c[name] else None
        s["idx"] = None
        if c["k"] and not c["every"]:
            order = torch.randperm(c["stored"], generator=g, device="cuda")[:c["k"]].sort().values.to(torch.int32)
            if c["holes"]:
                order[torch.randperm(c["k"], generator=g, device="cuda")[:c["holes"]]] = -1
            s["idx"] = order
        if own:
            from paper_2510_18269_amd import oqm
            s["memory"] = _memory(c, codes, meta, keys, c["stored"])
            rows = c["front"] + c["k"] * c["tokens"] + c["recent"]
            s["workspace"] = torch.empty(oqm.tom_oqm_attend_workspace_bytes(s["memory"].handle, c["t_q"], rows), dtype=torch.uint8, device="cuda")
        return s
    s["codes"], s["meta"], s["keys"] = _storage(c, seed, c["stored"], c["stored"])
    rng = np.random.RandomState(seed % (1 << 31))
    chosen = np.sort(rng.permutation(c["stored"])[:c["n"]]) if c["kind"] == "keep" else rng.randint(0, c["stored"], c["n"])
    s["idx"] = torch.from_numpy(chosen.astype(np.int32)).cuda()
    if c["kind"] == "copy":
        s["to_codes"], s["to_meta"], s["to_keys"] = _storage(c, seed, c["into"], c["into"] + c["n"], salt=4)
    if own:
        s["memory"] = _memory(c, s["codes"], s["meta"], s["keys"], c["stored"])
        if c["kind"] == "copy":
            s["to"] = _memory(c, s["to_codes"], s["to_meta"], s["to_keys"], c["into"])
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


def _values(s, kv):
    """The selected groups' values in 32 bits, [H][k * G][d], code * scale + zero."""
    c, layer = s["c"], s["layer"]
    H, G, d = c["kv_heads"], c["tokens"], c["head_dim"]
    codes, meta = s["codes"][layer, kv, :c["k"]], s["meta"][layer, kv, :c["k"]]
    if s["idx"] is not None:
        at = s["idx"].clamp(min=0).long()
        codes, meta = s["codes"][layer, kv].index_select(0, at), s["meta"][layer, kv].index_select(0, at)
    if c["bits"] == 4:
        x = torch.stack([codes & 15, codes >> 4], -1)
    else:
        x = torch.stack([codes & 3, (codes >> 2) & 3, (codes >> 4) & 3, codes >> 6], -1)
    x = x.reshape(c["k"], H, G, d).float()
    meta = meta.float()
    if c["axis"] == "head_dim":
        p = meta.reshape(c["k"], H, G, d // c["qgroup"], 1, 2)
        x = x.reshape(c["k"], H, G, d // c["qgroup"], c["qgroup"]) * p[..., 0] + p[..., 1]
    else:
        p = meta.reshape(c["k"], H, 1, d, 2)
        x = x * p[..., 0] + p[..., 1]
    return x.reshape(c["k"], H, G, d).transpose(0, 1).reshape(H, c["k"] * G, d)


def _visible(s):
    """[t_q][rows]: what each new token sees.  Rows in front and groups are for all, a hole in the list is for none, and
    of the recent rows a token sees those up to its own, which are the last t_q where the call is causal."""
    c = s["c"]
    t = torch.arange(c["t_q"], device="cuda")[:, None]
    front = torch.ones((c["t_q"], c["front"]), dtype=torch.bool, device="cuda")
    there = torch.ones(c["k"], dtype=torch.bool, device="cuda") if s["idx"] is None else s["idx"] >= 0
    groups = there.repeat_interleave(c["tokens"])[None].expand(c["t_q"], -1)
    j = torch.arange(c["recent"], device="cuda")[None]
    recent = j <= t + (c["recent"] - c["t_q"]) if c["causal"] else (j >= 0).expand(c["t_q"], -1)
    return torch.cat([front, groups, recent], 1)


def run(s):
    c = s["c"]
    if c["kind"] == "turn":
        if own:
            from paper_2510_18269_amd import oqm
            oqm.tom_oqm_rotate(s["rotary"], s["positions"], q=s["q"], q_out=s["q_out"], k=s["k"], k_out=s["k_out"][:, c["rows_after"]:].transpose(0, 1),
                               v=s["v"] if c["values"] else None, v_out=s["v_out"][:, c["rows_after"]:].transpose(0, 1) if c["values"] else None,
                               q_norm=s["q_norm"], k_norm=s["k_norm"], norm_eps=1e-6)
        else:
            angle = s["positions"].double()[:, None] * s["radians"][None]
            cos = (torch.cos(angle) * s["factor"]).float()[:, None]
            sin = (torch.sin(angle) * s["factor"]).float()[:, None]
            if s["q"] is not None:
                s["q_out"].copy_(_turned(s["q"], s["q_norm"], cos, sin, c))
            s["k_out"][:, c["rows_after"]:] = _turned(s["k"], s["k_norm"], cos, sin, c).transpose(0, 1).to(s["k_out"].dtype)
            if c["values"]:
                s["v_out"][:, c["rows_after"]:] = s["v"].transpose(0, 1)
        return [x for x in (s["q_out"], s["k_out"], s["v_out"]) if x is not None]
    if c["kind"] == "attend":
        if own:
            from paper_2510_18269_amd import oqm
            oqm.tom_oqm_attend(s["memory"].handle, s["layer"], s["q"], s["out"], idx=s["idx"], k_eff=c["k"], front_k=s["front_k"],
                               front_v=s["front_v"], recent_k=s["recent_k"], recent_v=s["recent_v"], causal=c["causal"],
                               scale=c["head_dim"] ** -0.5, softcap=c["softcap"], lse=s["lse"], workspace=s["workspace"])
            return [s["out"], s["lse"]]
        H, R, d = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"]
        parts = [[s["front_%s" % n], s["recent_%s" % n]] for n in ("k", "v")]
        k, v = (torch.cat([x.float() for x in (p[0], _values(s, i) if c["k"] else None, p[1]) if x is not None], 1) for i, p in enumerate(parts))
        q = s["q"].float().reshape(H, R * c["t_q"], d)
        scores = torch.bmm(q, k.transpose(1, 2).contiguous()) * c["head_dim"] ** -0.5
        if c["softcap"]:
            scores = c["softcap"] * torch.tanh(scores / c["softcap"])
        scores = scores.reshape(H, R, c["t_q"], -1).masked_fill(~_visible(s), -math.inf)
        top = scores.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.exp(scores - top)
        total = p.sum(-1, keepdim=True)
        out = torch.bmm(p.reshape(H, R * c["t_q"], -1), v).reshape(H, R, c["t_q"], d) / torch.where(total > 0, total, torch.ones_like(total))
        s["out"].copy_(out.reshape(H * R, c["t_q"], d))
        s["lse"].copy_((top + torch.log(total)).reshape(H * R, c["t_q"]))
        return [s["out"], s["lse"]]
    names = ("codes", "meta", "keys")
    if c["kind"] == "keep":
        if own:
            from paper_2510_18269_amd import oqm
            oqm.tom_oqm_set_num_groups(s["memory"].handle, c["stored"])
            oqm.tom_oqm_keep_groups(s["memory"].handle, s["idx"], c["n"])
        else:
            at = s["idx"].long()
            s["codes"][:, :, :c["n"]] = s["codes"].index_select(2, at)
            s["meta"][:, :, :c["n"]] = s["meta"].index_select(2, at)
            s["keys"][:, :c["n"]] = s["keys"].index_select(1, at)
        return [s[n] for n in names]
    if own:
        from paper_2510_18269_amd import oqm
        oqm.tom_oqm_set_num_groups(s["to"].handle, c["into"])
        oqm.tom_oqm_copy_groups(s["to"].handle, s["memory"].handle, s["idx"], c["n"])
    else:
        at = s["idx"].long()
        s["to_codes"][:, :, c["into"]:] = s["codes"].index_select(2, at)
        s["to_meta"][:, :, c["into"]:] = s["meta"].index_select(2, at)
        s["to_keys"][:, c["into"]:] = s["keys"].index_select(1, at)
    return [s["to_" + n] for n in names]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(c):
    if c["kind"] == "turn":
        e = 4 if c["dtype"] == "f32" else 2
        heads = c["q_heads"] + c["kv_heads"] * (2 if c["values"] else 1)
        turned = (c["q_heads"] + c["kv_heads"]) * c["tokens"]
        return {"bytes": 2 * e * heads * c["tokens"] * c["head_dim"] + 8 * c["tokens"] + 8 * c["rotary_dim"] // 2,
                "flops": turned * (3 * c["rotary_dim"] + (4 * c["head_dim"] if c["norm"] else 0))}
    if c["kind"] == "attend":
        e = 4 if c["dtype"] == "f32" else 2
        H, d, G, k = c["kv_heads"], c["head_dim"], c["tokens"], c["k"] - c["holes"]
        pairs = G * d // c["qgroup"] if c["axis"] == "head_dim" else d
        group = H * 2 * (G * d * c["bits"] // 8 + pairs * (8 if c["meta"] == "f32" else 4))
        rows = H * d * 2 * e * (c["front"] + c["recent"])
        own_rows = c["t_q"] * c["q_heads"] * (2 * d * e + 4)
        if c["causal"]:
            seen = sum(max(0, min(c["recent"], t + 1 + c["recent"] - c["t_q"])) for t in range(c["t_q"]))
        else:
            seen = c["t_q"] * c["recent"]
        seen += c["t_q"] * (c["front"] + k * G)
        return {"bytes": group * k + rows + own_rows + (0 if c["every"] else 4 * c["k"]), "flops": 4 * c["q_heads"] * d * seen}
    frame = c["layers"] * c["kv_heads"] * (2 * c["tokens"] * (c["head_dim"] * c["bits"] // 8 + c["head_dim"] // c["qgroup"] * (8 if c["meta"] == "f32" else 4))
                                           + 4 * c["head_dim"])
    return {"bytes": 2 * frame * c["n"] + 4 * c["n"], "flops": 0}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] in ("keep", "copy"):
        n = c["n"]
        to = "to_" if c["kind"] == "copy" else ""
        result = []
        for name in ("codes", "meta", "keys"):
            source, target = s[name].cpu(), s[to + name].cpu().clone()
            for i, t in enumerate(s["idx"].tolist()):
                if name == "keys":
                    target[:, c["into"] + i] = source[:, t]
                else:
                    target[:, :, c["into"] + i] = source[:, :, t]
            assert target.shape[1 if name == "keys" else 2] >= c["into"] + n
            result.append(target.to(torch.int64) if name == "codes" else target.double())
        return result
    if c["kind"] == "turn":
        n, d = c["rotary_dim"], c["head_dim"]
        half = torch.arange(n // 2, device="cuda")
        one, two = (half, half + n // 2) if c["layout"] == "half" else (2 * half, 2 * half + 1)
        f, factor = _frequencies(c)
        turn = torch.polar(torch.full((c["tokens"], n // 2), float(factor), dtype=torch.float64, device="cuda"),
                           s["positions"].double().outer(f.cuda()))
        result = []
        for x, w, out in ((s["q"], s["q_norm"], s["q_out"]), (s["k"], s["k_norm"], s["k_out"]), (s["v"], None, s["v_out"])):
            if out is None:
                continue
            y = torch.zeros(out.shape, dtype=torch.float64, device="cuda")
            for h in range(x.shape[1]):
                z = x[:, h].double()
                if w is not None:
                    z = z / torch.sqrt(z.square().sum(-1, keepdim=True) / d + 1e-6) * w.double()
                if out is not s["v_out"]:
                    r = torch.complex(z[:, one], z[:, two]) * turn
                    z = z.clone()
                    z[:, one], z[:, two] = r.real, r.imag
                if out is s["q_out"]:
                    y[:, h] = z
                else:
                    y[h, c["rows_after"]:] = z
            result.append(y)
        return result
    H, R, d, G = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["tokens"]
    groups = list(range(c["k"])) if s["idx"] is None else [t for t in s["idx"].tolist() if t >= 0]
    out = torch.zeros((H * R, c["t_q"], d), dtype=torch.float64, device="cuda")
    lse = torch.full((H * R, c["t_q"]), -math.inf, dtype=torch.float64, device="cuda")
    at = torch.tensor(groups, dtype=torch.int64, device="cuda")
    shift = torch.arange(0, 8, c["bits"], device="cuda")
    for h in range(H):
        both = []
        for kv, name in ((0, "k"), (1, "v")):
            x = s["codes"][s["layer"], kv, :, h][at].to(torch.int64)[..., None]
            x = ((x >> shift) & (2 ** c["bits"] - 1)).reshape(len(groups), G, d).double()
            m = s["meta"][s["layer"], kv, :, h][at].double()
            if c["axis"] == "head_dim":
                m = m.reshape(len(groups), G, d // c["qgroup"], 2).repeat_interleave(c["qgroup"], 2)
            else:
                m = m.reshape(len(groups), 1, d, 2)
            x = (m[..., 0] * x + m[..., 1]).reshape(-1, d)
            rows = [s["%s_%s" % (part, name)] for part in ("front", "recent")]
            rows = [torch.zeros((0, d), dtype=torch.float64, device="cuda") if r is None else r[h].double() for r in rows]
            both.append(torch.cat([rows[0], x, rows[1]]))
        fixed = c["front"] + len(groups) * G
        step = max(1, 40_000_000 // max(1, both[0].shape[0]))
        for r in range(h * R, h * R + R):
            for t in range(0, c["t_q"], step):
                mine = torch.arange(t, min(t + step, c["t_q"]), device="cuda")
                w = s["q"][r, mine].double() @ both[0].T / math.sqrt(d)
                if c["softcap"]:
                    w = torch.tanh(w / c["softcap"]) * c["softcap"]
                if c["causal"]:
                    last = fixed + c["recent"] - c["t_q"] + mine
                    w[torch.arange(both[0].shape[0], device="cuda")[None] > last.clamp(min=fixed - 1)[:, None]] = -math.inf
                lse[r, mine] = torch.logsumexp(w, 1)
                w = torch.exp(w - torch.where(lse[r, mine] == -math.inf, 0.0, lse[r, mine])[:, None])
                out[r, mine] = w @ both[1]
    return [out, lse]
