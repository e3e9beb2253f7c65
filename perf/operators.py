"""The serving operators between the quantized projections of a decoder block, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` names the operator:

  append    queries and keys of new tokens normalised (or not) and rotated, keys and values stored in a paged cache
            (aser_kv_append)
  decode    attention of one or a few new tokens per request over the paged cache (aser_paged_attention)
  prompt    the same call for prompts: thousands of new tokens, with or without earlier ones in the cache
  adapters  low-rank adapters of many requests beside a shared projection (aser_adapter_forward)

Head counts and widths are those of the blocks this library is measured on (32 query heads of 128 channels, 8 or 32
key/value heads, hidden width 4096, MLP width 14336) or generic.  Lengths of the requests of a batch follow from the
case alone; values, the order of the pages in the cache and the numbering of the adapters come from the seed.

The plain forms compute in 32 bits and round once to the type of the output.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # one request decodes its next token: launches and latency
        {"name": "append_decode_1", "kind": "append", "seqs": 1, "new": 1, "past": 1023, "heads": 32, "kv_heads": 8, "d": 128, "page": 64,
         "x": "f32", "norm": False, "style": "half", "rot": 128},
        # a batch of requests decodes, bf16 projections, query/key norms
        {"name": "append_decode_96", "kind": "append", "seqs": 96, "new": 1, "past": 2049, "heads": 32, "kv_heads": 8, "d": 128, "page": 32,
         "x": "bf16", "norm": True, "style": "half", "rot": 128},
        # ragged prompts, straight from the fp32 output of the compensated projections
        {"name": "append_prompt_ragged", "kind": "append", "seqs": 5, "new": 3400, "past": 0, "heads": 32, "kv_heads": 8, "d": 128, "page": 64,
         "x": "f32", "norm": True, "style": "half", "rot": 128},
        # one request decodes far into its context: few rows, a long axis
        {"name": "decode_1_long", "kind": "decode", "seqs": 1, "new": 1, "kv": 32771, "ragged": False, "heads": 32, "kv_heads": 8, "d": 128, "page": 64,
         "cache": "bf16", "window": 0, "sinks": 0},
        # a ragged batch of requests decodes, the ordinary load
        {"name": "decode_64_ragged", "kind": "decode", "seqs": 64, "new": 1, "kv": 8192, "ragged": True, "heads": 32, "kv_heads": 8, "d": 128, "page": 64,
         "cache": "bf16", "window": 0, "sinks": 0},
        # the cache held in 8 bits, small pages, narrower heads
        {"name": "decode_40_int8", "kind": "decode", "seqs": 40, "new": 1, "kv": 12003, "ragged": True, "heads": 32, "kv_heads": 8, "d": 64, "page": 16,
         "cache": "int8", "window": 0, "sinks": 0},
        # a key/value head for every query head, a window with sinks over a long cache, four tokens at once
        {"name": "decode_16_window", "kind": "decode", "seqs": 16, "new": 4, "kv": 9001, "ragged": True, "heads": 32, "kv_heads": 32, "d": 128, "page": 32,
         "cache": "bf16", "window": 2048, "sinks": 4},
        # one long prompt
        {"name": "prompt_8192", "kind": "prompt", "seqs": 1, "new": 8192, "past": 0, "ragged": False, "heads": 32, "kv_heads": 8, "d": 128, "page": 64,
         "cache": "bf16", "window": 0, "sinks": 0},
        # ragged pieces of prompts behind earlier ones, cache in 8 bits
        {"name": "prompt_4_int8", "kind": "prompt", "seqs": 4, "new": 777, "past": 3001, "ragged": True, "heads": 32, "kv_heads": 8, "d": 64, "page": 16,
         "cache": "int8", "window": 0, "sinks": 0},
        # prompts under a window with sinks
        {"name": "prompt_2_window", "kind": "prompt", "seqs": 2, "new": 6001, "past": 0, "ragged": True, "heads": 32, "kv_heads": 8, "d": 128, "page": 32,
         "cache": "bf16", "window": 1024, "sinks": 4},
        # a decoding batch, most requests with an adapter, beside an attention projection
        {"name": "adapters_decode_48", "kind": "adapters", "rows": 48, "run": 1, "n": 4096, "m": 4096, "r": 16, "adapters": 16, "bare": 7, "x": "bf16"},
        # prompts of several requests beside a wide projection
        {"name": "adapters_prompt_4099", "kind": "adapters", "rows": 4099, "run": 513, "n": 4096, "m": 14336, "r": 64, "adapters": 6, "bare": 4, "x": "f32"},
    ]


# ------------------------------------------------------------------------------------------------ more cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "prompt", "prompt", "adapters"])
    if kind == "adapters":
        rows = _log(rng, 1, 6000)
        n, m = _log(rng, 256, 8192), _log(rng, 256, 8192)
        if rng.random() < 0.7:                                  # widths of models, otherwise odd ones
            n, m = max(256, n // 128 * 128), max(256, m // 128 * 128)
        return {"kind": kind, "rows": rows, "run": _log(rng, 1, max(1, rows // 2)), "n": n, "m": m, "r": rng.choice([4, 8, 13, 16, 32, 64, 128]),
                "adapters": _log(rng, 1, 24), "bare": rng.choice([0, 3, 5, 9]), "x": rng.choice(["bf16", "f32"])}
    d = rng.choice([64, 128, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 4, 4, 8])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        decode = rng.random() < 0.5
        seqs = _log(rng, 1, 128) if decode else _log(rng, 1, 6)
        return {"kind": kind, "seqs": seqs, "new": 1 if decode else _log(rng, 16, 12000 // seqs), "past": _log(rng, 1, 4000), "heads": heads,
                "kv_heads": kv_heads, "d": d, "page": page, "x": rng.choice(["bf16", "f32"]), "norm": rng.random() < 0.5,
                "style": rng.choice(["half", "pairs"]), "rot": rng.choice([d, d, d // 2])}
    window = rng.choice([0, 0, _log(rng, 16, 4096)])
    more = {"ragged": True, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "cache": rng.choice(["bf16", "bf16", "int8"]),
            "window": window, "sinks": rng.choice([0, 4, 17]) if window else 0}
    if kind == "decode":
        seqs = _log(rng, 1, 128)
        most = min(60000, (64 * 8192 * 8 * 128) // (seqs * kv_heads * d))
        new = rng.choice([1, 1, 1, 3])
        return {"kind": kind, "seqs": seqs, "new": new, "kv": _log(rng, 8, max(16, most)), **more}
    seqs = _log(rng, 1, 8)
    new = _log(rng, 64, 5000 // seqs)
    case = {"kind": kind, "seqs": seqs, "new": new, "past": rng.choice([0, 0, _log(rng, 1, 3000)]), **more}
    while work(case)["flops"] > 4e11:                               # no dearer than the longest listed prompt
        case["new"] = case["new"] * 3 // 4
    return case


# ------------------------------------------------------------------------------------------------ lengths, from the case alone
def _lengths(case):
    """New tokens and cached tokens (the new ones among them) of each request."""
    seqs, kind = case["seqs"], case["kind"]
    part = [1.0 - 0.8 * ((0.618034 * s) % 1.0) for s in range(seqs)]
    if kind == "decode":
        kv = [max(case["new"], round(case["kv"] * (f if case["ragged"] else 1.0))) for f in part]
        return [case["new"]] * seqs, kv
    if case["new"] == 1:
        new = [1] * seqs
    else:
        new = [max(1, round(case["new"] * (f if case.get("ragged", True) else 1.0))) for f in part]
    past = [round(case["past"] * part[-1 - s]) if seqs > 1 else case["past"] for s in range(seqs)]
    return new, [a + b for a, b in zip(new, past)]


def _adapter_of_row(case):
    """Number of the adapter of each row before the seed renumbers them; -1: none."""
    req = np.arange(case["rows"]) // case["run"]
    ids = (req * 5 + 2) % case["adapters"]
    if case["bare"]:
        ids = np.where(req % case["bare"] == case["bare"] - 1, -1, ids)
    return ids


def _visible(case, new, kv):
    """Keys that at least one new token sees, and pairs of a new token and a key it sees, over the batch."""
    keys = pairs = 0
    for q, n in zip(new, kv):
        p = np.arange(n - q, n, dtype=np.int64)
        w, s = case["window"], case["sinks"]
        if w:
            low = np.maximum(0, p - w + 1)
            pairs += int((p - low + 1 + np.minimum(low, s)).sum())
            keys += n - int(low[0]) + min(int(low[0]), s)
        else:
            pairs += int((p + 1).sum())
            keys += n
    return keys, pairs


def work(case):
    if case["kind"] == "adapters":
        ids = _adapter_of_row(case)
        rows, n, m, r = case["rows"], case["n"], case["m"], case["r"]
        used = len(set(ids.tolist()) - {-1})
        return {"bytes": rows * n * (4 if case["x"] == "f32" else 2) + 2 * rows * m * 4 + used * r * (n + m) * 2 + rows * 4,
                "flops": 2 * int((ids >= 0).sum()) * r * (n + m)}
    new, kv = _lengths(case)
    tokens, d, h, hk = sum(new), case["d"], case["heads"], case["kv_heads"]
    if case["kind"] == "append":
        values = tokens * (h + 2 * hk) * d
        return {"bytes": values * ((4 if case["x"] == "f32" else 2) + 2) + max(new) * case["rot"] * 4, "flops": 6 * values}
    keys, pairs = _visible(case, new, kv)
    per_key = 2 * hk * (d * 2 if case["cache"] == "bf16" else d + 4)
    return {"bytes": keys * per_key + 2 * tokens * h * d * 2, "flops": 4 * pairs * h * d}


# ------------------------------------------------------------------------------------------------ inputs
def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32 if dtype == torch.float32 else dtype)


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if case["kind"] == "adapters":
        rows, n, m, r, na = case["rows"], case["n"], case["m"], case["r"], case["adapters"]
        name = torch.cat([torch.randperm(na, generator=g, device=DEV), torch.tensor([-1], device=DEV)])    # renumbered; -1 stays
        ids = name[torch.from_numpy(_adapter_of_row(case)).to(DEV)].to(torch.int32)
        x = _randn(g, rows, n)
        x[:, torch.randperm(n, generator=g, device=DEV)[:max(1, n // 256)]] *= 20.0                          # a few large channels
        return {"x": x.to(torch.bfloat16) if case["x"] == "bf16" else x, "ids": ids,
                "A": (_randn(g, na, r, n) / math.sqrt(n)).to(torch.bfloat16), "B": (_randn(g, na, m, r) * 0.05).to(torch.bfloat16),
                "scale": torch.rand(na, generator=g, device=DEV) + 0.5, "y0": _randn(g, rows, m)}
    new, kv = _lengths(case)
    d, h, hk, page = case["d"], case["heads"], case["kv_heads"], case["page"]
    per = [-(-n // page) for n in kv]
    total, width = sum(per), max(per)
    order = torch.randperm(total + 3, generator=g, device=DEV)[:total].to(torch.int32).cpu().numpy()
    table = np.full((len(kv), width), -1, np.int32)
    at = 0
    for s, c in enumerate(per):
        table[s, :c] = order[at:at + c]
        at += c
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    st = {"new": new, "kv": kv, "tokens": int(start[-1]), "start": torch.from_numpy(start).to(DEV), "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
          "pages": torch.from_numpy(table).to(DEV)}
    shape = (total + 3, hk, page, d)
    if case["kind"] == "append":
        # one projection's output, queries, keys and values side by side in each row
        qkv = _randn(g, st["tokens"], (h + 2 * hk) * d)
        qkv = qkv.to(torch.bfloat16) if case["x"] == "bf16" else qkv
        st["q"], st["k"], st["v"] = qkv[:, :h * d], qkv[:, h * d:(h + hk) * d], qkv[:, (h + hk) * d:]
        st["k_cache"], st["v_cache"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV), torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        freq = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
        angle = torch.arange(max(kv), dtype=torch.float64, device=DEV)[:, None] * freq
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        if case["norm"]:
            st["q_norm"], st["k_norm"] = 1.0 + 0.1 * _randn(g, d), 1.0 + 0.1 * _randn(g, d)
        else:
            st["q_norm"] = st["k_norm"] = None
        return st
    st["q"] = (1.5 * _randn(g, st["tokens"], h * d)).to(torch.bfloat16)
    if case["cache"] == "bf16":
        st["k_cache"], st["v_cache"] = _randn(g, *shape, dtype=torch.bfloat16), _randn(g, *shape, dtype=torch.bfloat16)
        st["k_scale"] = st["v_scale"] = None
    else:
        st["k_cache"] = torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int8)
        st["v_cache"] = torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int8)
        st["k_scale"] = (torch.rand(shape[:3], generator=g, device=DEV) + 0.5) / 73.0
        st["v_scale"] = (torch.rand(shape[:3], generator=g, device=DEV) + 0.5) / 73.0
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if own:
        import paper_2411_07762_amd as aser
        st["ctx"] = ctx = aser.Context(0)
        if case["kind"] == "adapters":
            st["out"] = torch.empty_like(st["y0"])
            ctx.ensure_workspace(aser.aser_adapter_workspace_bytes(case["rows"], case["n"], case["m"], case["r"]))
        else:
            st["cache"] = aser.KvCache(st["k_cache"], st["v_cache"], st.get("k_scale"), st.get("v_scale"))
            st["batch"] = aser.KvBatch(st["start"], st["kv_len"], st["pages"], tokens=st["tokens"], max_new=max(st["new"]), max_kv=max(st["kv"]))
            st["out"] = torch.empty(st["tokens"], case["heads"] * case["d"], dtype=torch.bfloat16, device=DEV)
            if case["kind"] != "append":
                ctx.ensure_workspace(aser.aser_paged_attention_workspace_bytes(st["cache"], st["batch"], case["heads"]))
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    if not own:
        return {"append": _plain_append, "adapters": _plain_adapters}.get(case["kind"], _plain_attention)(st, case)
    import paper_2411_07762_amd as aser
    ctx = st["ctx"]
    if case["kind"] == "append":
        ctx.check(aser.aser_kv_append(ctx, st["q"], st["k"], st["v"], st["cache"], st["batch"], st["out"], rope_cos=st["cos"], rope_sin=st["sin"],
                                      interleaved=case["style"] == "pairs", q_norm=st["q_norm"], k_norm=st["k_norm"], eps=1e-6))
        return {"q": st["out"], "k": st["k_cache"], "v": st["v_cache"]}
    if case["kind"] == "adapters":
        ctx.check(aser.aser_adapter_forward(ctx, st["x"], st["ids"], st["A"], st["B"], st["scale"], st["y0"], st["out"]))
        return st["out"]
    ctx.check(aser.aser_paged_attention(ctx, st["q"], st["cache"], st["batch"], st["out"], scale=case["d"] ** -0.5, window=case["window"],
                                        sinks=case["sinks"]))
    return st["out"]


def _token_places(st):
    """Request and position of every new token."""
    start, kv = st["start"].long(), st["kv_len"].long()
    t = torch.arange(st["tokens"], device=DEV)
    seq = torch.bucketize(t, start[1:], right=True)
    return seq, kv[seq] - (start[1:] - start[:-1])[seq] + t - start[seq]


def _plain_append(st, case):
    seq, pos = _token_places(st)
    d, rot, page = case["d"], case["rot"], case["page"]
    cos, sin = st["cos"][pos][:, None], st["sin"][pos][:, None]

    def turned(x, weight):
        x = x.reshape(st["tokens"], -1, d).float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
        if case["style"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)

    at, slot = st["pages"].long()[seq, pos // page], pos % page
    q = turned(st["q"], st["q_norm"]).to(torch.bfloat16).reshape(st["tokens"], -1)
    st["k_cache"][at, :, slot] = turned(st["k"], st["k_norm"]).to(torch.bfloat16)
    st["v_cache"][at, :, slot] = st["v"].reshape(st["tokens"], -1, d).to(torch.bfloat16)
    return {"q": q, "k": st["k_cache"], "v": st["v_cache"]}


def _plain_attention(st, case):
    d, h, hk = case["d"], case["heads"], case["kv_heads"]
    seq, pos = _token_places(st)
    place = torch.arange(st["tokens"], device=DEV) - st["start"].long()[seq]
    seqs, most = len(st["new"]), max(st["new"])
    pages = st["pages"].long().clamp(min=0)

    def gathered(cache, scale):
        x = cache[pages].float()                                  # requests x pages x heads x slots x channels
        if scale is not None:
            x = x * scale[pages][..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(seqs, hk, -1, d)

    q = torch.zeros(seqs, most, h, d, device=DEV)
    q[seq, place] = st["q"].reshape(-1, h, d).float()
    q = q.reshape(seqs, most, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(seqs, hk, -1, d)
    s = torch.matmul(q, gathered(st["k_cache"], st["k_scale"]).transpose(-1, -2)).mul_(d ** -0.5)
    key = torch.arange(s.shape[-1], device=DEV)
    at = torch.full((seqs, most), -1, device=DEV)
    at[seq, place] = pos
    seen = key <= at[..., None]
    if case["window"]:
        seen &= (key > at[..., None] - case["window"]) | (key < case["sinks"])
    s = s.reshape(seqs, hk, h // hk, most, -1).masked_fill_(~seen[:, None, None], float("-inf"))
    s = s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    s = s.div_(s.sum(-1, keepdim=True).clamp(min=1e-30)).reshape(seqs, hk, -1, s.shape[-1])
    o = torch.matmul(s, gathered(st["v_cache"], st["v_scale"])).reshape(seqs, hk, h // hk, most, d).permute(0, 3, 1, 2, 4).reshape(seqs, most, h * d)
    return o[seq, place].to(torch.bfloat16)


def _plain_adapters(st, case):
    na, r, n, m = case["adapters"], case["r"], case["n"], case["m"]
    mine = (st["ids"].long()[:, None] == torch.arange(na, device=DEV)) * st["scale"]
    p = torch.matmul(st["x"].float(), st["A"].float().reshape(na * r, n).t()).reshape(-1, na, r) * mine[..., None]
    return st["y0"] + torch.matmul(p.reshape(-1, na * r), st["B"].float().permute(0, 2, 1).reshape(na * r, m))


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "adapters":
        y = st["y0"].double()
        for a in range(case["adapters"]):
            rows = (st["ids"] == a).nonzero()[:, 0]
            if rows.numel():
                y[rows] += st["scale"][a].double() * (st["x"][rows].double() @ st["A"][a].double().t() @ st["B"][a].double().t())
        return y
    d, h, hk, page = case["d"], case["heads"], case["kv_heads"], case["page"]
    start = np.concatenate([[0], np.cumsum(st["new"])])
    if case["kind"] == "append":
        k_cache, v_cache = st["k_cache"].double(), st["v_cache"].double()
        out = torch.empty(st["tokens"], h * d, dtype=torch.float64, device=DEV)
        half = case["rot"] // 2
        first = torch.arange(half, device=DEV) * (1 if case["style"] == "half" else 2)
        second = first + (half if case["style"] == "half" else 1)
        for s in range(case["seqs"]):
            rows = slice(int(start[s]), int(start[s + 1]))
            pos = torch.arange(st["kv"][s] - st["new"][s], st["kv"][s], device=DEV)
            turn = torch.complex(st["cos"][pos].double(), st["sin"][pos].double())[:, None]
            for name, weight in (("q", st["q_norm"]), ("k", st["k_norm"])):
                x = st[name][rows].double().reshape(pos.numel(), -1, d)
                if weight is not None:
                    x = x / (x.pow(2).sum(-1, keepdim=True) / d + 1e-6).sqrt() * weight.double()
                z = torch.complex(x[..., first], x[..., second]) * turn
                x = x.clone()
                x[..., first], x[..., second] = z.real, z.imag
                if name == "q":
                    out[rows] = x.reshape(pos.numel(), -1)
                else:
                    k_cache[st["pages"][s].long()[pos // page], :, pos % page] = x
            v_cache[st["pages"][s].long()[pos // page], :, pos % page] = st["v"][rows].double().reshape(pos.numel(), -1, d)
        return {"q": out, "k": k_cache, "v": v_cache}
    out = torch.zeros(st["tokens"], h, d, dtype=torch.float64, device=DEV)
    for s in range(case["seqs"]):
        n, new = st["kv"][s], st["new"][s]
        pages = st["pages"][s, :-(-n // page)].long()
        sides = []
        for cache, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])):
            x = cache[pages].double() if scale is None else cache[pages].double() * scale[pages].double()[..., None]
            sides.append(x.transpose(0, 1).reshape(hk, -1, d)[:, :n])
        keys, values = sides
        j = torch.arange(n, device=DEV)
        for lo in range(0, new, 1024):
            hi = min(new, lo + 1024)
            i = torch.arange(n - new + lo, n - new + hi, device=DEV)[:, None]
            hidden = (j > i) | ((j <= i - case["window"]) & (j >= case["sinks"]) if case["window"] else j < 0)
            q = st["q"][int(start[s]) + lo:int(start[s]) + hi].double().reshape(hi - lo, h, d)
            for a in range(h):
                logits = (q[:, a] @ keys[a * hk // h].t()) / math.sqrt(d)
                out[int(start[s]) + lo:int(start[s]) + hi, a] = logits.masked_fill(hidden, -math.inf).softmax(-1) @ values[a * hk // h]
    return out.reshape(st["tokens"], h * d)
