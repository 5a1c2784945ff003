"""What the operators for paged caches are judged on: rotary positions, head norms with the rotation, appending to a paged
cache and attention over it, through the public entry points of paper_2409_09086_amd.binding and in a plain form of
elementary torch operations.

A case's kind:

  rotate   rotary positions of queries and keys                                            (Rotary.apply)
  norm     the head norms of queries and keys and the rotation in one pass                 (Rotary.apply with weights)
  append   a batch's new keys and values into their pages, rotated (and normed) on the
           way, the queries with them                                                      (PagedCache.append)
  attend   attention of a batch's new tokens over the pages                                (PagedCache.attend)

Batches: `chunks` sequences that bring new_lo .. new_hi tokens each and `singles` sequences that bring one, with
len_lo .. len_hi tokens in the cache before them.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-6
_BASE = 500000.0


def _case(name, kind, dtype, heads, kv_heads, head_dim, **more):
    c = {"kind": kind, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim}
    if name:
        c["name"] = name
    if kind != "attend":
        c.update({"layout": "half", "dims": head_dim, "factor": 1.0, "positions": 131072, "norm": kind == "norm"})
    if kind in ("rotate", "norm"):
        c["tokens"] = 1
    else:
        c.update({"page": 64, "chunks": 0, "new_lo": 1, "new_hi": 1, "singles": 0, "len_lo": 0, "len_hi": 0})
    if kind == "attend":
        c.update({"window": 0, "lse": False})
    c.update(more)
    return c


def listed():
    return [
        # one decoded token far into a long context: latency
        _case("rotate_token", "rotate", "bf16", 32, 8, 128),
        # single precision, half of a 64-wide head turned, neighbouring pairs, an odd number of tokens
        _case("rotate_part_fp32", "rotate", "fp32", 16, 4, 64, tokens=1537, layout="interleaved", dims=32),
        # a long prompt of an 8B-shaped layer with frequencies scaled for a longer context than the trained one
        _case("rotate_prompt_scaled", "rotate", "bf16", 32, 8, 128, tokens=8192, factor=8.0),
        # the tokens of a decoding batch of a model with head norms
        _case("norm_batch", "norm", "bf16", 32, 8, 128, tokens=64),
        # a prompt of the same with as many key heads as query heads, neighbouring pairs
        _case("norm_prompt", "norm", "bf16", 32, 32, 128, tokens=4099, layout="interleaved"),
        # one token of each of 64 sequences enters the cache
        _case("append_batch", "append", "bf16", 32, 8, 128, norm=True, singles=64, len_lo=256, len_hi=2048),
        # prompts of three sequences enter the cache
        _case("append_prompts", "append", "bf16", 32, 8, 128, chunks=3, new_lo=1000, new_hi=2000, len_lo=0, len_hi=1000),
        # one sequence, one token, a short context, small pages: latency
        _case("attend_token", "attend", "bf16", 32, 32, 128, page=16, singles=1, len_lo=1000, len_hi=1000),
        # a decoding batch of an 8B-shaped layer with grouped heads: bound by the cache that it reads
        _case("attend_batch", "attend", "bf16", 32, 8, 128, singles=64, len_lo=256, len_hi=8192),
        # a chunk of a prompt between decoding sequences, small pages, the log-sum-exp wanted
        _case("attend_mixed", "attend", "bf16", 32, 8, 128, page=16, chunks=1, new_lo=512, new_hi=512, singles=31, len_lo=512,
              len_hi=4096, lse=True),
        # a chunk of a long prompt, 7B-shaped: bound by the matrix cores
        _case("attend_prompt", "attend", "bf16", 32, 32, 128, page=128, chunks=1, new_lo=2048, new_hi=2048, len_lo=8192, len_hi=8192),
        # single precision, 64-wide heads, a sliding window, ragged chunks
        _case("attend_window_fp32", "attend", "fp32", 8, 2, 64, page=32, chunks=5, new_lo=33, new_hi=197, len_lo=0, len_hi=1500,
              window=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "norm", "append", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    heads = kv * rng.choice([g for g in (1, 2, 4, 5, 8) if kv * g <= 40])
    more = {}
    if kind != "attend":
        more["layout"] = rng.choice(["half", "half", "interleaved"])
        more["dims"] = rng.choice([d, d, d // 2, 16, d - 16])
        more["factor"] = rng.choice([1.0, 1.0, 4.0, 8.0])
        more["positions"] = rng.choice([8192, 32768, 131072])
    if kind in ("rotate", "norm"):
        more["tokens"] = _log_int(rng, 1, 8192 if dtype == "bf16" else 4096)
    else:
        more["page"] = rng.choice([16, 16, 32, 64, 128, 256])
        if rng.random() < 0.6:
            more["singles"] = _log_int(rng, 1, 128)
        if "singles" not in more or rng.random() < 0.5:
            more["chunks"] = rng.randint(1, 4)
            more["new_lo"] = _log_int(rng, 2, 256)
            more["new_hi"] = more["new_lo"] + _log_int(rng, 1, 512 if dtype == "bf16" else 128)
        more["len_lo"] = rng.choice([0, _log_int(rng, 1, 1024)])
        most = 4096 if kind == "append" else 8192
        more["len_hi"] = more["len_lo"] + _log_int(rng, 1, most if dtype == "bf16" else 1024)
    if kind == "append":
        more["norm"] = rng.random() < 0.5
        more["len_hi"] = min(more["len_hi"], 4096)
    if kind == "attend":
        more["window"] = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
        more["lse"] = rng.random() < 0.3
    return _case(None, kind, dtype, heads, kv, d, **more)


def _spread(i, lo, hi):
    """The i-th of a sequence of whole numbers spread over lo .. hi."""
    return lo + int((hi - lo) * ((i + 1) * 0.6180339887498949 % 1.0)) if hi > lo else lo


def _lengths(case):
    """New tokens and cached tokens before them of each sequence; the chunks stand between the singles."""
    n = [1] * case["singles"]
    at = len(n) // 2
    n[at:at] = [_spread(i, case["new_lo"], case["new_hi"]) for i in range(case["chunks"])]
    return n, [_spread(i, case["len_lo"], case["len_hi"]) for i in range(len(n))]


def _frequencies(case):
    """Angle per position of each pair, 64 bits.  With a factor: by parts, for a model trained on 8192 positions."""
    f = _BASE ** (-2.0 * torch.arange(case["dims"] // 2, dtype=torch.float64) / case["dims"])
    if case["factor"] != 1.0:
        g = ((8192 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (g + (1.0 - g) / case["factor"])
    return f


def prepare(case, seed):
    dev, dt = torch.device("cuda:0"), _DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["head_dim"]

    def normal(*shape, scale=1.0):
        return (scale * torch.randn(shape, generator=gen, device=dev)).to(dt)

    st = {"case": case}
    if case["kind"] != "attend":
        if case["norm"]:
            st["q_weight"], st["k_weight"] = (torch.rand(d, generator=gen, device=dev).add(0.5).to(dt) for _ in range(2))
        else:
            st["q_weight"] = st["k_weight"] = None
        if own:
            from paper_2409_09086_amd import binding
            scaled = {"trained": 8192, "factor": case["factor"], "low_turns": 1.0, "high_turns": 4.0} if case["factor"] != 1.0 else {}
            st["rotary"] = binding.Rotary(d, case["positions"], dtype=dt, base=_BASE, dims=case["dims"], layout=case["layout"],
                                          norm_eps=_EPS, device=dev, **scaled)
        else:
            ang = torch.arange(case["positions"], dtype=torch.float64, device=dev)[:, None] * _frequencies(case).to(dev)
            st["cos"], st["sin"] = ang.cos().float(), ang.sin().float()
    if case["kind"] in ("rotate", "norm"):
        # a projection's output: queries, keys and values of a token side by side
        T = case["tokens"]
        qkv = normal(T, Hq + 2 * Hkv, d)
        st["q"], st["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
        p0 = int(torch.randint(0, case["positions"] - T + 1, (1,), generator=gen, device=dev).item())
        st["positions"] = torch.arange(p0, p0 + T, dtype=torch.int32, device=dev)
        return st
    n, before = _lengths(case)
    S, P, T = len(n), case["page"], sum(n)
    lens = [a + b for a, b in zip(n, before)]
    need = [-(-x // P) for x in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    table = torch.full((S, max(need)), -1, dtype=torch.int32, device=dev)
    at = 0
    for s in range(S):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    starts = [0]
    for x in n:
        starts.append(starts[-1] + x)
    st["n"], st["lens"], st["table"] = n, lens, table
    st["K"], st["V"] = normal(pages, Hkv, P, d), normal(pages, Hkv, P, d)
    if own:
        from paper_2409_09086_amd import binding
        st["cache"] = binding.PagedCache(pages, P, Hq, Hkv, d, dtype=dt, window=case.get("window") or None, device=dev)
        st["batch"] = binding.PagedBatch(torch.tensor(starts, dtype=torch.int32, device=dev),
                                         torch.tensor(lens, dtype=torch.int32, device=dev), table, tokens=T, max_new=max(n),
                                         max_len=max(lens))
    if case["kind"] == "append":
        qkv = normal(T, Hq + 2 * Hkv, d)
        st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        if not own:
            st["positions"] = torch.tensor([len_ - m + r for m, len_ in zip(n, lens) for r in range(m)], device=dev)
            st["seq"] = torch.tensor([s for s in range(S) for _ in range(n[s])], device=dev)
    else:
        st["q"] = normal(T, Hq, d)
    return st


def _rotated(x, weight, positions, st):
    """Norm and rotation of x [T, H, d], 32 bits, rounded once."""
    case = st["case"]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + _EPS) * weight.float()
    rd = case["dims"]
    cos, sin = st["cos"][positions.long()][:, None], st["sin"][positions.long()][:, None]
    out = y.clone()
    if case["layout"] == "half":
        a, b = y[..., :rd // 2], y[..., rd // 2:rd]
        out[..., :rd // 2], out[..., rd // 2:rd] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., 0:rd:2], y[..., 1:rd:2]
        out[..., 0:rd:2], out[..., 1:rd:2] = a * cos - b * sin, b * cos + a * sin
    return out.to(x.dtype)


def _gathered(pool, rows, n):
    """The first n rows of a sequence, [Hkv, n, d], from its pages."""
    x = pool[rows.long()]                                    # [pages, Hkv, P, d]
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _run_plain(st):
    case = st["case"]
    if case["kind"] in ("rotate", "norm"):
        return _rotated(st["q"], st["q_weight"], st["positions"], st), _rotated(st["k"], st["k_weight"], st["positions"], st)
    P = case["page"]
    if case["kind"] == "append":
        q, k = _rotated(st["q"], st["q_weight"], st["positions"], st), _rotated(st["k"], st["k_weight"], st["positions"], st)
        page, row = st["table"][st["seq"], st["positions"] // P].long(), st["positions"] % P
        st["K"][page, :, row] = k
        st["V"][page, :, row] = st["v"]
        return q, st["K"], st["V"]
    Hkv, d = case["kv_heads"], case["head_dim"]
    G = case["heads"] // Hkv
    outs, lses, at = [], [], 0
    for s, (m, n) in enumerate(zip(st["n"], st["lens"])):
        rows = st["table"][s, :-(-n // P)]
        K, V = _gathered(st["K"], rows, n).float(), _gathered(st["V"], rows, n).float()
        q = st["q"][at:at + m].float().reshape(m, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, m * G, d)
        at += m
        logits = torch.matmul(q, K.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
        j = torch.arange(n, device=q.device)
        p = torch.arange(n - m, n, device=q.device).repeat_interleave(G)[:, None]
        hidden = j > p
        if case["window"]:
            hidden = hidden | (j <= p - case["window"])
        logits = logits.masked_fill(hidden, -math.inf)
        top = logits.amax(dim=-1, keepdim=True)
        w = torch.exp(logits - top)
        total = w.sum(dim=-1, keepdim=True)
        o = torch.matmul(w, V) / total
        outs.append(o.reshape(Hkv, m, G, d).permute(1, 0, 2, 3).reshape(m, Hkv * G, d))
        lses.append((top + total.log()).reshape(Hkv, m, G).permute(1, 0, 2).reshape(m, Hkv * G))
    out = torch.cat(outs).to(st["q"].dtype)
    return (out, torch.cat(lses)) if case["lse"] else out


def run(st):
    if not own:
        return _run_plain(st)
    case = st["case"]
    if case["kind"] in ("rotate", "norm"):
        return st["rotary"].apply(st["positions"], st["q"], st["k"], q_weight=st["q_weight"], k_weight=st["k_weight"])
    if case["kind"] == "append":
        q = st["cache"].append(st["batch"], st["k"], st["v"], st["K"], st["V"], rotary=st["rotary"], k_weight=st["k_weight"],
                               q=st["q"], q_weight=st["q_weight"])
        return q, st["K"], st["V"]
    if case["lse"]:
        lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device=st["q"].device)
        return st["cache"].attend(st["batch"], st["q"], st["K"], st["V"], lse=lse), lse
    return st["cache"].attend(st["batch"], st["q"], st["K"], st["V"])


def exact(case, seed):
    """From the definitions, in 64 bits: rotations as products of complex numbers, one head and one sequence at a time."""
    st = prepare(case, seed)
    dev = st["q"].device

    def turned(x, weight, positions):
        y = x.double()
        if weight is not None:
            y = y / ((y ** 2).sum(dim=-1, keepdim=True) / y.shape[-1] + _EPS).sqrt() * weight.double()
        rd = case["dims"]
        unit = torch.polar(torch.ones((), dtype=torch.float64, device=dev),
                           positions.double()[:, None] * _frequencies(case).to(dev))[:, None]
        if case["layout"] == "half":
            z = torch.complex(y[..., :rd // 2].contiguous(), y[..., rd // 2:rd].contiguous()) * unit
            front = torch.cat([z.real, z.imag], dim=-1)
        else:
            z = torch.view_as_complex(y[..., :rd].reshape(*y.shape[:-1], rd // 2, 2).contiguous()) * unit
            front = torch.view_as_real(z).reshape(*y.shape[:-1], rd)
        return torch.cat([front, y[..., rd:]], dim=-1)

    if case["kind"] in ("rotate", "norm"):
        return turned(st["q"], st["q_weight"], st["positions"]), turned(st["k"], st["k_weight"], st["positions"])
    n, lens, table, P = st["n"], st["lens"], st["table"].cpu(), case["page"]
    if case["kind"] == "append":
        pos = torch.cat([torch.arange(len_ - m, len_, device=dev) for m, len_ in zip(n, lens)])
        q, k = turned(st["q"], st["q_weight"], pos), turned(st["k"], st["k_weight"], pos)
        K, V, at = st["K"].double(), st["V"].double(), 0
        for s, (m, len_) in enumerate(zip(n, lens)):
            for page in range((len_ - m) // P, (len_ - 1) // P + 1):
                lo, hi = max(page * P, len_ - m), min(page * P + P, len_)
                src = slice(at + lo - (len_ - m), at + hi - (len_ - m))
                dst = int(table[s, page])
                K[dst, :, lo - page * P:hi - page * P] = k[src].transpose(0, 1)
                V[dst, :, lo - page * P:hi - page * P] = st["v"][src].double().transpose(0, 1)
            at += m
        return q, K, V
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty((sum(n), Hq, d), dtype=torch.float64, device=dev)
    lse = torch.empty((sum(n), Hq), dtype=torch.float64, device=dev)
    at = 0
    for s, (m, len_) in enumerate(zip(n, lens)):
        p, j = torch.arange(len_ - m, len_, device=dev)[:, None], torch.arange(len_, device=dev)[None]
        seen = (j <= p) & (j > p - case["window"]) if case["window"] else j <= p
        rows = [int(x) for x in table[s, :-(-len_ // P)]]
        for h in range(Hkv):
            K, V = (torch.cat([pool[x, h] for x in rows])[:len_].double() for pool in (st["K"], st["V"]))
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                logits = (st["q"][at:at + m, g].double() @ K.t()) / math.sqrt(d)
                logits[~seen] = -math.inf
                lse[at:at + m, g] = torch.logsumexp(logits, dim=-1)
                out[at:at + m, g] = torch.softmax(logits, dim=-1) @ V
        at += m
    return (out, lse) if case["lse"] else out


def work(case):
    """Inputs read once, outputs written once; of the pages what the new tokens see."""
    Hq, Hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("rotate", "norm"):
        T = case["tokens"]
        values = T * (Hq + Hkv) * d
        return {"bytes": 2 * values * e + 4 * T, "flops": (6 if case["norm"] else 3) * values}
    n, before = _lengths(case)
    T = sum(n)
    if case["kind"] == "append":
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * d * e + 8 * len(n), "flops": (6 if case["norm"] else 3) * T * (Hq + Hkv) * d}
    keys = pairs = 0
    for m, b in zip(n, before):
        w = case["window"] or b + m
        keys += min(b + m, w + m - 1)
        pairs += sum(min(b + r + 1, w) for r in range(m))
    return {"bytes": 2 * keys * Hkv * d * e + 2 * T * Hq * d * e + (4 * T * Hq if case["lse"] else 0), "flops": 4 * d * Hq * pairs}
