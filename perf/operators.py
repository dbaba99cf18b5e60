"""The operators of a decoder's attention block on the packed layout: what is called, with which inputs, how much
work a call cannot do without, and what it computes in plain operations.

  causal  - fmha_causal_fwd / _bwd: causal attention with grouped heads over packed sequences
  rope    - fmha_qk_norm_rope_fwd / _bwd: norm of every query and key head and its rotation by the token's position
  append  - fmha_cache_append: new keys and values into a paged cache, rotated (and queries beside them)
  cached  - fmha_cache_attention: one query token per sequence against its pages

`own` False: `run` computes them with elementary torch operations in 32 bits (angles of positions and long sums in 64).
`own` True: `run` makes the library's calls.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one short prompt of a small model: launch latency
        {"name": "causal_short_prompt", "op": "causal", "lens": "equal", "batch": 1, "longest": 37, "heads": 12,
         "kv_heads": 4, "dim": 64, "type": "f16", "train": False, "lens_seed": 1},
        # prompts of different lengths that a server takes up together
        {"name": "causal_prompts", "op": "causal", "lens": "uniform", "batch": 12, "longest": 4000, "heads": 32,
         "kv_heads": 8, "dim": 128, "type": "bf16", "train": False, "lens_seed": 2},
        # one long document
        {"name": "causal_long_prompt", "op": "causal", "lens": "equal", "batch": 1, "longest": 16384, "heads": 16,
         "kv_heads": 2, "dim": 128, "type": "bf16", "train": False, "lens_seed": 3},
        # a training step on the length mixture that the attention benchmark uses: 56 sequences, 16 heads of 64
        {"name": "causal_train_mixture", "op": "causal", "lens": "mixture", "batch": 56, "longest": 512, "heads": 16,
         "kv_heads": 16, "dim": 64, "type": "f16", "train": True, "lens_seed": 4},
        # a training step on documents packed to a long context
        {"name": "causal_train_long", "op": "causal", "lens": "uniform", "batch": 6, "longest": 4096, "heads": 32,
         "kv_heads": 8, "dim": 128, "type": "bf16", "train": True, "lens_seed": 5},
        # queries and keys of a few prompts, far positions, part of the head in neighbouring pairs, no norm
        {"name": "rope_prompts", "op": "rope", "lens": "uniform", "batch": 3, "longest": 700, "heads": 12, "kv_heads": 12,
         "dim": 64, "rotary": 32, "layout": "interleaved", "norm": False, "far": 900000, "type": "f16", "train": False,
         "lens_seed": 6},
        # a training step's norms and rotations, forward and backward
        {"name": "rope_train", "op": "rope", "lens": "uniform", "batch": 12, "longest": 4096, "heads": 32, "kv_heads": 8,
         "dim": 128, "rotary": 128, "layout": "half", "norm": True, "far": 0, "type": "bf16", "train": True, "lens_seed": 7},
        # the step of a serving loop: one token per sequence, queries normed and rotated in the same call
        {"name": "append_step", "op": "append", "lens": "one", "batch": 64, "longest": 1, "context": 8000, "heads": 32,
         "kv_heads": 8, "dim": 128, "rotary": 128, "layout": "half", "norm": True, "page": 16, "type": "bf16", "lens_seed": 8},
        # prompts going into the cache
        {"name": "append_prompts", "op": "append", "lens": "uniform", "batch": 12, "longest": 4000, "context": 500, "heads": 32,
         "kv_heads": 8, "dim": 128, "rotary": 64, "layout": "half", "norm": False, "page": 64, "type": "bf16", "lens_seed": 9},
        # a few short chats
        {"name": "cached_small", "op": "cached", "lens": "uniform", "batch": 4, "longest": 600, "heads": 12, "kv_heads": 12,
         "dim": 64, "page": 16, "type": "f16", "lens_seed": 10},
        # a full serving batch of ragged contexts
        {"name": "cached_batch", "op": "cached", "lens": "uniform", "batch": 64, "longest": 8000, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "type": "bf16", "lens_seed": 11},
        # two very long contexts
        {"name": "cached_long", "op": "cached", "lens": "equal", "batch": 2, "longest": 131072, "heads": 64, "kv_heads": 8,
         "dim": 128, "page": 64, "type": "bf16", "lens_seed": 12},
    ]


def _spread(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["causal", "causal", "rope", "append", "cached"])
    dim = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8, 12]) if dim == 64 else rng.choice([1, 2, 4, 8])
    case = {"op": op, "lens": rng.choice(["uniform", "uniform", "equal", "mixture", "skewed"]), "dim": dim, "kv_heads": kv,
            "heads": min(64, kv * rng.choice([1, 2, 3, 4, 6, 8])) // kv * kv, "type": rng.choice(["bf16", "f16"]),
            "lens_seed": rng.randrange(1 << 30)}
    if op == "causal":
        case["longest"] = _spread(rng, 1, 8000)
        case["train"] = rng.random() < 0.6
        most = 1_200_000_000 if case["train"] else 2_000_000_000  # scores that the plain form holds
        most = max(1, most // (case["heads"] * case["longest"] ** 2))
        most = min(most, max(1, 60000 // case["longest"]))
        case["batch"] = _spread(rng, 1, min(300, most))
    elif op in ("rope", "append"):
        case["longest"] = _spread(rng, 1, 4000)
        case["batch"] = _spread(rng, 1, max(1, min(300, 24000 // case["longest"])))
        case["rotary"] = rng.choice([r for r in (16, 32, 48, 64, 96, 128) if r <= dim])
        case["layout"] = rng.choice(["half", "interleaved"])
        case["norm"] = rng.random() < 0.5
        if op == "rope":
            case["far"] = rng.choice([0, 0, _spread(rng, 1, 1000000)])
            case["train"] = rng.random() < 0.6
        else:
            case["context"] = _spread(rng, 1, 4000)
            case["page"] = rng.choice([1, 16, 32, 64, 128])
            if rng.random() < 0.5:
                case.update(lens="one", longest=1, batch=_spread(rng, 1, 300))
    else:
        case["longest"] = _spread(rng, 1, 100000)
        case["batch"] = _spread(rng, 1, max(1, min(256, 2_000_000 // (case["longest"] * kv))))
        case["page"] = rng.choice([1, 16, 32, 64, 128])
    return case


def lengths(case):
    """Tokens of each sequence: a matter of the case, whatever the seed of its inputs."""
    r, n, m = np.random.default_rng(case["lens_seed"]), case["batch"], case["longest"]
    if case["lens"] in ("equal", "one"):
        return [m] * n
    if case["lens"] == "mixture":  # 30 % short, 40 % middling, 30 % of full length
        kind = r.random(n)
        out = np.where(kind < 0.3, r.integers(1, max(2, m // 4), n), np.where(kind < 0.7, r.integers(m // 4 + 1, m + 1, n), m))
    elif case["lens"] == "skewed":  # most are short
        out = np.where(r.random(n) < 0.8, r.integers(1, max(2, m // 16), n), r.integers(1, m + 1, n))
    else:
        out = r.integers(max(1, m // 50), m + 1, n)
    out[int(r.integers(0, n))] = m
    return [int(x) for x in out]


def contexts(case):
    """Tokens that each sequence has in the cache before the new ones."""
    r = np.random.default_rng(case["lens_seed"] + 1)
    return [int(x) for x in r.integers(0, case["context"] + 1, case["batch"])]


def work(case):
    lens = lengths(case)
    t, h, hk, d = sum(lens), case["heads"], case["kv_heads"], case["dim"]
    pairs = sum(n * (n + 1) // 2 for n in lens)
    if case["op"] == "causal":
        b = 2 * d * t * (2 * h + 2 * hk) + 4 * h * t
        f = 4 * d * h * pairs
        if case["train"]:
            b += 2 * d * t * (4 * h + 4 * hk) + 4 * h * t
            f += 10 * d * h * pairs
    elif case["op"] == "rope":
        b = 4 * d * t * (h + hk)
        f = 8 * d * t * (h + hk)
        if case["train"]:
            b += 2 * d * t * (h + hk) * (3 if case["norm"] else 2)
            f *= 3
    elif case["op"] == "append":
        b = 4 * d * t * (h + 2 * hk)
        f = 8 * d * t * (h + hk)
    else:
        b = 4 * d * hk * t + 4 * d * h * len(lens)
        f = 4 * d * h * t
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------------------ the inputs
def frequencies(rotary, far):
    """Radians per position of each pair; far positions are brought closer by a factor of four (linear scaling)."""
    f = 10000.0 ** (-np.arange(0, rotary, 2, dtype=np.float64) / rotary)
    return f / 4 if far else f


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 2 + 1)
    lens = lengths(case)
    b, t, h, hk, d = len(lens), sum(lens), case["heads"], case["kv_heads"], case["dim"]
    dt = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).to(dt)

    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=dev)
    s = {"case": case, "cu": cu, "longest": max(lens), "total": t, "scale": 1 / math.sqrt(d)}
    if case["op"] == "causal":
        s.update(q=normal(t, h, d), k=normal(t, hk, d), v=normal(t, hk, d))
        s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(h, t, device=dev)
        if case["train"]:
            s["do"] = normal(t, h, d)
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in "qkv")
        if own:
            from paper_2208_08124_amd import fmha
            s["workspace"] = fmha.alloc_causal_workspace(b, t, h, hk, d, case["train"])
    if case["op"] in ("rope", "append"):
        s["rope"] = (torch.tensor(frequencies(case["rotary"], case.get("far", 0)), device=dev), case["layout"], 1.0)
        s["gq"] = s["gk"] = None
        if case["norm"]:
            s["gq"], s["gk"] = (1 + 0.2 * torch.randn(d, generator=gen, device=dev) for _ in range(2))
        s["q"], s["k"] = normal(t, h, d), normal(t, hk, d)
        s["q_out"] = torch.empty_like(s["q"])
    if case["op"] == "rope":
        s["positions"] = None
        if case["far"]:
            start = torch.tensor(np.repeat(np.asarray([0] + lens[:-1]).cumsum(), lens), device=dev)
            s["positions"] = (torch.arange(t, device=dev) - start + case["far"]).to(torch.int32)
        s["k_out"] = torch.empty_like(s["k"])
        if case["train"]:
            s["dq_out"], s["dk_out"] = normal(t, h, d), normal(t, hk, d)
            s["dq"], s["dk"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
            s["dgq"], s["dgk"] = (torch.empty(d, device=dev) if case["norm"] else None for _ in range(2))
            if own:
                from paper_2208_08124_amd import fmha
                s["workspace"] = fmha.alloc_qk_norm_rope_workspace(t, h, hk, d)
    if case["op"] in ("append", "cached"):
        held = [n + c for n, c in zip(lens, contexts(case))] if case["op"] == "append" else lens
        page = case["page"]
        columns = -(-max(held) // page)
        count = [-(-n // page) for n in held]
        pages = sum(count) + 3
        order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        first = torch.tensor(np.cumsum([0] + count[:-1]), device=dev)
        at = first[:, None] + torch.arange(columns, device=dev)[None]
        inside = torch.arange(columns, device=dev)[None] < torch.tensor(count, device=dev)[:, None]
        s["table"] = torch.where(inside, order[at.clamp(max=pages - 1)], torch.full_like(order[:1], -1)).contiguous()
        s["seqlens"] = torch.tensor(held, dtype=torch.int32, device=dev)
        if case["op"] == "append":
            s["v"] = normal(t, hk, d)
            s["k_cache"], s["v_cache"] = (torch.zeros(pages, hk, page, d, dtype=dt, device=dev) for _ in range(2))
        else:
            s["k_cache"], s["v_cache"] = normal(pages, hk, page, d), normal(pages, hk, page, d)
            s["q"] = normal(b, h, d)
            s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(b, h, device=dev)
            if own:
                from paper_2208_08124_amd import fmha
                s["workspace"] = fmha.alloc_cache_attention_workspace(b, h, hk, d, s["longest"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_causal(s):
    from paper_2208_08124_amd import fmha
    fmha.fmha_causal_fwd(s["q"], s["k"], s["v"], s["cu"], s["longest"], s["scale"], s["o"], s["lse"], s["workspace"])
    if not s["case"]["train"]:
        return {"o": s["o"], "lse": s["lse"]}
    fmha.fmha_causal_bwd(s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["cu"], s["longest"], s["scale"],
                         s["dq"], s["dk"], s["dv"], s["workspace"], reuse_schedule=True)
    return {"o": s["o"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _own_rope(s):
    from paper_2208_08124_amd import fmha
    far = {"positions": s["positions"]} if s["positions"] is not None else {"cu_seqlens": s["cu"]}
    how = dict(rope=s["rope"], gamma_q=s["gq"], gamma_k=s["gk"], eps=EPS, **far)
    fmha.fmha_qk_norm_rope_fwd(s["q"], s["k"], s["q_out"], s["k_out"], **how)
    out = {"q": s["q_out"], "k": s["k_out"]}
    if s["case"]["train"]:
        fmha.fmha_qk_norm_rope_bwd(s["dq_out"], s["dk_out"], s["q"], s["k"], s["dq"], s["dk"], s["dgq"], s["dgk"],
                                   s["workspace"], **how)
        out.update(dq=s["dq"], dk=s["dk"], dgq=s["dgq"], dgk=s["dgk"])
    return out


def _own_append(s):
    from paper_2208_08124_amd import fmha
    cu = None if s["case"]["lens"] == "one" else s["cu"]
    fmha.fmha_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["seqlens"], cu_seqlens=cu,
                           q=s["q"], q_out=s["q_out"], rope=s["rope"], gamma_q=s["gq"], gamma_k=s["gk"], eps=EPS)
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_cached(s):
    from paper_2208_08124_amd import fmha
    fmha.fmha_cache_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["seqlens"], s["longest"], s["scale"],
                              s["o"], s["lse"], s["workspace"])
    return {"o": s["o"], "lse": s["lse"]}


# ---- plain forms
def _places(s):
    """Sequence and position in it of every packed row."""
    row = torch.arange(s["total"], device=s["cu"].device)
    seq = torch.searchsorted(s["cu"].long(), row, right=True) - 1
    return seq, row - s["cu"].long()[seq]


def _padded(x, s):
    """[T, H, D] packed -> [B, H, longest, D] in 32 bits, zeros behind the sequences."""
    cu, n = s["cu"].long(), s["longest"]
    col = torch.arange(n, device=x.device)
    inside = col[None] < (cu[1:] - cu[:-1])[:, None]
    at = torch.where(inside, cu[:-1, None] + col[None], torch.zeros_like(cu[:1]))
    return (x.float()[at] * inside[..., None, None]).permute(0, 2, 1, 3).contiguous()


def _plain_causal(s):
    c = s["case"]
    seq, pos = _places(s)
    n, d, hk, g, b = s["longest"], c["dim"], c["kv_heads"], c["heads"] // c["kv_heads"], s["cu"].numel() - 1
    q = _padded(s["q"], s).reshape(b * hk, g * n, d)  # the g heads that share a key head stand one below the other
    k = _padded(s["k"], s).reshape(b * hk, n, d)
    v = _padded(s["v"], s).reshape(b * hk, n, d)
    p = torch.matmul(q, k.transpose(1, 2)).mul_(s["scale"]).view(b * hk, g, n, n)
    col = torch.arange(n, device=q.device)
    p.masked_fill_(col[None, :] > col[:, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(total)
    lse = (top + total.log()).view(b, hk * g, n)
    p = p.view(b * hk, g * n, n)
    o = torch.matmul(p, v)

    def packed(x, heads, like):
        return x.view(b, heads, n, d)[seq, :, pos].to(like.dtype)

    out = {"o": packed(o, hk * g, s["o"]), "lse": lse[seq, :, pos].t().contiguous()}
    if not c["train"]:
        return out
    do = _padded(s["do"], s).reshape(b * hk, g * n, d)
    out["dv"] = packed(torch.matmul(p.transpose(1, 2), do), hk, s["v"])
    ds = torch.matmul(do, v.transpose(1, 2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    out["dq"] = packed(torch.matmul(ds, k), hk * g, s["q"])
    out["dk"] = packed(torch.matmul(ds.transpose(1, 2), q), hk, s["k"])
    return out


def _turned(x, cos, sin, layout):
    """Pairs (a, b) of the leading elements of [T, H, D] become (a cos - b sin, a sin + b cos); cos, sin are [T, 1, pairs]."""
    r = 2 * cos.shape[-1]
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)
    a, b = x[..., :r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., r:]], -1)


def _angles(s, positions):
    angle = positions.double()[:, None] * s["rope"][0][None]
    return angle.cos().float()[:, None] * s["rope"][2], angle.sin().float()[:, None] * s["rope"][2]


def _normed(x, gamma):
    x = x.float()
    return x if gamma is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma


def _plain_rope(s):
    layout = s["rope"][1]
    cos, sin = _angles(s, _places(s)[1] if s["positions"] is None else s["positions"])

    def forward(x, gamma):
        return _turned(_normed(x, gamma), cos, sin, layout).to(x.dtype)

    def backward(dy, x, gamma):
        g = _turned(dy.float(), cos, -sin, layout)
        if gamma is None:
            return g.to(x.dtype), None
        x = x.float()
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xh = x * rstd
        gg = g * gamma
        return (rstd * (gg - xh * (gg * xh).mean(-1, keepdim=True))).to(dy.dtype), (g * xh).sum((0, 1), dtype=torch.float64).float()

    out = {"q": forward(s["q"], s["gq"]), "k": forward(s["k"], s["gk"])}
    if s["case"]["train"]:
        out["dq"], out["dgq"] = backward(s["dq_out"], s["q"], s["gq"])
        out["dk"], out["dgk"] = backward(s["dk_out"], s["k"], s["gk"])
    return out


def _plain_append(s):
    seq, pos = _places(s)
    pos = pos + (s["seqlens"].long() - (s["cu"][1:] - s["cu"][:-1]).long())[seq]
    cos, sin = _angles(s, pos)
    page = s["case"]["page"]
    where, slot = s["table"].long()[seq, pos // page], pos % page
    s["k_cache"][where, :, slot] = _turned(_normed(s["k"], s["gk"]), cos, sin, s["rope"][1]).to(s["k"].dtype)
    s["v_cache"][where, :, slot] = s["v"]
    return {"q": _turned(_normed(s["q"], s["gq"]), cos, sin, s["rope"][1]).to(s["q"].dtype), "k_cache": s["k_cache"],
            "v_cache": s["v_cache"]}


def _plain_cached(s):
    c = s["case"]
    b, h, d = s["q"].shape
    hk = c["kv_heads"]
    table = s["table"].long().clamp(min=0)

    def pages(cache):
        return cache[table].permute(0, 2, 1, 3, 4).reshape(b * hk, -1, d).float()

    k, v = pages(s["k_cache"]), pages(s["v_cache"])
    p = torch.matmul(s["q"].float().reshape(b * hk, h // hk, d), k.transpose(1, 2)).mul_(s["scale"]).view(b, h, -1)
    p.masked_fill_((torch.arange(p.shape[-1], device=p.device)[None] >= s["seqlens"].long()[:, None])[:, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.div_(total).view(b * hk, h // hk, -1), v).view(b, h, d)
    return {"o": o.to(s["o"].dtype), "lse": (top + total.log()).squeeze(-1)}


_own = {"causal": _own_causal, "rope": _own_rope, "append": _own_append, "cached": _own_cached}
_plain = {"causal": _plain_causal, "rope": _plain_rope, "append": _plain_append, "cached": _plain_cached}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """The definition, sequence by sequence and token by token where that is quick enough, in float64."""
    s = prepare(case, seed)
    return {"causal": _exact_causal, "rope": _exact_rope, "append": _exact_append, "cached": _exact_cached}[case["op"]](s)


def _exact_causal(s):
    c, dev = s["case"], s["q"].device
    h, hk, t = c["heads"], c["kv_heads"], s["total"]
    names = ["o"] + (["dq", "dk", "dv"] if c["train"] else [])
    src = {"o": "q", "dq": "q", "dk": "k", "dv": "v"}
    out = {n: torch.zeros(s[src[n]].shape, dtype=torch.float64, device=dev) for n in names}
    out["lse"] = torch.zeros(h, t, dtype=torch.float64, device=dev)
    begin = 0
    for n in lengths(c):
        rows = slice(begin, begin + n)
        begin += n
        seen = torch.ones(n, n, dtype=torch.bool, device=dev).tril()
        for i in range(h):
            j = i * hk // h
            q, k, v = s["q"][rows, i].double(), s["k"][rows, j].double(), s["v"][rows, j].double()
            score = torch.where(seen, (q @ k.t()) * s["scale"], torch.full((), -math.inf, dtype=torch.float64, device=dev))
            lse = torch.logsumexp(score, 1)
            p = torch.exp(score - lse[:, None])
            del score
            out["lse"][i, rows] = lse
            out["o"][rows, i] = p @ v
            if c["train"]:
                do = s["do"][rows, i].double()
                dp = do @ v.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * s["scale"]
                out["dq"][rows, i] = ds @ k
                out["dk"][rows, j] += ds.t() @ q
                out["dv"][rows, j] += p.t() @ do
    return out


def _exact_pairs(r, layout):
    i = np.arange(r // 2)
    return (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)


def _exact_turn(x, pos, s):
    """The rotation as a product with complex numbers of modulus one."""
    freq, layout, magnitude = s["rope"]
    one, two = _exact_pairs(2 * freq.numel(), layout)
    z = torch.complex(x[..., one], x[..., two]) * torch.polar(torch.full((), magnitude, dtype=torch.float64, device=x.device).expand(
        pos.numel(), freq.numel()), pos.double()[:, None] * freq)[:, None]
    y = x.clone()
    y[..., one], y[..., two] = z.real, z.imag
    return y


def _exact_norm(x, gamma):
    x = x.double()
    return x if gamma is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gamma.double()


def _exact_positions(s):
    return torch.cat([torch.arange(n, device=s["cu"].device) for n in lengths(s["case"])])


def _exact_rope(s):
    pos = _exact_positions(s) + s["case"]["far"]
    out = {}
    for n, dy, gamma in (("q", "dq_out", "gq"), ("k", "dk_out", "gk")):
        x = s[n].double().requires_grad_(s["case"]["train"])
        w = None if s[gamma] is None else s[gamma].double().requires_grad_(s["case"]["train"])
        y = _exact_turn(_exact_norm(x, w), pos, s)
        out[n] = y.detach()
        if s["case"]["train"]:
            got = torch.autograd.grad(y, [x] if w is None else [x, w], s[dy].double())
            out["d" + n], out["d" + gamma] = got[0], (got[1] if w is not None else None)
    return out


def _exact_append(s):
    lens, page = lengths(s["case"]), s["case"]["page"]
    held = [n + c for n, c in zip(lens, contexts(s["case"]))]
    pos = torch.cat([torch.arange(m - n, m, device=s["q"].device) for n, m in zip(lens, held)])
    y, q = (_exact_turn(_exact_norm(s[n], s[g]), pos, s) for n, g in (("k", "gk"), ("q", "gq")))
    out = {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double(), "q": q}
    row = 0
    for b, n in enumerate(lens):
        p = pos[row:row + n]
        at = s["table"][b].long()[torch.div(p, page, rounding_mode="floor")] * page + p % page
        for name, x in (("k_cache", y), ("v_cache", s["v"].double())):
            flat = out[name].transpose(1, 2).reshape(-1, x.shape[1], x.shape[2])
            flat[at] = x[row:row + n]
            out[name] = flat.view(out[name].shape[0], page, x.shape[1], x.shape[2]).transpose(1, 2).contiguous()
        row += n
    return out


def _exact_cached(s):
    c = s["case"]
    out = {"o": torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device),
           "lse": torch.zeros(s["lse"].shape, dtype=torch.float64, device=s["q"].device)}
    for b, n in enumerate(lengths(c)):
        pages = s["table"][b, :-(-n // c["page"])].long()
        for j in range(c["kv_heads"]):
            k, v = (s[name][pages, j].reshape(-1, c["dim"])[:n].double() for name in ("k_cache", "v_cache"))
            g = c["heads"] // c["kv_heads"]
            score = s["q"][b, j * g:(j + 1) * g].double() @ k.t() * s["scale"]
            out["lse"][b, j * g:(j + 1) * g] = torch.logsumexp(score, 1)
            out["o"][b, j * g:(j + 1) * g] = torch.softmax(score, 1) @ v
    return out
