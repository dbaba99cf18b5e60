"""The operators of a decoder's attention block as they are used together: a training pass, and a server's prompts
followed by single tokens.

Tolerances, in Frobenius norm.  Training: the norms and rotations, the probabilities, O (inside D), dS, and the outputs of each call
round once, eight times on the longest way; each rounding is at most eps / 2 of what it rounds, and what follows
is linear in it with a factor of about one (queries and keys are normed).  Serving: four (k, q, P, o)."""
import math

import pytest
import torch

from paper_2208_08124_amd import fmha

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def turned(x, pos, freq, layout):
    r = 2 * freq.numel()
    i = torch.arange(r // 2, device=x.device)
    a, b = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    angle = pos.double()[:, None] * freq
    z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def normed(x, gamma):
    return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gamma


def attention(q, k, v, scale):
    """[n, heads, D] queries that are the last n of the keys' tokens."""
    n, m, g = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0).contiguous()) * scale
    s = s.masked_fill(torch.arange(m, device=q.device)[None, :] > torch.arange(m - n, m, device=q.device)[:, None], -math.inf)
    return torch.matmul(torch.softmax(s, -1), v.transpose(0, 1).contiguous()).transpose(0, 1)


def near(got, want, dtype, roundings, what):
    want = want.detach()
    off = float((got.double() - want).norm() / want.norm())
    assert off <= roundings * torch.finfo(dtype).eps / 2, (what, off)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens,heads,kv,d,rot,layout", [
    ([200, 1, 0, 77, 130], 8, 2, 64, 64, "half"),
    ([200, 1, 0, 77, 130], 4, 4, 128, 64, "interleaved"),
    ([30, 17] * 50, 6, 3, 64, 32, "half"),
])
def test_training_pass(lens, heads, kv, d, rot, layout, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    t, dt = sum(lens), DT[dtype]
    new = lambda h: torch.randn(t, h, d, generator=g, device="cuda").to(dt)
    q, k, v, do = new(heads), new(kv), new(kv), new(heads)
    gq, gk = (1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
    freq = fmha.fmha_rope_frequencies(rot, 10000.0, "parts", 4.0, 128)[0].cuda()
    cu = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    how = dict(rope=(freq, layout, 1.0), gamma_q=gq, gamma_k=gk, eps=EPS, cu_seqlens=cu)
    qn, kn, o = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    lse = torch.empty(heads, t, device="cuda")
    ws = fmha.alloc_causal_workspace(len(lens), t, heads, kv, d, True)
    dqn, dkn, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dgq, dgk = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    scale = d ** -0.5
    fmha.fmha_qk_norm_rope_fwd(q, k, qn, kn, **how)
    fmha.fmha_causal_fwd(qn, kn, v, cu, max(lens), scale, o, lse, ws)
    fmha.fmha_causal_bwd(qn, kn, v, o, do, lse, cu, max(lens), scale, dqn, dkn, dv, ws, reuse_schedule=True)
    fmha.fmha_qk_norm_rope_bwd(dqn, dkn, q, k, dqn, dkn, dgq, dgk, fmha.alloc_qk_norm_rope_workspace(t, heads, kv, d), **how)

    leaves = [x.double().requires_grad_() for x in (q, k, v, gq, gk)]
    pos = torch.cat([torch.arange(n, device="cuda") for n in lens])
    q64, k64 = (turned(normed(leaves[i], leaves[i + 3]), pos, freq, layout) for i in (0, 1))
    outs, start = [], 0
    for n in lens:
        r = slice(start, start + n)
        start += n
        outs.append(attention(q64[r], k64[r], leaves[2][r], scale))
    want = torch.cat(outs)
    near(o, want, dt, 4, "o")
    grads = torch.autograd.grad(want, leaves, do.double())
    for name, got, ref in zip(("dq", "dk", "dv", "dgamma_q", "dgamma_k"), (dqn, dkn, dv, dgq, dgk), grads):
        near(got, ref, dt, 8, name)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,d,page,rot,layout", [(8, 2, 128, 16, 128, "half"), (6, 6, 64, 64, 32, "interleaved"), (20, 1, 64, 1, 64, "half")])
def test_prompts_and_then_single_tokens(heads, kv, d, page, rot, layout, dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    lens, steps, dt, scale = [150, 1, 33, 64], 3, DT[dtype], d ** -0.5
    b, t = len(lens), sum(lens)
    new = lambda n, h: torch.randn(n, h, d, generator=g, device="cuda").to(dt)
    gq, gk = (1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
    freq = fmha.fmha_rope_frequencies(rot)[0].cuda()
    how = dict(rope=(freq, layout, 1.0), gamma_q=gq, gamma_k=gk, eps=EPS)
    cols = -(-(max(lens) + steps) // page)
    table = torch.randperm(b * cols, generator=g, device="cuda").to(torch.int32).view(b, cols).contiguous()
    k_cache, v_cache = (torch.full((b * cols, kv, page, d), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    cu = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    held = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q, k, v = new(t, heads), new(t, kv), new(t, kv)
    qn, kn, qc, o = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(heads, t, device="cuda")
    fmha.fmha_qk_norm_rope_fwd(q, k, qn, kn, cu_seqlens=cu, **how)
    fmha.fmha_causal_fwd(qn, kn, v, cu, max(lens), scale, o, lse, fmha.alloc_causal_workspace(b, t, heads, kv, d, False))
    fmha.fmha_cache_append(k, v, k_cache, v_cache, table, held, cu_seqlens=cu, q=q, q_out=qc, **how)
    assert torch.equal(qc, qn)  # the same arithmetic on both ways

    keys = [list(x) for x in (k.split(lens), v.split(lens))]

    def reference(i, q_raw):
        n = keys[0][i].shape[0]
        pos = torch.arange(n, device="cuda")
        k64 = turned(normed(keys[0][i].double(), gk.double()), pos, freq, layout)
        q64 = turned(normed(q_raw.double(), gq.double()), pos[n - q_raw.shape[0]:], freq, layout)
        return attention(q64, k64, keys[1][i].double(), scale)

    near(o, torch.cat([reference(i, x) for i, x in enumerate(q.split(lens))]), dt, 4, "prompts")
    ws = fmha.alloc_cache_attention_workspace(b, heads, kv, d, max(lens) + steps)
    last = torch.empty(b, heads, d, dtype=dt, device="cuda")
    lse1 = torch.empty(b, heads, device="cuda")
    ends = cu[1:].long() - 1
    fmha.fmha_cache_attention(qn[ends].contiguous(), k_cache, v_cache, table, held, max(lens), scale, last, lse1, ws)
    near(last, o[ends].double(), dt, 4, "the prompts' last tokens")
    assert float((lse1 - lse[:, ends].t()).abs().max()) <= 2.0 ** -18 * (1 + float(lse1.abs().max()))
    for step in range(steps):
        q, k, v = new(b, heads), new(b, kv), new(b, kv)
        held += 1
        fmha.fmha_cache_append(k, v, k_cache, v_cache, table, held, q=q, q_out=q.clone(), **how)
        q_out = torch.empty_like(q)
        fmha.fmha_cache_append(k, v, k_cache, v_cache, table, held, q=q, q_out=q_out, **how)  # (again: the same places, the same values)
        fmha.fmha_cache_attention(q_out, k_cache, v_cache, table, held, max(lens) + steps, scale, last, lse1, ws)
        for i in range(b):
            for x, y in zip(keys, (k, v)):
                x[i] = torch.cat([x[i], y[i:i + 1]])
        near(last, torch.cat([reference(i, q[i:i + 1]) for i in range(b)]), dt, 4, step)


def test_tensors_elsewhere_are_refused():
    q = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    lse, ws = torch.empty(2, 4, device="cuda"), fmha.alloc_causal_workspace(1, 4, 2, 2, 64, True)
    with pytest.raises(fmha.FmhaError):
        fmha.fmha_causal_fwd(q, q, q, cu, 4, 0.1, q.clone(), lse.cpu(), ws)
    with pytest.raises(fmha.FmhaError):
        fmha.fmha_causal_bwd(q, q, q, q, q, lse, cu.cpu(), 4, 0.1, q.clone(), q.clone(), q.clone(), ws)
    with pytest.raises(fmha.FmhaError):
        fmha.fmha_qk_norm_rope_fwd(q, None, q.cpu(), None, cu_seqlens=cu)
    table, held = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(fmha.FmhaError):
        fmha.fmha_cache_append(q, q, cache, cache.clone(), table.cpu(), held)
    with pytest.raises(fmha.FmhaError):
        fmha.fmha_cache_attention(q, cache, cache.cpu(), table, held, 1, 0.1, q.clone(), torch.empty(4, 2, device="cuda"), None)
