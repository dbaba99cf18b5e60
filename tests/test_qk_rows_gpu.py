"""Norm and rotation of query and key heads, forward and backward, and the same on the way into a paged
cache, against the formulas in float64 on the CPU.

Tolerances: a 16-bit output is off by the rounding of its value, eps / 2 relative, plus what fp32 arithmetic adds, which is
counted as 2^-20 of the largest magnitude that enters the element (the two channels of a pair, after the norm); a
backward's dx sums over the head: 2^-18 of the head's largest term."""
import math

import pytest
import torch

from paper_2208_08124_amd import fmha

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def pairs(rot, layout):
    i = torch.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def turn(x, pos, rope, back=False):
    """[T, H, D] float64 turned by pos * inv_freq."""
    if rope is None:
        return x
    freq, layout, m = rope
    a, b = pairs(2 * freq.numel(), layout)
    ang = pos.double()[:, None] * freq.double().cpu()[None]
    cos, sin = ang.cos()[:, None] * m, ang.sin()[:, None] * m * (-1 if back else 1)
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., a] * sin + x[..., b] * cos
    return y


def norm(x, gamma):
    return x if gamma is None else x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gamma.double().cpu()


def close(got, want, dtype, scale, what, share=2.0 ** -20):
    got, want = got.double().cpu(), want
    tol = want.abs() * torch.finfo(dtype).eps / 2 + share * scale + torch.finfo(dtype).tiny * 2.0 ** -(8 if dtype == torch.bfloat16 else 11)
    bad = (got - want).abs() - tol
    assert torch.isfinite(got).all() and (bad <= 0).all(), (what, float(bad.max()))


def make(t, heads, dim, dtype, seed, spare=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(t, heads * dim + spare, generator=g).to(DT[dtype]).cuda()
    return x[:, :heads * dim].unflatten(1, (heads, dim)) if heads else None


def positions_of(lens):
    return torch.cat([torch.arange(n) for n in lens]) if lens else torch.zeros(0, dtype=torch.long)


def cu_of(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device="cuda")


CASES = [  # lens, Hq, Hk, D, rotary, layout, normed, magnitude
    ([1], 1, 1, 16, 16, "half", True, 1.0),
    ([5, 0, 3], 2, 1, 16, 16, "interleaved", True, 1.0),
    ([37, 1, 0, 90], 12, 4, 64, 64, "half", True, 1.0),
    ([37, 1, 0, 90], 12, 12, 64, 32, "interleaved", False, 1.0),
    ([130, 7], 8, 1, 128, 128, "half", True, 1.1),
    ([130, 7], 32, 8, 128, 96, "half", True, 1.0),
    ([130, 7], 3, 3, 128, 48, "interleaved", True, 0.9),
    ([65], 6, 2, 96, 80, "half", True, 1.0),
    ([65], 5, 0, 96, 96, "interleaved", True, 1.0),
    ([33], 0, 3, 80, 16, "half", True, 1.0),
    ([70, 2], 4, 2, 256, 256, "half", True, 1.0),
    ([70, 2], 4, 2, 256, 64, "interleaved", True, 1.0),
    ([9] * 70, 2, 2, 64, 64, "half", True, 1.0),          # more sequences than lanes
    ([1, 0] * 2500 + [40], 1, 1, 64, 64, "half", False, 1.0),  # two levels of the search and a third
    ([2000, 1500], 16, 2, 128, 128, "half", True, 1.0),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d_%d+%d_of_%d" % (len(c[0]), sum(c[0]), *c[1:4]))
def test_forward_and_backward(case, dtype):
    lens, hq, hk, d, rot, layout, normed, magnitude = case
    t = sum(lens)
    pos, cu = positions_of(lens), cu_of(lens)
    freq, _ = fmha.fmha_rope_frequencies(rot)
    rope = (freq.cuda(), layout, magnitude)
    q, k = make(t, hq, d, dtype, 1, spare=8), make(t, hk, d, dtype, 2)
    dyq, dyk = make(t, hq, d, dtype, 3), make(t, hk, d, dtype, 4, spare=16)
    g = torch.Generator().manual_seed(5)
    gq, gk = ((1 + 0.3 * torch.randn(d, generator=g)).cuda() if normed else None for _ in range(2))
    new = lambda x: None if x is None else torch.full_like(x, float("nan"), memory_format=torch.contiguous_format)
    q_out, k_out, dq, dk = new(q), new(k), new(q), new(k)
    dgq, dgk = (torch.full((d,), float("nan"), device="cuda") if normed and h else None for h in (hq, hk))
    how = dict(rope=rope, gamma_q=gq, gamma_k=gk, eps=EPS, cu_seqlens=cu)
    fmha.fmha_qk_norm_rope_fwd(q, k, q_out, k_out, **how)
    ws = fmha.alloc_qk_norm_rope_workspace(t, hq, hk, d)
    keep = (q, k) if normed else (None, None)
    fmha.fmha_qk_norm_rope_bwd(dyq, dyk, *keep, dq, dk, dgq, dgk, ws, **how)
    for x, y, dy, dx, gamma, dgamma in ((q, q_out, dyq, dq, gq, dgq), (k, k_out, dyk, dk, gk, dgk)):
        if x is None:
            continue
        x64 = x.double().cpu()
        z = norm(x64, gamma)
        close(y, turn(z, pos, rope), DT[dtype], 2 * magnitude * z.abs().amax(-1, keepdim=True), "y")
        gr = turn(dy.double().cpu(), pos, rope, back=True)
        if gamma is None:
            close(dx, gr, DT[dtype], 2 * gr.abs().amax(-1, keepdim=True), "dx")
            continue
        w = gamma.double().cpu()
        rstd = 1 / (x64.square().mean(-1, keepdim=True) + EPS).sqrt()
        xh = x64 * rstd
        want = rstd * (gr * w - xh * (gr * w * xh).mean(-1, keepdim=True))
        term = (rstd * (gr * w).abs()).amax(-1, keepdim=True) * (1 + xh.abs().amax(-1, keepdim=True))
        close(dx, want, DT[dtype], term, "dx", 2.0 ** -18)
        # fp32 products, and a sum whose partial sums are at most the sum of magnitudes
        terms = gr * xh
        err = (dgamma.double().cpu() - terms.sum((0, 1))).abs()
        assert (err <= terms.abs().sum((0, 1)) * 2.0 ** -20 + 1e-30).all(), float(err.max())


def test_gradients_against_differences():
    """The backward against central differences of the float64 forward, along random directions.  The difference of a function
    with third derivatives of order one is off by about h^2; dx carries its 16-bit rounding."""
    lens, h, d, rot = [7, 4], 2, 64, 32
    t = sum(lens)
    freq, _ = fmha.fmha_rope_frequencies(rot)
    rope, pos = (freq.cuda(), "half", 1.0), positions_of(lens)
    q, dy = make(t, h, d, "f16", 1), make(t, h, d, "f16", 2)
    gamma = (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(3))).cuda()
    dq, dg = torch.empty_like(q), torch.empty(d, device="cuda")
    fmha.fmha_qk_norm_rope_bwd(dy, None, q, None, dq, None, dg, None, fmha.alloc_qk_norm_rope_workspace(t, h, 0, d), rope=rope,
                               gamma_q=gamma, eps=EPS, cu_seqlens=cu_of(lens))
    f = lambda x, w: float((turn(norm(x, w), pos, rope) * dy.double().cpu()).sum())
    x, w, step = q.double().cpu(), gamma.double().cpu(), 1e-4
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        u, r = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(d, generator=g, dtype=torch.float64)
        along = (f(x + step * u, w) - f(x - step * u, w)) / (2 * step)
        room = float((u * dq.double().cpu()).abs().sum()) * 2.0 ** -11 + 1e-5
        assert abs(along - float((u * dq.double().cpu()).sum())) <= room
        along = (f(x, w + step * r) - f(x, w - step * r)) / (2 * step)
        assert abs(along - float((r * dg.double().cpu()).sum())) <= 1e-4


def test_far_positions_and_the_scalings():
    """Positions around a million, and negative ones: the angle is formed in 64 bits."""
    t, d = 64, 64
    pos = torch.tensor([1_000_000 + 977 * i for i in range(t // 2)] + [-5 * i for i in range(t // 4)]
                       + [2 ** 31 - 1 - i for i in range(t // 4)], dtype=torch.int32)
    for scaling in ("plain", "linear", "base", "parts"):
        freq, m = fmha.fmha_rope_frequencies(d, 10000.0, scaling, 8.0, 4096)
        for layout in ("half", "interleaved"):
            rope = (freq.cuda(), layout, m)
            q = make(t, 3, d, "f16", 1)
            out = torch.empty_like(q)
            fmha.fmha_qk_norm_rope_fwd(q, None, out, None, rope=rope, positions=pos.cuda())
            x = q.double().cpu()
            # (2^31 radians times 2^-53 of rounding in the product: below the share counted)
            close(out, turn(x, pos, rope), torch.float16, 2 * m * x.abs().amax(-1, keepdim=True), (scaling, layout))


@pytest.mark.parametrize("by", ["cu_seqlens", "n_rows"])
def test_rows_behind_the_last_sequence_stay_as_they_are(by):
    t, present, d = 50, 31, 128
    freq, _ = fmha.fmha_rope_frequencies(d)
    rope = (freq.cuda(), "half", 1.0)
    q, k, dyq, dyk = (make(t, h, d, "bf16", h) for h in (4, 2, 4, 2))
    gamma = torch.ones(d, device="cuda")
    for x in (q, k, dyq, dyk):
        x[present:] = float("nan")
    how = dict(rope=rope, gamma_q=gamma, gamma_k=gamma)
    if by == "cu_seqlens":
        how["cu_seqlens"] = cu_of([20, present - 20])
    else:
        how.update(positions=torch.arange(t, dtype=torch.int32, device="cuda"),
                   n_rows=torch.tensor([present], dtype=torch.int32, device="cuda"))
    outs = [torch.full_like(x, 7.0) for x in (q, k, q, k)]
    dg = [torch.empty(d, device="cuda") for _ in range(2)]
    fmha.fmha_qk_norm_rope_fwd(q, k, outs[0], outs[1], **how)
    fmha.fmha_qk_norm_rope_bwd(dyq, dyk, q, k, outs[2], outs[3], *dg, fmha.alloc_qk_norm_rope_workspace(t, 4, 2, d), **how)
    for o in outs:
        assert (o[present:] == 7).all() and torch.isfinite(o[:present]).all()
    assert all(torch.isfinite(x).all() for x in dg)


def test_in_place_and_without_rows():
    t, d = 40, 64
    freq, _ = fmha.fmha_rope_frequencies(32)
    how = dict(rope=(freq.cuda(), "interleaved", 1.0), cu_seqlens=cu_of([t]), gamma_q=torch.full((d,), 1.5, device="cuda"))
    q = make(t, 3, d, "f16", 1)
    apart, x = torch.empty_like(q), q.clone()
    fmha.fmha_qk_norm_rope_fwd(q, None, apart, None, **how)
    fmha.fmha_qk_norm_rope_fwd(x, None, x, None, **how)
    assert torch.equal(apart, x)
    ws, dg = fmha.alloc_qk_norm_rope_workspace(t, 3, 0, d), torch.empty(d, device="cuda")
    dy, dq = make(t, 3, d, "f16", 2), torch.empty_like(q)
    fmha.fmha_qk_norm_rope_bwd(dy, None, q, None, dq, None, dg, None, ws, **how)
    first = dg.clone()
    fmha.fmha_qk_norm_rope_bwd(dy, None, q, None, dy, None, dg, None, ws, **how)  # dq in the place of its dq_out
    assert torch.equal(dy, dq) and torch.equal(first, dg)
    # a batch without a token: gamma's gradient is still written
    none = torch.empty(0, 3, d, dtype=torch.float16, device="cuda")
    dg.fill_(float("nan"))
    fmha.fmha_qk_norm_rope_bwd(none, None, none, None, none, None, dg, None, ws, **dict(how, cu_seqlens=cu_of([0])))
    assert (dg == 0).all()


def test_one_row_far_apart():
    """Rows 2^24 elements apart: offsets beyond 32 bits."""
    rows, d, far = 200, 64, 1 << 24
    base = torch.zeros(rows * far, dtype=torch.float16, device="cuda")  # 6.7 GB
    q = base.as_strided((rows, 2, d), (far, d, 1))
    src = make(rows, 2, d, "f16", 9)
    q.copy_(src)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    freq, _ = fmha.fmha_rope_frequencies(d)
    rope = (freq.cuda(), "half", 1.0)
    out = torch.empty_like(src)
    fmha.fmha_qk_norm_rope_fwd(q, None, out, None, rope=rope, positions=pos)
    want = torch.empty_like(src)
    fmha.fmha_qk_norm_rope_fwd(src, None, want, None, rope=rope, positions=pos)
    assert torch.equal(out, want)


# ------------------------------------------------------------------------------------------- the cache
def append_case(lens, held, hq, hk, d, page, dtype, rot, layout, normed, stride_pages=0, seed=0):
    """Inputs, a cache with garbage, and what it has to be afterwards."""
    g = torch.Generator().manual_seed(seed)
    t, b = sum(lens), len(lens)
    cols = max(1, -(-max(held) // page))
    pages = b * cols + 2
    table = torch.randperm(pages, generator=g)[:b * cols].view(b, cols).to(torch.int32)
    full = [torch.randn(pages, 1 + stride_pages, hk, page, d, generator=g).to(DT[dtype]).cuda() for _ in range(2)]
    k_cache, v_cache = (x[:, 0] for x in full)
    k, v, q = make(t, hk, d, dtype, 1), make(t, hk, d, dtype, 2, spare=8), make(t, hq, d, dtype, 3)
    freq, _ = fmha.fmha_rope_frequencies(rot)
    rope = (freq.cuda(), layout, 1.0)
    gq, gk = ((1 + 0.3 * torch.randn(d, generator=g)).cuda() if normed else None for _ in range(2))
    pos = torch.cat([torch.arange(m - n, m) for n, m in zip(lens, held)]) if t else torch.zeros(0, dtype=torch.long)
    return dict(t=t, b=b, table=table, full=full, k_cache=k_cache, v_cache=v_cache, k=k, v=v, q=q, rope=rope, gq=gq, gk=gk,
                pos=pos, held=torch.tensor(held, dtype=torch.int32), lens=lens, page=page)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", [
    # lens, held, Hq, Hk, D, page, rotary, layout, normed, unrelated pages between
    ([1, 1, 1], [1, 40, 17], 4, 4, 64, 16, 64, "half", True, 0),
    ([5, 0, 130, 1], [5, 9, 200, 64], 8, 2, 128, 16, 128, "half", True, 1),
    ([5, 0, 130, 1], [5, 9, 200, 64], 0, 3, 64, 1, 32, "interleaved", False, 0),
    ([33, 700], [33, 700], 32, 8, 128, 64, 64, "half", True, 0),
    ([3] * 100, [3 + i for i in range(100)], 2, 1, 80, 8, 80, "interleaved", True, 0),
], ids=lambda c: "%dx%d_%d+%d_of_%d_page_%d" % (len(c[0]), sum(c[0]), *c[2:6]))
def test_append(case, dtype):
    lens, held, hq, hk, d, page, rot, layout, normed, between = case
    s = append_case(lens, held, hq, hk, d, page, dtype, rot, layout, normed, between)
    want = [x.clone() for x in s["full"]]
    q_out = None if s["q"] is None else torch.full_like(s["q"], float("nan"))
    cu = None if all(n == 1 for n in lens) else cu_of(lens)
    fmha.fmha_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"].cuda(), s["held"].cuda(), cu_seqlens=cu,
                           q=s["q"], q_out=q_out, rope=s["rope"], gamma_q=s["gq"], gamma_k=s["gk"], eps=EPS)
    z = norm(s["k"].double().cpu(), s["gk"])
    y = turn(z, s["pos"], s["rope"])
    row = 0
    seen = torch.zeros(s["full"][0].shape[0], page, dtype=torch.bool)
    for b, n in enumerate(lens):
        for i in range(n):
            p = int(s["pos"][row])
            g, slot = int(s["table"][b, p // page]), p % page
            close(s["k_cache"][g, :, slot], y[row], DT[dtype], 2 * z[row].abs().amax(-1, keepdim=True), ("k", b, i))
            assert torch.equal(s["v_cache"][g, :, slot], s["v"][row])
            seen[g, slot] = True
            row += 1
    for full, old in zip(s["full"], want):  # nothing else has changed
        old[:, 0] = torch.where(seen[:, None, :, None].cuda(), full[:, 0], old[:, 0])
        assert torch.equal(full, old)
    if s["q"] is not None:
        z = norm(s["q"].double().cpu(), s["gq"])
        close(q_out, turn(z, s["pos"], s["rope"]), DT[dtype], 2 * z.abs().amax(-1, keepdim=True), "q")


def test_append_drops_what_has_no_page():
    """Page numbers out of range, tokens behind the table, positions below zero, rows behind the last sequence."""
    lens, held, page, d = [4, 3, 2, 5], [4, 3, 1, 6], 2, 64
    s = append_case(lens, held, 2, 2, d, page, "f16", 64, "half", False)
    table = s["table"].clone()[:, :2].contiguous()  # sequence 3 has tokens 1 .. 5, its table ends at 3
    table[0, 1], table[1, 0] = -1, s["full"][0].shape[0]
    before = [x.clone() for x in s["full"]]
    k, v, q = (torch.cat([x, torch.full_like(x[:3], float("nan"))]) for x in (s["k"], s["v"], s["q"]))
    q_out = torch.full_like(q, 7.0)
    fmha.fmha_cache_append(k, v, s["k_cache"], s["v_cache"], table.cuda(), s["held"].cuda(), cu_seqlens=cu_of(lens), q=q,
                           q_out=q_out, rope=s["rope"])
    keep = {(0, 0), (0, 1), (1, 2), (2, 0), (3, 1), (3, 2), (3, 3)}  # (sequence, position) that have a place
    changed = (s["v_cache"] != before[1][:, 0]).any(-1).any(1).cpu()
    places = {(int(table[b, p // page]), p % page) for b, p in keep}
    assert {tuple(x) for x in changed.nonzero().tolist()} == places
    assert (q_out[14:] == 7).all() and torch.isfinite(q_out[:14]).all()


def test_append_beyond_32_bits():
    """A cache of more than 4 GiB, its last page written and nothing near its start."""
    hk, page, d, pages = 8, 64, 128, 34000  # 4.5 GB each
    k_cache, v_cache = (torch.zeros(pages, hk, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = make(1, hk, d, "bf16", 1), make(1, hk, d, "bf16", 2)
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda")
    fmha.fmha_cache_append(k, v, k_cache, v_cache, table, torch.tensor([page], dtype=torch.int32, device="cuda"))
    assert torch.equal(v_cache[-1, :, -1], v[0]) and torch.equal(k_cache[-1, :, -1], k[0])
    assert int((v_cache != 0).sum()) == int((v != 0).sum())


def test_streams_and_a_captured_graph():
    s = append_case([1, 1], [30, 2], 4, 2, 128, 16, "bf16", 128, "half", True)
    q_out = torch.empty_like(s["q"])
    table, held = s["table"].cuda(), s["held"].cuda()

    def call():
        fmha.fmha_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], table, held, q=s["q"], q_out=q_out, rope=s["rope"],
                               gamma_q=s["gq"], gamma_k=s["gk"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        s["k"].normal_()
        s["q"].normal_()
        held.copy_(torch.tensor([20 + i, 3 + i], dtype=torch.int32))
        call()
        want = [x.clone() for x in (q_out, s["k_cache"], s["v_cache"])]
        q_out.zero_()
        s["k_cache"][:] = 0
        s["v_cache"][:] = 0
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want[0])
        for got, w in zip((s["k_cache"], s["v_cache"]), want[1:]):
            p = [(int(s["table"][b, (int(held[b]) - 1) // 16]), (int(held[b]) - 1) % 16) for b in range(2)]
            assert all(torch.equal(got[g, :, at], w[g, :, at]) for g, at in p)
