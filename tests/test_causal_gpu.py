"""Causal attention with grouped heads over packed sequences, forward and backward, against the formulas in float64.

Tolerances, element by element.  h = eps / 2 of the 16-bit type (a rounding), u = 2^-25 for fp16 (a rounding among its
subnormals, values up to 1) and 0 for bf16, f = 2^-16 for what fp32 scores, exponentials and sums add:
  O    h |O| + (h + f) sum p |v| + u sum |v| 2^8 / ...     (the probabilities are rounded before the second product; they may stand
                                                        up to 2^8 above or anywhere below the largest)
  dV   h |dV| + (h + f) sum p |dO| + u sum |dO|
  dS   (h + f) |dS| + f p (|dP| + |D|) + p dD + u,  with dD = sum |dO| (the tolerance of O), since D is formed from the stored O
  dQ   h |dQ| + |scale| sum (tolerance of dS) |K|,  dK likewise with Q
lse: 2^-20 (1 + |lse| + the largest |score|)."""
import math

import pytest
import torch

from paper_2208_08124_amd import fmha

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
F = 2.0 ** -16


class Batch:
    def __init__(self, lens, heads, kv_heads, d, dtype, seed=0, behind=0, scale=None, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.heads, self.kv_heads, self.d, self.dtype = lens, heads, kv_heads, d, DT[dtype]
        self.t = sum(lens) + behind
        self.scale = d ** -0.5 if scale is None else scale
        new = lambda h: (torch.randn(self.t, h, d, generator=g, device="cuda") * spread).to(self.dtype)
        self.q, self.k, self.v, self.do = new(heads), new(kv_heads), new(kv_heads), new(heads)
        self.cu = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
        self.longest = max(lens)
        nan = lambda x: torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda")
        self.o, self.dq, self.dk, self.dv = nan(self.q), nan(self.q), nan(self.k), nan(self.v)
        self.lse = torch.full((heads, self.t), float("nan"), device="cuda")
        self.ws = fmha.alloc_causal_workspace(len(lens), self.t, heads, kv_heads, d, True)

    def fwd(self, **kw):
        fmha.fmha_causal_fwd(self.q, self.k, self.v, self.cu, kw.pop("longest", self.longest), self.scale, self.o, self.lse, self.ws, **kw)

    def bwd(self, **kw):
        fmha.fmha_causal_bwd(self.q, self.k, self.v, self.o, self.do, self.lse, self.cu, kw.pop("longest", self.longest), self.scale,
                             self.dq, self.dk, self.dv, self.ws, **kw)

    def outputs(self):
        return [x.clone() for x in (self.o, self.lse, self.dq, self.dk, self.dv)]


def within(got, want, tol, what):
    off = (got.double() - want).abs() - tol
    assert torch.isfinite(got).all() and (off <= 0).all(), (what, float(off.max()))


def check(b, backward=True, sequences=None):
    h = torch.finfo(b.dtype).eps / 2
    u = 2.0 ** -25 if b.dtype == torch.float16 else 0.0
    group, start = b.heads // b.kv_heads, 0
    for i, n in enumerate(b.lens):
        rows = slice(start, start + n)
        start += n
        if n == 0 or (sequences is not None and i not in sequences):
            continue
        for j in range(b.kv_heads):
            k, v = b.k[rows, j].double(), b.v[rows, j].double()
            dk = torch.zeros_like(k)
            dv, dk_tol, dv_tol = dk.clone(), dk.clone(), dk.clone()
            for e in range(j * group, (j + 1) * group):
                q, do = b.q[rows, e].double(), b.do[rows, e].double()
                seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
                score = (q @ k.t() * b.scale).masked_fill(~seen, -math.inf)
                lse = torch.logsumexp(score, 1)
                p = torch.exp(score - lse[:, None])
                o = p @ v
                largest = score.masked_fill(~seen, 0).abs().amax(1)
                within(b.lse[e, rows], lse, 2.0 ** -20 * (1 + lse.abs() + largest), ("lse", i, e))
                o_tol = h * o.abs() + (h + F) * (p @ v.abs()) + u * seen.double() @ v.abs() * p.amax(1, keepdim=True) + 1e-7
                within(b.o[rows, e], o, o_tol, ("o", i, e))
                if not backward:
                    continue
                dp = do @ v.t()
                dsum = (do * o).sum(1, keepdim=True)
                ds = p * (dp - dsum)
                ds_tol = (h + F) * ds.abs() + F * p * (dp.abs() + dsum.abs()) + p * (do.abs() * o_tol).sum(1, keepdim=True) + u * seen.double()
                want = b.scale * ds @ k
                within(b.dq[rows, e], want, h * want.abs() + abs(b.scale) * ds_tol @ k.abs() + 1e-7, ("dq", i, e))
                dk += b.scale * ds.t() @ q
                dk_tol += abs(b.scale) * ds_tol.t() @ q.abs()
                dv += p.t() @ do
                dv_tol += (h + F) * (p.t() @ do.abs()) + u * seen.double().t() @ do.abs()
            if backward:
                within(b.dk[rows, j], dk, h * dk.abs() + dk_tol + 1e-7, ("dk", i, j))
                within(b.dv[rows, j], dv, h * dv.abs() + dv_tol + 1e-7, ("dv", i, j))


CASES = [  # lens, heads, kv_heads, D
    ([1], 1, 1, 64),
    ([1, 2, 0, 3], 2, 1, 128),
    ([31, 32, 33, 0, 63, 64, 65], 4, 2, 64),
    ([31, 32, 33, 0, 63, 64, 65], 4, 4, 128),
    ([127, 128, 129], 6, 2, 128),
    ([255, 1, 257, 192], 3, 1, 64),
    ([300], 16, 2, 128),
    ([700, 90], 8, 8, 64),
    ([1300, 5], 5, 5, 128),
    ([5, 0, 140] * 23, 2, 1, 64),         # more sequences than a wavefront has lanes: the list
    ([129, 7, 0, 64, 1] * 60, 1, 1, 128),
    ([2500], 2, 1, 64),
    ([1500], 8, 1, 128),                  # few key heads: the dK/dV pass in parts
    ([40, 1100, 0, 300], 12, 2, 64),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d_%d-%d_of_%d" % (len(c[0]), max(c[0]), *c[1:]))
def test_forward_and_backward(case, dtype):
    b = Batch(*case, dtype)
    b.fwd()
    b.bwd()
    check(b)


@pytest.mark.parametrize("scale", [0.0, -0.11, 0.9])
def test_scales(scale):
    b = Batch([200, 70], 4, 2, 64, "bf16", scale=scale)
    b.fwd()
    b.bwd()
    check(b)


def test_scores_that_climb_and_fall():
    """The running maximum is raised in every block, or never after the first."""
    for sign in (1, -1):
        b = Batch([600], 2, 1, 128, "f16")
        rise = torch.linspace(0, 60 * sign, 600, device="cuda")
        q = b.q[:, :1].float()
        q[:] = q[:1]
        b.q[:] = q.half()
        b.k[:, 0] = (rise[:, None] * q[0, 0] / q[0, 0].square().sum() / b.scale).half()
        b.fwd()
        b.bwd()
        check(b)


def test_rows_behind_the_last_sequence():
    """Neither read nor written: NaN there stays out, and what the outputs hold there stays."""
    for d, dtype in ((64, "bf16"), (128, "f16")):
        b = Batch([100, 29], 4, 2, d, dtype, behind=77)
        for x in (b.q, b.k, b.v, b.do):
            x[129:] = float("nan")
        for x in (b.o, b.dq, b.dk, b.dv):
            x[129:] = 7.0
        b.lse[:, 129:] = 7.0
        b.fwd()
        b.bwd()
        check(b)
        assert all((x[129:] == 7).all() for x in (b.o, b.dq, b.dk, b.dv)) and (b.lse[:, 129:] == 7).all()


def test_sequences_keep_to_themselves():
    """NaN and infinities in one sequence leave the others as they are; what comes later leaves what was earlier as it is."""
    b = Batch([50, 60, 70], 4, 2, 128, "bf16")
    b.fwd()
    b.bwd()
    want = b.outputs()
    for x, bad in zip((b.q, b.k, b.v, b.do), (float("nan"), float("inf"), float("-inf"), float("nan"))):
        x[50:110] = bad
    b.fwd()
    b.bwd()
    for x, w in zip(b.outputs(), want):
        if x.dim() == 2:
            x, w = x.t(), w.t()
        assert torch.equal(x[:50], w[:50]) and torch.equal(x[110:], w[110:])
    b = Batch([400], 2, 1, 64, "f16")
    b.fwd()
    want = b.o.clone()
    b.k[300:] *= 3
    b.v[300:] += 1
    b.fwd()
    assert torch.equal(b.o[:300], want[:300]) and not torch.equal(b.o[300:], want[300:])


def test_shared_heads_are_the_same_as_repeated_ones():
    b = Batch([333, 40], 6, 2, 128, "f16")
    b.fwd()
    b.bwd()
    r = Batch([333, 40], 6, 6, 128, "f16")
    r.q, r.do = b.q, b.do
    r.k, r.v = b.k.repeat_interleave(3, 1).contiguous(), b.v.repeat_interleave(3, 1).contiguous()
    r.fwd()
    r.bwd()
    assert torch.equal(b.o, r.o) and torch.equal(b.lse, r.lse) and torch.equal(b.dq, r.dq)
    for x, y in ((b.dk, r.dk), (b.dv, r.dv)):
        parts = y.view(-1, 2, 3, 128).double()
        # three roundings on one side, one on the other
        assert ((x.double() - parts.sum(2)).abs() <= 2.0 ** -11 * (parts.abs().sum(2) + x.double().abs()) + 1e-6).all()


@pytest.mark.parametrize("d", [64, 128])
def test_strides_and_one_buffer_for_all(d):
    b = Batch([150, 33, 64], 4, 2, d, "bf16")
    wide = torch.full((b.t, 8 * d + 24), 3.0, dtype=b.dtype, device="cuda")
    q, k, v = wide[:, :4 * d].unflatten(1, (4, d)), wide[:, 4 * d:6 * d].unflatten(1, (2, d)), wide[:, 6 * d:8 * d].unflatten(1, (2, d))
    for x, y in ((q, b.q), (k, b.k), (v, b.v)):
        x.copy_(y)
    b.fwd()
    b.bwd()
    want = b.outputs()
    grads = torch.full_like(wide, 5.0)
    out = torch.full((b.t, 9 * d), 5.0, dtype=b.dtype, device="cuda")
    b.q, b.k, b.v = q, k, v
    b.o = out[:, :4 * d].unflatten(1, (4, d))
    b.do = torch.cat([b.do, b.do], 1)[:, :4]
    b.dq, b.dk, b.dv = (grads[:, c].unflatten(1, (-1, d)) for c in (slice(0, 4 * d), slice(4 * d, 6 * d), slice(6 * d, 8 * d)))
    b.fwd()
    b.bwd()
    assert all(torch.equal(x, w) for x, w in zip(b.outputs(), want))
    assert (grads[:, 8 * d:] == 5).all() and (out[:, 4 * d:] == 5).all()


def test_wrong_bounds_on_the_length():
    for lens in ([500, 300, 40], [200, 3] * 40):
        b = Batch(lens, 3, 1, 64, "f16")
        b.fwd()
        b.bwd()
        want = b.outputs()
        for longest in (0, 1, 10 ** 6):
            for x in (b.o, b.lse, b.dq, b.dk, b.dv):
                x.fill_(float("nan"))
            b.fwd(longest=longest)
            b.bwd(longest=longest)
            assert all(torch.equal(x, w) for x, w in zip(b.outputs()[:3], want[:3])), longest
            check(b)  # (dK and dV may be summed in other parts)


def test_prefix_sums_that_disagree_with_the_sizes():
    """Device prefix sums beyond the tensors, or falling: results are of no use, but nothing outside is touched, and a
    well-formed sequence beside them is right."""
    b = Batch([100, 60, 90], 2, 1, 64, "f16")
    b.fwd()
    want = b.o.clone()
    for cu in ([0, 100, 900, 250], [0, 100, -5, 40], [0, 100, 2 ** 31 - 1, -2 ** 31]):
        b.cu.copy_(torch.tensor(cu, dtype=torch.int32))
        b.fwd()
        b.bwd()
        torch.cuda.synchronize()
        assert torch.equal(b.o[:40], want[:40])


@pytest.mark.parametrize("batch", [64, 400])
def test_prefix_sums_that_rise_again_and_again(batch):
    """More tiles than any well-formed prefix sums have: what stands behind the workspace and the rows is left alone."""
    b = Batch([1500], 8, 1, 128, "bf16", behind=100)
    b.cu = torch.tensor([0, 1500] * (batch // 2) + [0], dtype=torch.int32, device="cuda")
    n = fmha.fmha_causal_workspace_size(batch, b.t, 8, 1, 128, True)
    whole = torch.full((n + (1 << 20),), 7, dtype=torch.uint8, device="cuda")
    b.ws = whole[:n]
    b.fwd()
    b.bwd()
    torch.cuda.synchronize()
    assert (whole[n:] == 7).all()
    assert all(torch.isnan(x[1500:]).all() for x in (b.o, b.dq, b.dk, b.dv)) and torch.isnan(b.lse[:, 1500:]).all()


@pytest.mark.parametrize("batch", [1, 5, 300])
def test_nothing_but_empty_sequences(batch):
    b = Batch([0] * batch, 8, 1, 128, "f16", behind=2000)
    for longest in (0, 2000):
        b.fwd(longest=longest)
        b.bwd(longest=longest)
    assert all(torch.isnan(x).all() for x in b.outputs())


def test_reruns_reuse_of_the_list_and_refusal():
    b = Batch([129, 7, 0, 64, 1] * 60, 4, 2, 64, "bf16")
    b.fwd()
    b.bwd(reuse_schedule=True)
    want = b.outputs()
    for _ in range(3):
        b.fwd(reuse_schedule=True)
        b.bwd()
        assert all(torch.equal(x, w) for x, w in zip(b.outputs(), want))
    with pytest.raises(fmha.FmhaError):
        b.fwd(cu_seqlens_host=b.cu.cpu(), longest=100)
    b.ws = b.ws[:256]
    with pytest.raises(fmha.FmhaError) as e:
        b.fwd()
    assert e.value.code == fmha.FMHA_ERR_WORKSPACE


@pytest.mark.parametrize("heads,kv_heads,d", [(6, 2, 64), (4, 4, 64), (2, 1, 128)])
def test_reuse_after_a_forward_that_needs_no_list(heads, kv_heads, d):
    """More than 256 sequences of one tile each: the forward makes no list, so the backward has none to use again."""
    b = Batch([1 + (37 * i) % 100 for i in range(300)], heads, kv_heads, d, "bf16", seed=5)
    b.ws.fill_(0x7F)
    b.fwd()
    b.bwd(reuse_schedule=True)
    again = b.outputs()
    b.bwd()
    assert all(torch.equal(x, y) for x, y in zip(again, b.outputs()))
    check(b, sequences=range(0, 300, 23))


@pytest.mark.parametrize("longest", [0, 1])
def test_more_items_than_a_launch_has_workgroups(longest):
    """2^18 sequences of one token, 64 heads: a token's output is its value, its dV the sum of dO over the group."""
    b = Batch([1] * (1 << 18), 64, 8, 64, "bf16", seed=6)
    b.fwd(longest=longest)
    b.bwd(longest=longest)
    assert torch.equal(b.o.view(-1, 8, 8, 64), b.v[:, :, None].expand(-1, 8, 8, 64))
    want = b.do.view(-1, 8, 8, 64).float().sum(2)
    # eight summands in fp32: seven sums, each off by at most 2^-24 of the summands' magnitudes; then one rounding, on both sides
    assert ((b.dv.float() - want).abs() <= 2.0 ** -8 * want.abs() + 14 * 2.0 ** -24 * b.do.view(-1, 8, 8, 64).float().abs().sum(2)).all()
    # (dS = P (dP - D), D being rowsum(P o dP) for such rows: 64 products on both sides)
    tol = b.scale * 130 * 2.0 ** -24 * (b.do.float().abs() * b.o.float().abs()).sum(2, keepdim=True)
    assert (b.dq.float().abs() <= tol * b.k.float().abs().repeat_interleave(8, 1) + 1e-30).all()


def test_gradients_against_differences():
    """Central differences of the float64 forward along random directions, h^2 = 1e-8 of third derivatives of order one; the
    kernel's gradients carry their 16-bit roundings, 2^-9 of the sum of magnitudes."""
    b = Batch([40, 25], 4, 2, 64, "f16")
    b.fwd()
    b.bwd()
    x64 = [x.double() for x in (b.q, b.k, b.v)]

    def loss(q, k, v):
        total, start = 0.0, 0
        for n in b.lens:
            r = slice(start, start + n)
            start += n
            for e in range(4):
                s = (q[r, e] @ k[r, e // 2].t() * b.scale).masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf)
                total += float((torch.softmax(s, 1) @ v[r, e // 2] * b.do[r, e].double()).sum())
        return total

    for which, grad in enumerate((b.dq, b.dk, b.dv)):
        for seed in range(2):
            u = torch.randn(grad.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.float64)
            step = 1e-4
            moved = [[x + sg * step * u if i == which else x for i, x in enumerate(x64)] for sg in (1, -1)]
            along = (loss(*moved[0]) - loss(*moved[1])) / (2 * step)
            got = float((grad.double() * u).sum())
            assert abs(along - got) <= 2.0 ** -9 * float((grad.double() * u).abs().sum()) + 1e-4, (which, along, got)


def test_captured_graphs_on_two_streams():
    """Forward and backward captured twice, each with a workspace of its own, replayed together with new inputs."""
    bs = [Batch([300, 41], 4, 2, 128, "bf16", seed=1), Batch([30, 5] * 40, 4, 2, 128, "bf16", seed=2)]
    streams = [torch.cuda.Stream() for _ in bs]
    graphs = [torch.cuda.CUDAGraph() for _ in bs]
    for b in bs:
        b.fwd()
        b.bwd()
    torch.cuda.synchronize()
    for b, s, gr in zip(bs, streams, graphs):
        with torch.cuda.graph(gr, stream=s):
            b.fwd()
            b.bwd(reuse_schedule=True)
    for i in range(4):
        for b in bs:
            for x in (b.q, b.k, b.v, b.do):
                x.normal_()
        if i == 2:  # other lengths under the same graphs
            bs[0].cu.copy_(torch.tensor([0, 100, 341], dtype=torch.int32))
        wants = []
        for b in bs:
            b.fwd(longest=341)
            b.bwd(longest=341)
            wants.append(b.outputs())
            for x in (b.o, b.lse, b.dq, b.dk, b.dv):
                x.fill_(float("nan"))
        torch.cuda.synchronize()
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        for b, want in zip(bs, wants):
            assert all(torch.equal(x, w) for x, w in zip(b.outputs(), want)), i


def test_offsets_beyond_32_bits():
    """Rows 2^24 elements apart."""
    rows, d, far = 300, 64, 1 << 24
    b = Batch([rows], 1, 1, d, "f16")
    b.fwd()
    b.bwd()
    want = b.outputs()
    base = torch.zeros(rows * far, dtype=torch.float16, device="cuda")  # 10 GB
    k = base.as_strided((rows, 1, d), (far, d, 1))
    dk = base[4096:].as_strided((rows, 1, d), (far, d, 1))
    k.copy_(b.k)
    b.k, b.dk = k, dk
    b.fwd()
    b.bwd()
    assert all(torch.equal(x, w) for x, w in zip(b.outputs(), want))
