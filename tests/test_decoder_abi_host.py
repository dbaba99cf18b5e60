"""The entry points of a decoder's attention block without a GPU: struct layouts, the frequencies' formulas, workspace
sizes, and refusals.  Validation reads host memory only; the pointers below are never dereferenced."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2208_08124_amd", "libfmha_varlen.so")
HEADER = os.path.join(ROOT, "include", "fmha_varlen.h")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())")

BUF = np.zeros(8192, dtype=np.uint8)
P = (BUF.ctypes.data + 255) // 256 * 256  # stands for a device pointer


def layout_rows(tmp_path, structs):
    src = tmp_path / "layout.c"
    body = "".join('  printf("%%zu%s\\n", sizeof(%s)%s);\n' % (
        " %zu" * len(mirror._fields_), name, "".join(", offsetof(%s, %s)" % (name, f[0]) for f in mirror._fields_))
        for name, mirror in structs)
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "%s"\nint main(void) {\n%s  return 0;\n}\n' % (HEADER, body))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-o", str(exe), str(src)])
    return [[int(x) for x in l.split()] for l in subprocess.check_output([str(exe)]).decode().splitlines()]


def test_struct_layouts_against_the_c_compiler(tmp_path):
    from paper_2208_08124_amd import fmha
    structs = [("fmha_rope_t", fmha.RopeArgs), ("fmha_qk_params_t", fmha.QkParams), ("fmha_cache_t", fmha.Cache),
               ("fmha_append_params_t", fmha.AppendParams), ("fmha_causal_params_t", fmha.CausalParams)]
    for (name, mirror), row in zip(structs, layout_rows(tmp_path, structs)):
        assert row == [ctypes.sizeof(mirror)] + [getattr(mirror, f[0]).offset for f in mirror._fields_], name


def test_frequencies():
    from paper_2208_08124_amd import fmha
    i = np.arange(32)
    plain = 10000.0 ** (-2 * i / 64)
    got, m = fmha.fmha_rope_frequencies(64)
    assert m == 1.0 and np.allclose(got.numpy(), plain, rtol=1e-14)
    got, m = fmha.fmha_rope_frequencies(64, 500000.0, "linear", 4.0)
    assert m == 1.0 and np.allclose(got.numpy(), 500000.0 ** (-2 * i / 64) / 4, rtol=1e-14)
    got, m = fmha.fmha_rope_frequencies(64, 10000.0, "base", 8.0)
    assert got[0] == 1.0 and abs(float(got[-1]) / (plain[-1] / 8) - 1) < 1e-12  # ends: kept, and slowed by the factor
    got, m = fmha.fmha_rope_frequencies(64, 10000.0, "parts", 8.0, 4096, 32.0, 1.0)
    turns = 4096 * plain / (2 * math.pi)
    assert abs(m - (0.1 * math.log(8.0) + 1)) < 1e-6
    assert np.allclose(got.numpy()[turns > 40], plain[turns > 40], rtol=1e-14)
    assert np.allclose(got.numpy()[turns < 0.7], plain[turns < 0.7] / 8, rtol=1e-14)
    share = got.numpy() / plain
    assert (np.diff(share) <= 1e-15).all() and len(set(np.round(share, 6))) > 5
    low = math.floor(64 * math.log(4096 / (2 * math.pi * 32)) / (2 * math.log(10000)))
    high = math.ceil(64 * math.log(4096 / (2 * math.pi)) / (2 * math.log(10000)))
    ramp = np.clip((i - low) / (high - low), 0, 1)
    assert np.allclose(got.numpy(), plain * (1 - ramp) + plain / 8 * ramp, rtol=1e-14)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")), dict(scaling="other"),
                dict(scaling="base", factor=2.0, rotary_dim=2), dict(scaling="parts", factor=2.0),
                dict(scaling="parts", factor=2.0, original_context=10, fast=1.0, slow=1.0),
                dict(scaling="parts", factor=2.0, original_context=10, fast=1.0, slow=0.0)):
        with pytest.raises(fmha.FmhaError):
            fmha.fmha_rope_frequencies(**{"rotary_dim": 64, **bad})
    assert fmha.lib().fmha_rope_frequencies(64, 10000.0, 0, 1.0, 0, 0.0, 0.0, None, None) == fmha.FMHA_ERR_INVALID_ARG


def qk(fmha, **over):
    p = fmha.QkParams(rows=4, q_heads=2, k_heads=1, head_dim=64, dtype=0, eps=1e-6, gamma_q=P, gamma_k=P, cu_seqlens=P, batch=1)
    p.rope = fmha.RopeArgs(64, 0, P, 1.0)
    for n, v in over.items():
        setattr(p.rope if hasattr(fmha.RopeArgs, n) else p, n, v)
    return p


def test_norm_and_rotation_refusals():
    from paper_2208_08124_amd import fmha
    lib, (INV, UNS, WS) = fmha.lib(), (fmha.FMHA_ERR_INVALID_ARG, fmha.FMHA_ERR_UNSUPPORTED, fmha.FMHA_ERR_WORKSPACE)
    bad = [(dict(rows=-1), INV, "rows"), (dict(dtype=3), UNS, "dtype"), (dict(q_heads=-1), INV, "heads"), (dict(head_dim=72), INV, "head_dim"),
           (dict(head_dim=0), INV, "head_dim"), (dict(head_dim=272), UNS, "256"), (dict(eps=-1.0), INV, "eps"), (dict(eps=float("nan")), INV, "eps"),
           (dict(gamma_q=P + 4), INV, "gamma"), (dict(rotary_dim=24), INV, "rotary_dim"), (dict(rotary_dim=80), INV, "rotary_dim"),
           (dict(rotary_dim=-16), INV, "rotary_dim"), (dict(layout=2), INV, "layout"), (dict(inv_freq=None), INV, "inv_freq"),
           (dict(inv_freq=P + 4), INV, "inv_freq"), (dict(magnitude=float("inf")), INV, "magnitude"),
           (dict(cu_seqlens=None), INV, "positions"), (dict(batch=0), INV, "batch"), (dict(positions=P + 2), INV, "aligned"),
           (dict(q_stride=64), INV, "q_stride"), (dict(k_stride=68), INV, "k_stride"), (dict(q_out_stride=(1 << 24) + 8), INV, "q_out_stride")]
    for over, code, frag in bad:
        p = qk(fmha, **over)
        for rc in (lib.fmha_qk_norm_rope_fwd(ctypes.byref(p), P, P, P, P, None),
                   lib.fmha_qk_norm_rope_bwd(ctypes.byref(p), P, P, P, P, P, P, P, P, P, 1 << 20, None)):
            assert rc == code and frag in fmha.last_error(), (over, rc, fmha.last_error())
    p = ctypes.byref(qk(fmha))
    assert lib.fmha_qk_norm_rope_fwd(None, P, P, P, P, None) == INV
    for i in range(4):
        a = [P] * 4
        a[i] = None if i % 2 else P + 8
        assert lib.fmha_qk_norm_rope_fwd(p, *a, None) == INV, i
    for i in range(8):
        a = [P] * 8
        a[i] = None
        assert lib.fmha_qk_norm_rope_bwd(p, *a, P, 1 << 20, None) == INV, i
    assert lib.fmha_qk_norm_rope_bwd(p, *[P] * 8, None, 1 << 20, None) == WS
    assert lib.fmha_qk_norm_rope_bwd(p, *[P] * 8, P + 4, 1 << 20, None) == WS
    assert lib.fmha_qk_norm_rope_bwd(p, *[P] * 8, P, 8, None) == WS and "needed" in fmha.last_error()
    assert lib.fmha_qk_norm_rope_bwd(ctypes.byref(qk(fmha, dq_stride=64)), *[P] * 8, P, 1 << 20, None) == INV
    # nothing to do: no launch, and no pointers looked at
    assert lib.fmha_qk_norm_rope_fwd(ctypes.byref(qk(fmha, rows=0)), None, None, None, None, None) == 0
    f = fmha.fmha_qk_norm_rope_bwd_workspace_size
    assert f(-1, 1, 1, 64) == 0 and f(1, 1, 1, 60) == 0 and f(1, 1, 1, 512) == 0
    assert 0 < f(1, 1, 1, 64) <= f(100, 1, 1, 64) <= f(100000, 32, 8, 64) <= 1024 * 2 * 64 * 4


def cache(fmha, **over):
    c = fmha.Cache(batch=2, kv_heads=2, head_dim=64, dtype=1, page_size=16, num_pages=4, max_pages=2, block_table=P, seqlens=P)
    for n, v in over.items():
        setattr(c, n, v)
    return c


def append(fmha, **over):
    p = fmha.AppendParams(rows=2, q_heads=2, eps=1e-6)
    p.rope = fmha.RopeArgs(64, 0, P, 1.0)
    for n, v in over.items():
        setattr(p.rope if hasattr(fmha.RopeArgs, n) else p, n, v)
    return p


CACHE_REFUSALS = [(dict(batch=-1), "batch"), (dict(kv_heads=0), "kv_heads"), (dict(page_size=0), "page_size"), (dict(page_size=24), "page_size"),
                  (dict(page_size=1 << 17), "page_size"), (dict(num_pages=-1), "num_pages"), (dict(max_pages=-1), "max_pages"),
                  (dict(max_pages=(1 << 26) + 1), "max_pages"), (dict(page_stride=1024), "page_stride"), (dict(page_stride=2 * 16 * 64 + 4), "page_stride"),
                  (dict(block_table=None), "block_table"), (dict(seqlens=None), "seqlens"), (dict(seqlens=P + 2), "seqlens")]


def test_append_refusals():
    from paper_2208_08124_amd import fmha
    lib, (INV, UNS) = fmha.lib(), (fmha.FMHA_ERR_INVALID_ARG, fmha.FMHA_ERR_UNSUPPORTED)
    run = lambda c, p, *a: lib.fmha_cache_append(ctypes.byref(c), ctypes.byref(p), *(a or [P] * 6), None)
    for over, frag in CACHE_REFUSALS:
        assert run(cache(fmha, **over), append(fmha, **({"rows": over["batch"]} if "batch" in over else {}))) == INV, over
        assert frag in fmha.last_error(), (over, fmha.last_error())
    assert run(cache(fmha, dtype=4), append(fmha)) == UNS and run(cache(fmha, head_dim=512), append(fmha)) == UNS
    for over, frag in ((dict(rows=-1), "rows"), (dict(rows=3), "cu_seqlens"), (dict(eps=-1.0), "eps"), (dict(v_stride=64), "v_stride"),
                       (dict(k_stride=130), "k_stride"), (dict(q_heads=-2), "heads"), (dict(rotary_dim=72), "rotary_dim"),
                       (dict(gamma_k=P + 8), "gamma"), (dict(cu_seqlens=P + 1, rows=5), "cu_seqlens")):
        assert run(cache(fmha), append(fmha, **over)) == INV and frag in fmha.last_error(), (over, fmha.last_error())
    for i in range(6):
        a = [P] * 6
        a[i] = None
        assert run(cache(fmha), append(fmha), *a) == INV, i
    assert lib.fmha_cache_append(None, ctypes.byref(append(fmha)), *[P] * 6, None) == INV
    assert run(cache(fmha, batch=0), append(fmha, rows=0), *[None] * 6) == 0


def test_cache_attention_refusals():
    from paper_2208_08124_amd import fmha
    lib, (INV, UNS, WS) = fmha.lib(), (fmha.FMHA_ERR_INVALID_ARG, fmha.FMHA_ERR_UNSUPPORTED, fmha.FMHA_ERR_WORKSPACE)

    def run(c, heads=4, longest=4096, scale=0.125, q=P, qs=0, k=P, v=P, o=P, os_=0, lse=P, ws=P, nws=1 << 30):
        return lib.fmha_cache_attention(ctypes.byref(c) if c else None, heads, longest, scale, q, qs, k, v, o, os_, lse, ws, nws, None)

    for over, frag in CACHE_REFUSALS:
        assert run(cache(fmha, **over)) == INV and frag in fmha.last_error(), (over, fmha.last_error())
    assert run(None) == INV and run(cache(fmha, dtype=9)) == UNS and run(cache(fmha, head_dim=96)) == UNS
    for over in (dict(heads=3), dict(heads=0), dict(heads=-2), dict(scale=float("nan")), dict(scale=float("inf")), dict(qs=128), dict(os_=260),
                 dict(q=None), dict(o=None), dict(lse=None), dict(k=None), dict(v=None), dict(q=P + 2), dict(lse=P + 1)):
        assert run(cache(fmha), **over) == INV, over
    assert run(cache(fmha), ws=None) == WS and run(cache(fmha), ws=P + 16) == WS and run(cache(fmha), nws=64) == WS
    assert run(cache(fmha, batch=0), q=None, k=None, v=None, o=None, lse=None, ws=None) == 0
    f = fmha.fmha_cache_attention_workspace_size
    assert f(2, 4, 3, 64, 100) == 0 and f(2, 4, 2, 96, 100) == 0 and f(2, 4, 2, 64, -1) == 0
    assert f(2, 4, 2, 64, 100) == 0 and f(2, 4, 2, 64, 100000) > 0  # one workgroup each, and several


def test_sizes_that_no_launch_holds():
    """A launch has less than 2^32 threads."""
    from paper_2208_08124_amd import fmha
    lib, INV = fmha.lib(), fmha.FMHA_ERR_INVALID_ARG
    p = qk(fmha, rows=1 << 28, head_dim=256, q_heads=64, k_heads=64)
    assert lib.fmha_qk_norm_rope_fwd(ctypes.byref(p), P, P, P, P, None) == INV and "workgroups" in fmha.last_error(), fmha.last_error()
    c, p = cache(fmha, batch=1 << 28, kv_heads=64, head_dim=256), append(fmha, rows=1 << 28, q_heads=64)
    assert lib.fmha_cache_append(ctypes.byref(c), ctypes.byref(p), *[P] * 6, None) == INV and "workgroups" in fmha.last_error(), fmha.last_error()
    for batch, heads in ((1 << 23, 1), (1 << 20, 16)):
        c = cache(fmha, batch=batch, kv_heads=1)
        assert lib.fmha_cache_attention(ctypes.byref(c), heads, 4096, 0.125, P, 0, P, P, P, 0, P, P, 1 << 50, None) == INV
        assert "workgroups" in fmha.last_error(), fmha.last_error()


def causal(fmha, **over):
    p = fmha.CausalParams(batch=2, total_tokens=16, heads=4, kv_heads=2, head_dim=64, max_seqlen=8, dtype=0, scale=0.125, cu_seqlens=P,
                          workspace=P, workspace_bytes=1 << 20)
    keep = None
    for n, v in over.items():
        if n == "cu_host":
            keep = np.asarray(v, dtype=np.int32)
            n, v = "cu_seqlens_host", keep.ctypes.data
        setattr(p, n, v)
    return p, keep


def test_causal_refusals():
    from paper_2208_08124_amd import fmha
    lib, (INV, UNS, WS) = fmha.lib(), (fmha.FMHA_ERR_INVALID_ARG, fmha.FMHA_ERR_UNSUPPORTED, fmha.FMHA_ERR_WORKSPACE)
    bad = [(dict(head_dim=96), UNS, "head_dim"), (dict(dtype=2), UNS, "dtype"), (dict(batch=-1), INV, "batch"), (dict(total_tokens=-1), INV, "total"),
           (dict(heads=0), INV, "heads"), (dict(kv_heads=3), INV, "kv_heads"), (dict(kv_heads=0), INV, "kv_heads"), (dict(kv_heads=-2), INV, "kv_heads"),
           (dict(flags=2), INV, "flags"), (dict(scale=float("nan")), INV, "scale"), (dict(cu_seqlens=None), INV, "cu_seqlens"),
           (dict(cu_seqlens=P + 2), INV, "aligned"), (dict(total_tokens=2 ** 31 - 1, heads=65536, kv_heads=1), INV, "tiles"),
           (dict(cu_host=[1, 8, 16]), INV, "expected 0"), (dict(cu_host=[0, 8, 7]), INV, "decreases"), (dict(cu_host=[0, 8, 17]), INV, "max_seqlen"),
           (dict(cu_host=[0, 8, 16], total_tokens=15), INV, "exceeds"), (dict(workspace=None), WS, "null"), (dict(workspace=P + 16), WS, "aligned"),
           (dict(workspace_bytes=100), WS, "needed"), (dict(q_stride=64), INV, "q_stride"), (dict(k_stride=132), INV, "k_stride"),
           (dict(v_stride=(1 << 24) + 8), INV, "v_stride"), (dict(o_stride=8), INV, "o_stride")]
    for over, code, frag in bad:
        p, keep = causal(fmha, **over)
        for rc in (lib.fmha_causal_fwd(ctypes.byref(p), *[P] * 5, None), lib.fmha_causal_bwd(ctypes.byref(p), *[P] * 9, None)):
            assert rc == code and frag in fmha.last_error(), (over, rc, fmha.last_error())
    p, _ = causal(fmha)
    assert lib.fmha_causal_fwd(None, *[P] * 5, None) == INV
    for i in range(5):
        assert lib.fmha_causal_fwd(ctypes.byref(p), *[None if i == j else P for j in range(5)], None) == INV, i
    for i in range(9):
        assert lib.fmha_causal_bwd(ctypes.byref(p), *[P + 2 if i == j else P for j in range(9)], None) == INV, i
    for stride in ("do_stride", "dq_stride", "dk_stride", "dv_stride"):
        p, _ = causal(fmha, **{stride: 100})
        assert lib.fmha_causal_bwd(ctypes.byref(p), *[P] * 9, None) == INV and stride in fmha.last_error()
    p, _ = causal(fmha, total_tokens=0)
    assert lib.fmha_causal_fwd(ctypes.byref(p), *[None] * 5, None) == 0 and lib.fmha_causal_bwd(ctypes.byref(p), *[None] * 9, None) == 0
    f = fmha.fmha_causal_workspace_size
    assert f(-1, 10, 2, 1, 64, True) == 0 and f(1, 10, 3, 2, 64, True) == 0 and f(1, 10, 2, 1, 80, True) == 0
    assert 0 < f(1, 10, 2, 1, 64, False) < f(1, 10, 2, 1, 64, True) <= f(100, 10, 2, 1, 64, True) <= f(100, 10, 2, 2, 128, True)
