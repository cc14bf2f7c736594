"""Host-side checks of the operators of xshare_ops.h: exported symbols, refused
arguments, workspace sizes.  Nothing is launched (no GPU needed)."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import ops_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "xshare_ops.h")
P = 1 << 20   # an aligned pointer that is never followed
SHAPE, PARAM, NULL, WORKSPACE, ALIGN = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def ops():
    from paper_2602_07265_gb300 import _build
    _build.build()
    from paper_2602_07265_gb300 import ops
    return ops


def test_library_exports_every_declared_symbol(ops):
    from paper_2602_07265_gb300 import _build
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(xshare_\w+)\s*\(", text)))
    assert len(names) == 8
    out = subprocess.run(["nm", "-D", "--defined-only", _build.LIB], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\bT (\w+)$", out, flags=re.M))
    assert set(names) <= exported
    for name in names:
        assert getattr(ops.LIB, name).argtypes is not None


def gate_rc(ops, logits=P, dtype=0, bias=None, emask=None, tmask=None, B=8, N=64, k=4, prm=None, ids=P, w=P, scores=None,
            counts=None, offsets=None, perm=None, ws=P, ws_bytes=1 << 30):
    prm = ops.gate_params() if prm is None else prm
    return ops.LIB.xshare_gate(logits, dtype, bias, emask, tmask, B, N, k, ctypes.byref(prm) if prm else None, ids, w,
                               scores, counts, offsets, perm, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), SHAPE), (dict(B=8193), SHAPE), (dict(N=0), SHAPE), (dict(N=1025), SHAPE), (dict(k=0), SHAPE),
    (dict(k=17), SHAPE), (dict(N=3, k=4), SHAPE), (dict(dtype=3), PARAM), (dict(dtype=-1), PARAM),
    (dict(logits=None), NULL), (dict(ids=None), NULL), (dict(w=None), NULL), (dict(prm=False), NULL),
    (dict(logits=P + 2), ALIGN), (dict(bias=P + 4), ALIGN), (dict(emask=P + 1), ALIGN), (dict(tmask=P + 1), ALIGN),
    (dict(scores=P + 8), ALIGN), (dict(perm=P + 4), ALIGN),
    (dict(perm=P, ws=None), WORKSPACE), (dict(counts=P, ws=P + 16), WORKSPACE), (dict(offsets=P, ws_bytes=64), WORKSPACE),
])
def test_gate_refuses(ops, kw, code):
    assert gate_rc(ops, **kw) == code


@pytest.mark.parametrize("prm", [
    dict(n_groups=0, top_groups=1), dict(n_groups=3), dict(n_groups=64), dict(n_groups=8, top_groups=0),
    dict(n_groups=8, top_groups=9), dict(group_top=0), dict(group_top=3), dict(renorm=2),
    dict(scale=float("inf")), dict(scale=float("nan")),
])
def test_gate_refuses_parameters(ops, prm):
    assert gate_rc(ops, prm=ops.gate_params(**prm)) == PARAM


def test_gate_refuses_a_scoring(ops):
    prm = ops.gate_params()
    prm.scoring = 2
    assert gate_rc(ops, prm=prm) == PARAM
    with pytest.raises(ValueError):
        ops.gate_params("tanh")


@pytest.mark.parametrize("kw,code", [
    (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 20) + 1), SHAPE),
    (dict(dtype=3), PARAM), (dict(x=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL),
    (dict(x=P + 8), ALIGN), (dict(q=P + 1), ALIGN), (dict(s=P + 4), ALIGN),
])
def test_quant_refuses(ops, kw, code):
    a = dict(x=P, dtype=1, M=4, K=256, q=P, s=P, **{})
    a.update(kw)
    assert ops.LIB.xshare_quant_fp8_rows(a["x"], a["dtype"], a["M"], a["K"], a["q"], a["s"], None) == code
    assert ops.LIB.xshare_quant_fp8_blocks(a["x"], a["dtype"], 1, a["M"], a["K"], a["q"], a["s"], None) == code


@pytest.mark.parametrize("n", [0, 1025])
def test_quant_blocks_refuses_a_count(ops, n):
    assert ops.LIB.xshare_quant_fp8_blocks(P, 1, n, 4, 256, P, P, None) == SHAPE


@pytest.mark.parametrize("kw,code", [
    (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=24), SHAPE), (dict(K=8), SHAPE),
    (dict(M=(1 << 20) + 1), SHAPE), (dict(E=0), SHAPE), (dict(E=1025), SHAPE),
    (dict(E=1024, N=1 << 20, off=P), 0), (dict(E=1024, N=1 << 21, off=P), SHAPE), (dict(E=2), NULL),
    (dict(yt=3), PARAM), (dict(a=None), NULL), (dict(sa=None), NULL), (dict(b=None), NULL), (dict(sb=None), NULL),
    (dict(y=None), NULL), (dict(a=P + 8), ALIGN), (dict(b=P + 8), ALIGN), (dict(y=P + 2), ALIGN),
    (dict(off=P + 4), ALIGN), (dict(stats=P + 4), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=P + 128), WORKSPACE),
    (dict(wb=0), WORKSPACE),
])
def test_matmul_refuses(ops, kw, code):
    a = dict(a=P, sa=P, b=P, sb=P, off=None, M=4, N=64, K=256, E=1, y=P, yt=1, stats=None, ws=P, wb=1 << 30)
    a.update(kw)
    if code == 0:   # accepted as far as the host can tell: only the workspace is asked
        assert ops.xshare_matmul_fp8_workspace_size(a["M"], a["N"], a["K"], a["E"]) > 0
        return
    assert ops.LIB.xshare_matmul_fp8(a["a"], a["sa"], a["b"], a["sb"], a["off"], a["M"], a["N"], a["K"], a["E"], a["y"],
                                     a["yt"], a["stats"], a["ws"], a["wb"], None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), SHAPE), (dict(B=8193), SHAPE), (dict(k=0), SHAPE), (dict(k=33), SHAPE), (dict(d=64), SHAPE),
    (dict(d=200), SHAPE), (dict(F=0), SHAPE), (dict(F=192), SHAPE), (dict(n=0), SHAPE), (dict(n=1025), SHAPE),
    (dict(n=1024, d=1 << 20, F=1 << 20), 0), (dict(x=None), NULL), (dict(ids=None), NULL), (dict(w=None), NULL),
    (dict(y=None), NULL), (dict(gate=None), NULL), (dict(down_s=None), NULL), (dict(ex=False), NULL),
    (dict(x=P + 2), ALIGN), (dict(up=P + 8), ALIGN), (dict(stats=P + 4), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(ws=P + 16), WORKSPACE), (dict(wb=4096), WORKSPACE),
])
def test_experts_refuses(ops, kw, code):
    a = dict(x=P, ids=P, w=P, B=4, k=2, d=256, F=128, y=P, stats=None, ws=P, wb=1 << 30, n=8, gate=P, up=P, down_s=P)
    a.update(kw)
    if code == 0:
        assert ops.xshare_experts_fp8_workspace_size(a["B"], a["n"], a["k"], a["d"], a["F"]) > 0
        return
    ex = ops._Fp8ExpertsStruct(gate=a["gate"], up=a["up"], down=P, gate_s=P, up_s=P, down_s=a["down_s"], n=a["n"])
    assert ops.LIB.xshare_experts_fp8(a["x"], a["ids"], a["w"], None if a.get("ex") is False else ctypes.byref(ex),
                                      a["B"], a["k"], a["d"], a["F"], a["y"], a["stats"], a["ws"], a["wb"], None) == code


def test_workspace_sizes(ops):
    assert ops.xshare_gate_workspace_size(0, 8, 2) == 0
    assert ops.xshare_gate_workspace_size(8192, 1024, 16) >= 8192 * 16 * 4
    assert ops.xshare_matmul_fp8_workspace_size(8, 8, 24) == 0
    assert ops.xshare_experts_fp8_workspace_size(8, 8, 2, 100, 128) == 0
    small, large = (ops.xshare_experts_fp8_workspace_size(B, 64, 8, 2048, 1024) for B in (1, 8192))
    assert 0 < small < large
    # 64-bit sizes: 8192 tokens of 32 slots.
    assert ops.xshare_experts_fp8_workspace_size(8192, 64, 32, 7168, 2048) > 8192 * 32 * 7168 * 3


def test_binding_refuses(ops):
    with pytest.raises(ValueError):
        ops.xshare_gate(torch.zeros(2, 8), 2, ops.gate_params(), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2))
    with pytest.raises(ValueError):
        ops.xshare_quant_fp8_rows(torch.zeros(2, 8), torch.zeros(2, 9, dtype=ops.FP8), torch.zeros(2, 1))
    with pytest.raises(ValueError):
        ops.xshare_quant_fp8_blocks(torch.zeros(8), torch.zeros(8, dtype=ops.FP8), torch.zeros(1))
    with pytest.raises(ValueError):   # two matrices without offsets
        ops.xshare_matmul_fp8(torch.zeros(2, 16, dtype=ops.FP8), torch.zeros(2, 1),
                              torch.zeros(2, 4, 16, dtype=ops.FP8), torch.zeros(2, 1, 1), torch.zeros(2, 4), None)
    z = lambda *s: torch.zeros(*s)  # noqa: E731
    with pytest.raises(ValueError):   # widths that are no multiples of 128
        ops.Fp8Experts(z(2, 64, 128), z(2, 1, 1), z(2, 64, 128), z(2, 1, 1), z(2, 128, 64), z(2, 1, 1))


def test_reference_rounding_is_torchs():
    """The plain e4m3 rounding against torch's conversion, over every pair of
    neighbouring values, their middle and both sides of it."""
    v = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(0)),
                        np.nextafter(mid.astype(np.float32), np.float32(500))]).astype(np.float32)
    x = np.concatenate([x, -x])
    assert np.array_equal(R.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def gate_tensors(B=4, N=8, k=2):
    return dict(logits=torch.zeros(B, N), k=k, topk_ids=torch.zeros(B, k, dtype=torch.int32), topk_w=torch.zeros(B, k),
                scores_out=torch.zeros(B, N))


@pytest.mark.parametrize("name,shape", [("topk_ids", (2, 4)), ("topk_ids", (4, 6)), ("topk_ids", (8,)), ("topk_ids", (3, 2)),
                                        ("topk_w", (2, 4)), ("topk_w", (4, 3)), ("topk_w", (5, 2)),
                                        ("scores_out", (8, 4)), ("scores_out", (4, 9)), ("scores_out", (32,))])
def test_gate_binding_refuses_shapes(ops, name, shape):
    """Buffers that are large enough but of another shape: their rows would not be the tokens'."""
    a = gate_tensors()
    a[name] = torch.zeros(*shape, dtype=a[name].dtype)
    with pytest.raises(ValueError, match=name):
        ops.xshare_gate(a.pop("logits"), a.pop("k"), ops.gate_params(), a.pop("topk_ids"), a.pop("topk_w"), **a)
