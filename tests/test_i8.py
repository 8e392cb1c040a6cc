"""Projections in 8-bit integers (include/ebrl_i8.h) against their formulas: codes and
scales of rows, products bit for bit; the calls that are refused."""
import ctypes
import math
import random

import numpy as np
import pytest
import torch

from paper_2609_27547_amd import ebrl as E

gpu = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
LEAST = 2.0 ** -100


# ------------------------------------------------------------ no GPU needed --

def _quant_args(**kw):
    a = E.I8QuantArgs(dtype=E.DTYPE_BF16, op=E.I8_ROWS, rows=3, cols=40, eps=1e-6, x=4096, ldx=40, codes=8192, ldc=48,
                      scales=12288)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dtype=-1), dict(op=3), dict(op=-1), dict(rows=-1), dict(cols=0), dict(cols=(1 << 20) + 1),
    dict(x=0), dict(x=4097), dict(dtype=0, x=4098), dict(ldx=39), dict(codes=0), dict(codes=8200), dict(ldc=40),
    dict(ldc=32), dict(scales=0), dict(scales=12290), dict(up=4096), dict(gain=4096), dict(op=1, eps=-1.0),
    dict(op=1, eps=float("nan")), dict(op=1, gain=4098), dict(op=2), dict(op=2, up=4096, ldup=39),
    dict(op=2, up=4097, ldup=40)])
def test_quant_refuses_arguments(bad):
    assert E.lib().ebrl_op_i8_quant(ctypes.byref(_quant_args(**bad)), None) == -1


@pytest.mark.parametrize("eps", [float("inf"), -float("inf"), float("nan"), -1e-30])
def test_quant_refuses_an_eps_that_is_not_finite(eps):
    """At every width: a root of infinity would give zeros."""
    for cols in (1, 40, 5000, 20000):
        a = _quant_args(op=E.I8_RMSNORM, eps=eps, rows=0, cols=cols, ldx=cols, ldc=(cols + 15) // 16 * 16)
        assert E.lib().ebrl_op_i8_quant(ctypes.byref(a), None) == -1


def _gemm_args(**kw):
    a = E.I8GemmArgs(dtype=E.DTYPE_FP32, M=5, N=7, K=32, a=4096, b=8192, lda=32, ldb=48, scale_a=12288, scale_b=16384,
                     c=20480, ldc=7)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(M=-1), dict(N=-1), dict(K=0), dict(K=24), dict(K=131072), dict(a=0), dict(b=0), dict(a=4104),
    dict(b=8196), dict(lda=16), dict(lda=40), dict(ldb=-48), dict(lda=1 << 23), dict(ldb=1 << 23), dict(scale_a=0),
    dict(scale_b=0), dict(scale_a=12290), dict(bias=2), dict(c=0), dict(c=20482), dict(ldc=6), dict(residual=24576),
    dict(residual=24578, ldr=7), dict(residual=20480, ldr=8), dict(M=1 << 30, N=1 << 30)])
def test_gemm_refuses_arguments(bad):
    assert E.lib().ebrl_op_i8_gemm(ctypes.byref(_gemm_args(**bad)), None) == -1


def test_calls_of_nothing_are_ok():
    assert E.lib().ebrl_op_i8_quant(ctypes.byref(_quant_args(rows=0)), None) == 0
    for kw in (dict(M=0), dict(N=0)):
        assert E.lib().ebrl_op_i8_gemm(ctypes.byref(_gemm_args(**kw)), None) == 0
        assert E.lib().ebrl_op_i8_gemm_workspace(ctypes.byref(_gemm_args(**kw))) == 0
    assert E.lib().ebrl_op_i8_gemm_workspace(ctypes.byref(_gemm_args(K=24))) == -1
    assert E.lib().ebrl_op_i8_quant(None, None) == -1 and E.lib().ebrl_op_i8_gemm(None, None) == -1


def test_plans_are_refused():
    plan = (ctypes.c_int32 * 6)()
    for m, n, k in ((0, 1, 16), (1, 0, 16), (-1, 1, 16), (1, 1, 15), (1, 1, 131072), (1 << 30, 1 << 30, 16)):
        assert E.lib().ebrl_op_i8_gemm_plan(m, n, k, plan) == -1
    assert E.lib().ebrl_op_i8_gemm_plan(1, 1, 16, None) == -1


def test_plan_refuses_sizes_past_32_bits():
    for size in (((1 << 32) + 5, 64, 64), (5, (1 << 32) + 64, 64), (5, 64, (1 << 32) + 64), (-(1 << 32) + 5, 64, 64)):
        with pytest.raises(E.EbrlError, match="do not hold"):
            E.i8_gemm_plan(*size)


@pytest.mark.parametrize("m,n,k,kernel", [
    # kernels that are 10 % or more ahead of the others
    (1, 4096, 4096, "decode"), (8, 4096, 11008, "decode"), (37, 22016, 4096, "decode"), (256, 1024, 4096, "decode"),
    (781, 33, 11056, "decode"), (4094, 21, 8624, "decode"), (591, 1024, 4096, "ring"), (800, 1024, 1024, "ring"), (800, 12288, 4096, "large"), (3200, 8192, 1024, "large"),
    (9216, 12288, 4096, "large")])
def test_plan_is_the_measured_best(m, n, k, kernel):
    assert E.i8_gemm_plan(m, n, k)["kernel"] == kernel


@pytest.mark.parametrize("m", [1, 7, 64, 300, 512, 513, 5000])
def test_workgroups_cover_the_output(m):
    """Every plan's workgroups, and its workspace, for sizes up to the largest."""
    for n in (1, 63, 1000, 22016, 1 << 20, 1 << 25):
        for k in (16, 1040, 11008, 131056):
            if -(-m // 32) * -(-n // 64) > 1 << 23:
                continue
            p = E.i8_gemm_plan(m, n, k)
            tiles = -(-m // p["rows"]) * -(-n // p["cols"])
            assert 1 <= p["workgroups"] <= 1 << 23
            if p["kernel"] != "large":
                assert p["workgroups"] == tiles * p["splits"]
            else:
                assert p["workgroups"] == (256 if tiles >= 256 else tiles * p["cut"]) and p["cut"] in (1, 2, 4)
            a = _gemm_args(M=m, N=n, K=k)
            need = E.lib().ebrl_op_i8_gemm_workspace(ctypes.byref(a))
            assert need == (p["splits"] * m * ((n + 3) // 4 * 4) * 4 if p["splits"] > 1 else 0)


def test_binding_refuses():
    x = torch.zeros((3, 40), dtype=torch.bfloat16)
    codes, scales = E.i8_alloc(3, 40, device="cpu")
    assert codes.shape == (3, 48)
    ok = dict(x=x, codes=codes, scales=scales)
    for bad in (dict(), dict(x=x.half()), dict(x=x[0]), dict(x=x.t()), dict(x=x[:2]), dict(codes=codes[:, :40]),
                dict(codes=codes.float()), dict(codes=codes[:2]), dict(scales=scales[:2]), dict(scales=scales.double()),
                dict(up=x.float()), dict(up=x, norm_eps=1e-6), dict(gain=torch.ones(40)),
                dict(norm_eps=1e-6, gain=torch.ones(39)), dict(norm_eps=1e-6, gain=torch.ones(40).double())):
        with pytest.raises(E.EbrlError):
            E.op_i8_quant(**{**ok, **bad})
    out = torch.zeros((3, 5))
    b, sb = E.i8_alloc(5, 40, device="cpu")
    ok = dict(a=codes, scale_a=scales, b=b, scale_b=sb, out=out)
    for bad in (dict(), dict(a=codes[:, :32]), dict(b=b.int()), dict(out=out.half()), dict(out=out[:, :4]),
                dict(out=out.t().contiguous().t()), dict(scale_a=sb), dict(bias=torch.ones(4)),
                dict(residual=out.bfloat16()), dict(stream=0), dict(a=codes[:, 8:24], b=b[:, :16])):
        with pytest.raises(E.EbrlError):
            E.op_i8_gemm(**{**ok, **bad})


class _Elsewhere(torch.Tensor):
    """A tensor that says it is on another device."""

    def get_device(self):
        return 1


def _elsewhere(t):
    return t.as_subclass(_Elsewhere)


def _quant_calls():
    x, ones = torch.zeros((3, 40), dtype=torch.bfloat16), torch.ones(40)
    codes, scales = E.i8_alloc(3, 40, device="cpu")
    wide = torch.zeros((3, 80), dtype=torch.bfloat16)
    ok = dict(x=x, codes=codes, scales=scales)
    normed, gated = dict(norm_eps=1e-6, gain=ones), dict(up=x)
    for kw in ({}, dict(norm_eps=1e-6), normed, gated, dict(x=wide[:, :40]), dict(up=wide[:, 40:]),
               dict(codes=torch.zeros((3, 96), dtype=torch.int8)[:, 16:64]), dict(x=wide[:1, ::2][:, :1].expand(3, 1))):
        yield "not on a GPU", ok | kw
    for t in (x.half(), x[0], x[None], x.int()):
        yield r"x is bfloat16 or float32 \[rows, width\]", ok | dict(x=t)
    for t in (codes.float(), codes[0], codes.view(torch.uint8), codes[None]):
        yield r"codes are int8 \[rows, K\]", ok | dict(codes=t)
    yield "codes have contiguous rows", ok | dict(codes=torch.zeros((3, 96), dtype=torch.int8)[:, ::2])
    yield "codes have contiguous rows", ok | dict(codes=torch.zeros((48, 3), dtype=torch.int8).t())
    for t in (codes[:2], codes[:, :40], codes[:, :47]):
        yield r"codes are \[3, 48\]", ok | dict(codes=t)
    yield r"x is torch.bfloat16 \[3, 40\] where", ok | dict(x=_elsewhere(x))
    yield "x has contiguous rows", ok | dict(x=wide[:, ::2])
    yield "x has contiguous rows", ok | dict(x=torch.zeros((40, 3)).t())
    for t in (x[:2], x[:, :39], x.float(), _elsewhere(x)):
        yield r"up is torch.bfloat16 \[3, 40\] where", ok | dict(up=t)
    yield "up has contiguous rows", ok | dict(up=wide[:, ::2])
    for t in (scales[:2], scales.double(), torch.ones(6)[::2], _elsewhere(scales)):
        yield "scales is 3 contiguous float32", ok | dict(scales=t)
    for t in (ones[:39], ones.double(), torch.ones(80)[::2], _elsewhere(ones)):
        yield "gain is 40 contiguous float32", ok | dict(norm_eps=1e-6, gain=t)
    for kw in (normed | gated, dict(norm_eps=1e-6, up=x), dict(gain=ones), dict(gain=ones, up=x)):
        yield "normed .* or gated", ok | kw


def _gemm_calls():
    (a, sa), (b, sb) = E.i8_alloc(3, 48, device="cpu"), E.i8_alloc(5, 48, device="cpu")
    out, work = torch.zeros((3, 5)), torch.zeros(64, dtype=torch.uint8)
    ok = dict(a=a, scale_a=sa, b=b, scale_b=sb, out=out)
    for kw in ({}, dict(residual=out), dict(bias=torch.ones(5)), dict(workspace=work), dict(workspace=work, stream=0),
               dict(out=torch.zeros((3, 9))[:, 2:7]), dict(residual=torch.zeros((3, 9))[:, 2:7])):
        yield "not on a GPU", ok | kw
    for name, t in (("a", a), ("b", b)):
        for bad in (t.int(), t[0], t.view(torch.uint8)) + ((_elsewhere(t),) if name == "b" else ()):
            yield rf"{name} are int8 \[rows, K\]", ok | {name: bad}
        yield f"{name} have contiguous rows", ok | {name: torch.zeros((len(t), 96), dtype=torch.int8)[:, ::2]}
        yield "a and b have rows of one width", ok | {name: t[:, :32]}
    for t in (out.half(), out[0], out.double()):
        yield r"out is bfloat16 or float32 \[rows, width\]", ok | dict(out=t)
    for t in (out[:2], out[:, :4], torch.zeros((5, 3)), _elsewhere(out)):
        yield r"out is torch.float32 \[3, 5\] where", ok | dict(out=t)
    yield "out has contiguous rows", ok | dict(out=torch.zeros((5, 3)).t())
    for t in (out[:2], out[:, :4], out.bfloat16(), _elsewhere(out)):
        yield r"residual is torch.float32 \[3, 5\] where", ok | dict(residual=t)
    yield "residual has contiguous rows", ok | dict(residual=torch.zeros((3, 10))[:, ::2])
    for name, n, t in (("scale_a", 3, sa), ("scale_b", 5, sb), ("bias", 5, torch.ones(5))):
        for bad in (t[1:], t.double(), torch.ones(2 * n)[::2], _elsewhere(t)):
            yield f"{name} is {n} contiguous float32", ok | {name: bad}
    yield "explicit stream needs a workspace", ok | dict(stream=0)
    for t in (torch.zeros((8, 16))[:, ::2], _elsewhere(work)):
        yield "workspace is contiguous and where", ok | dict(workspace=t)


@pytest.mark.parametrize("calls,op", [(_quant_calls, "op_i8_quant"), (_gemm_calls, "op_i8_gemm")], ids=["quant", "gemm"])
def test_binding_refuses_each_argument(calls, op):
    """By the check that is meant: calls that are right get as far as the one that asks for a GPU."""
    for message, kw in calls():
        with pytest.raises(E.EbrlError, match=message):
            getattr(E, op)(**kw)


def test_workspaces_are_refused():
    a, b = torch.zeros((3, 48), dtype=torch.int8), torch.zeros((5, 48), dtype=torch.int8)
    assert E.i8_gemm_workspace(a, b).device == a.device
    for args in ((a[0], b), (a, b[0]), (a[None], b)):
        with pytest.raises(E.EbrlError, match=r"codes are \[rows, K\]"):
            E.i8_gemm_workspace(*args)
    with pytest.raises(E.EbrlError, match="EINVAL|INVALID|ebrl_op_i8_gemm_workspace"):
        E.i8_gemm_workspace(a[:, :40], b[:, :40])


# --------------------------------------------------------- rows to codes --

def _values(op, x, up, gain, eps):
    """y in float64, row by row, from the formulas."""
    x = x.double().cpu().numpy()
    if op == E.I8_RMSNORM:
        g = 1.0 if gain is None else gain.double().cpu().numpy()
        return x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * g
    if op == E.I8_SWIGLU:
        with np.errstate(over="ignore"):
            return x / (1 + np.exp(-x)) * up.double().cpu().numpy()
    return x


def _check_codes(y, codes, scales):
    """Codes and scales of finite rows y.  y is known to 2^-50 of its size here and in the
    kernel; a quotient is at most 127, so codes are within 1/2 + 127 * 2^-48 of it, and a
    scale is within half a step (2^-24, and 2^-48) of max |y| / 127."""
    cols = y.shape[1]
    codes, s = codes.cpu().numpy().astype(np.float64), scales.cpu().numpy().astype(np.float64)
    want = np.maximum(np.abs(y).max(1) / 127, LEAST)
    assert (np.abs(s - want) <= want * (2.0 ** -24 + 2.0 ** -48)).all()
    q = y / s[:, None]
    assert (np.abs(codes[:, :cols] - q) <= 0.5 + 127 * 2.0 ** -48).all()
    assert (codes[:, cols:(cols + 15) // 16 * 16] == 0).all()


def _rows(rows, cols, dtype, g, pad=0, shift=0):
    """Rows with a few large columns, `pad` elements apart, `shift` elements off an aligned start."""
    x = torch.randn((rows, cols), generator=g) * torch.where(torch.rand(cols, generator=g) < 0.02, 8.0, 1.0)
    wide = torch.empty(shift + rows * (cols + pad), dtype=DT[dtype], device="cuda")
    at = wide.as_strided((rows, cols), (cols + pad, 1), shift)
    at.copy_(x)
    return at


OPS = {"rows": E.I8_ROWS, "norm": E.I8_RMSNORM, "gate": E.I8_SWIGLU}


@gpu
@pytest.mark.parametrize("op", list(OPS))
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [
    (1, 1, 0, 0), (2, 15, 0, 0), (3, 16, 0, 0), (5, 17, 3, 1), (1, 64, 0, 0), (7, 256, 8, 0), (4, 1000, 0, 0),
    (9, 1024, 0, 0), (9, 1024, 1, 1), (33, 1283, 0, 0), (3, 2048, 16, 8), (70, 4096, 0, 0), (2, 4104, 0, 0),
    (5, 8191, 1, 0), (6, 8192, 0, 0), (3, 11008, 11008, 0), (2, 16384, 0, 0), (2, 16400, 0, 3), (1, 70000, 0, 0),
    (300, 48, 0, 0), (1025, 512, 0, 0)])
def test_codes_are_the_formulas(op, dtype, rows, cols, pad, shift):
    g = torch.Generator().manual_seed(rows * 7 + cols)
    x = _rows(rows, cols, dtype, g, pad, shift)
    up = _rows(rows, cols, dtype, g, pad, shift) if op == "gate" else None
    gain = 1 + 0.1 * torch.randn(cols, generator=g).cuda() if op == "norm" and rows % 2 else None
    k = (cols + 15) // 16 * 16
    held = torch.full((rows, k + 32), 77, dtype=torch.int8, device="cuda")
    codes, scales = held[:, :k + 16], torch.empty(rows, device="cuda")
    E.op_i8_quant(x, codes, scales, up=up, gain=gain, norm_eps=1e-6 if op == "norm" else None)
    torch.cuda.synchronize()
    _check_codes(_values(OPS[op], x, up, gain, 1e-6), held, scales)
    assert (held[:, k:] == 77).all()
    if op == "rows":
        # both sides' quotients of two floats are the same number in 64 bits
        s = scales.double().cpu().numpy()
        assert (held[:, :cols].cpu().numpy() == np.rint(x.double().cpu().numpy() / s[:, None])).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_codes_at_ties(dtype):
    """Values that are whole and half steps exactly: ties go to the even code."""
    half = torch.arange(-254, 255, dtype=torch.float32) / 2
    if dtype == "bf16":
        half = half[half.bfloat16().float() == half]
    x = torch.stack([half * 0.25, half * 2.0 ** -90]).to(DT[dtype]).cuda()
    codes, scales = E.i8_alloc(*x.shape)
    E.op_i8_quant(x, codes, scales)
    assert scales.tolist() == [0.25, 2.0 ** -90]
    assert (codes[:, :x.shape[1]].cpu().float() == torch.round(half)).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("op", list(OPS))
@pytest.mark.parametrize("cols", [512, 1000, 2048, 4095, 8192, 11008, 16384, 20001])
def test_halves_go_to_the_even_code(op, dtype, cols):
    """Quotients that are halves exactly, scales whose reciprocal no number holds.  Normed rows of one size r and eps
    0, whose root is r; gates of 40 and more, whose silu is the gate itself in 64 bits.  Every y is s k / 2, k a whole
    number up to 254, so the scale is s and each code k / 2, halves to even."""
    g = torch.Generator().manual_seed(cols)
    rows = 12
    k = torch.randint(-253, 254, (rows, cols), generator=g).double()
    k[:, cols // 3] = 254
    r = torch.tensor([1, 2, 3, 5, 0.75, 7, 12, 96, 1, 11, 2.5, 40]).double()[:, None]
    if op == "norm":
        # the gain is one for all rows
        k[:] = k[0]
        s = torch.full((rows, 1), 3.0 if cols % 2 else 0.6875).double()
        sign = torch.where(torch.rand((rows, cols), generator=g) < 0.5, -1.0, 1.0).double()
        kw = dict(norm_eps=0.0, gain=(s[0] * k[0] / 2).float().cuda())
        x, k = r * sign, k * sign
    elif op == "gate":
        gate = torch.tensor([40, 44, 48, 52, 56, 60, 72, 80, 88, 96, 120, 1000]).double()[:, None]
        s = gate / 4
        x, kw = gate.expand(rows, cols), dict(up=(k / 8).to(DT[dtype]).cuda())
    else:
        # (bf16's eight bits hold 127 s for scales of one bit)
        s = torch.tensor([3, 5, 7, 9, 11, 13, 1.25, 0.375, 6, 10, 14, 1.75] if dtype == "fp32" else
                         [1, 2, 4, 0.5, 0.25, 8, 16, 32, 1, 2, 4, 8]).double()[:, None]
        x, kw = s * k / 2, {}
    codes, scales = E.i8_alloc(rows, cols)
    E.op_i8_quant(x.to(DT[dtype]).cuda(), codes, scales, **kw)
    assert torch.equal(scales.cpu().double(), s[:, 0])
    wrong = codes[:, :cols].cpu().double() != torch.round(k / 2)
    assert not wrong.any(), f"{int(wrong.sum())} of {wrong.numel()} codes"


@gpu
@pytest.mark.parametrize("cols", [24, 1024, 5000, 20000])
def test_rows_of_any_size_of_number(cols):
    """Zeros, numbers below the least scale, denormals, the largest floats."""
    g = torch.Generator().manual_seed(cols)
    base = torch.randn((8, cols), generator=g).clamp(-4, 4)
    size = torch.tensor([0.0, 2.0 ** -140, 2.0 ** -100, 2.0 ** -93, 1.0, 2.0 ** 100, 2.0 ** 125, 2.0 ** 20])
    x = (base * size[:, None]).cuda()
    for op in ("rows", "norm"):
        codes, scales = E.i8_alloc(8, cols)
        E.op_i8_quant(x, codes, scales, norm_eps=1e-30 if op == "norm" else None)
        _check_codes(_values(OPS[op], x, None, None, float(np.float32(1e-30))), codes, scales)
    codes, scales = E.i8_alloc(8, cols)
    E.op_i8_quant(torch.zeros_like(x), codes, scales, norm_eps=0.0)       # 0 / 0
    assert scales.isnan().all() and (codes == 0).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("op", list(OPS))
@pytest.mark.parametrize("cols", [33, 512, 1024, 4096, 11008, 20001])
def test_rows_that_are_not_finite(op, dtype, cols):
    """One such value, anywhere in a row, gives the row codes of zero and the scale NaN; its
    neighbours keep theirs."""
    g = torch.Generator().manual_seed(cols)
    x = _rows(9, cols, dtype, g)
    up = _rows(9, cols, dtype, g) if op == "gate" else None
    bad = {1: float("nan"), 3: float("inf"), 5: -float("inf"), 7: float("nan")}
    for i, (row, v) in enumerate(bad.items()):
        (up if op == "gate" and i % 2 == 0 else x)[row, (cols - 1) * i // 3] = v
    kw = dict(up=up, norm_eps=1e-6 if op == "norm" else None)
    codes, scales = E.i8_alloc(9, cols)
    codes.fill_(5)
    E.op_i8_quant(x, codes, scales, **kw)
    rows = sorted(bad)
    good = [r for r in range(9) if r not in bad]
    assert scales[rows].isnan().all() and (codes[rows] == 0).all()
    y = _values(OPS[op], x[good], None if up is None else up[good], None, 1e-6)
    _check_codes(y, codes[good], scales[good])


@gpu
@pytest.mark.parametrize("cols", [33, 1024, 4096, 11008, 20001])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_gains_that_are_not_finite(cols, bad):
    """A gain of NaN or infinity, also where the row has a zero, leaves no row finite; a gain of zero takes a
    column out, but not an infinity in it."""
    g = torch.Generator().manual_seed(cols)
    x = _rows(4, cols, "fp32", g)
    gain = torch.ones(cols, device="cuda")
    gain[cols // 2] = bad
    x[1, cols // 2] = 0
    codes, scales = E.i8_alloc(4, cols)
    codes.fill_(5)
    E.op_i8_quant(x, codes, scales, norm_eps=1e-6, gain=gain)
    assert scales.isnan().all() and (codes == 0).all()
    gain[cols // 2] = 0
    x[2, cols // 2] = bad
    E.op_i8_quant(x, codes, scales, norm_eps=1e-6, gain=gain)
    assert scales[2].isnan() and (codes[2] == 0).all()
    good = [0, 1, 3]
    _check_codes(_values(E.I8_RMSNORM, x[good], None, gain, 1e-6), codes[good], scales[good])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [500, 1000, 2000, 4000, 8000, 11008, 16384])
def test_gates_of_every_size(dtype, cols):
    """Gates over and past the range in which 32 bits do for most codes, products spread over the codes:
    up = t / silu(gate) makes them t, but for up's rounding."""
    g = torch.Generator().manual_seed(cols)
    for lo, hi in ((-80, 80), (-79.9, -60), (-3, 3), (30, 80), (-100, 100), (-700, 5), (79.5, 80.5)):
        gate = torch.linspace(lo, hi, 4 * cols).reshape(cols, 4).t().contiguous().to(DT[dtype])
        silu = gate.double() / (1 + torch.exp(-gate.double()))
        t = torch.rand((4, cols), generator=g).double() * 2 - 1
        up = (t / torch.where(silu.abs() < 1e-37, 1.0, silu)).clamp(-3e38, 3e38).to(DT[dtype])
        codes, scales = E.i8_alloc(4, cols)
        E.op_i8_quant(gate.cuda(), codes, scales, up=up.cuda())
        _check_codes(_values(E.I8_SWIGLU, gate, up, None, 0), codes, scales)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [500, 4000, 11008, 20000])
def test_gates_below_the_normal_floats(dtype, cols):
    """Denormal gates of few bits, whose halves no float holds, against factors near the largest float."""
    g = torch.Generator().manual_seed(cols)
    least = 2.0 ** (-149 if dtype == "fp32" else -133)
    gate = (torch.randint(-100, 101, (4, cols), generator=g).double() * least).to(DT[dtype])
    up = ((torch.rand((4, cols), generator=g) + 0.5) * 2.0 ** 127).to(DT[dtype])
    codes, scales = E.i8_alloc(4, cols)
    E.op_i8_quant(gate.cuda(), codes, scales, up=up.cuda())
    _check_codes(_values(E.I8_SWIGLU, gate, up, None, 0), codes, scales)


@gpu
@pytest.mark.parametrize("op", list(OPS))
@pytest.mark.parametrize("cols", [512, 1024, 4096, 11008])
def test_many_rows_of_codes(op, cols):
    """A million codes each: none next to a border is off."""
    g = torch.Generator().manual_seed(cols)
    rows = (1 << 20) // cols
    x, up = _rows(rows, cols, "bf16", g), _rows(rows, cols, "bf16", g) if op == "gate" else None
    codes, scales = E.i8_alloc(rows, cols)
    E.op_i8_quant(x, codes, scales, up=up, norm_eps=1e-6 if op == "norm" else None)
    _check_codes(_values(OPS[op], x, up, None, 1e-6), codes, scales)
    # rows whose values are all alike, and one value alone
    x.fill_(0.75)
    if up is not None:
        up.fill_(-3.0)
    x[1::2, 1:] = 0
    E.op_i8_quant(x, codes, scales, up=up, norm_eps=1e-6 if op == "norm" else None)
    _check_codes(_values(OPS[op], x, up, None, 1e-6), codes, scales)
    assert (codes[0].abs() == 127).all() and codes[1, 0].abs() == 127 and (codes[1, 1:] == 0).all()


@gpu
def test_more_rows_than_a_launch_takes():
    rows = (1 << 21) + 1000
    x = torch.zeros((rows, 16), dtype=torch.bfloat16, device="cuda")
    x[:, 3] = 1 + torch.arange(rows, device="cuda") % 100
    codes, scales = E.i8_alloc(rows, 16)
    E.op_i8_quant(x, codes, scales)
    assert (codes[:, 3] == 127).all() and (codes.int().abs().sum(1) == 127).all()
    assert torch.equal(scales, (x[:, 3].double() / 127).float())


@gpu
def test_scales_past_the_range():
    """silu(x) up that no float holds: the row counts as not finite."""
    x = torch.full((2, 64), 3e38, device="cuda")
    up = torch.full((2, 64), 3e38, device="cuda")
    up[1] = 1e-38
    codes, scales = E.i8_alloc(2, 64)
    E.op_i8_quant(x, codes, scales, up=up)
    assert scales[0].isnan() and (codes[0] == 0).all() and (codes[1] == 127).all()
    _check_codes(_values(2, x[1:], up[1:], None, 0), codes[1:], scales[1:])


# -------------------------------------------------------------- products --

def _operand(rows, k, g, ld=0):
    held = torch.randint(-128, 128, (rows, ld or k), generator=g, dtype=torch.int8).cuda()
    return held[:, :k], (torch.rand(rows, generator=g) + 0.5).cuda() * 2.0 ** -7


def _sums(a, b):
    """Whole-number products on the GPU in 64-bit floats: below 2^53, so exact."""
    return torch.matmul(a.double(), b.double().t())


def _expected(a, sa, b, sb, bias, residual, dtype):
    """The steps of the documentation, each rounded to 32 bits."""
    v = _sums(a, b).float() * sb[None, :]
    v = v * sa[:, None]
    if bias is not None:
        v = v + bias
    if residual is not None:
        v = v + residual.float()
    return v.to(DT[dtype])


def _same(x, y):
    return torch.equal(x.isnan(), y.isnan()) and torch.equal(x.nan_to_num(), y.nan_to_num())


SHAPES = [(1, 1, 16), (1, 16, 64), (1, 4096, 4096), (2, 33, 48), (3, 1000, 128), (8, 4096, 11008), (15, 100, 1040),
          (16, 64, 1024), (17, 257, 256), (31, 22016, 4096), (32, 96, 8192), (33, 1024, 1024), (37, 4100, 272),
          (48, 512, 131056), (64, 64, 64), (65, 2048, 2048), (100, 1003, 1296), (128, 128, 128), (129, 4096, 4096),
          (200, 300, 400), (255, 1024, 4096), (256, 1024, 11008), (257, 513, 192), (300, 12288, 4096), (424, 1024, 4096),
          (591, 1003, 1296), (800, 1000, 2064), (1024, 2048, 1024), (2048, 8192, 272), (2304, 1024, 4096),
          (781, 33, 11056), (1650, 16, 3328), (2151, 55, 10784), (8446, 26, 9024),
          (3200, 8192, 1024), (4097, 4100, 1040), (5476, 1024, 4096), (9216, 64, 80), (40000, 16, 128)]


@gpu
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_bit_for_bit(m, n, k):
    g = torch.Generator().manual_seed(m + n + k)
    for dtype, extra, bias, resid in (("fp32", 0, False, True), ("bf16", 32, True, False), ("bf16", 0, False, True)):
        a, sa = _operand(m, k, g, k + extra)
        b, sb = _operand(n, k, g, k + extra)
        if not extra and m > 2:
            sa[m // 2] = float("nan")
        bias = torch.randn(n, generator=g).cuda() if bias else None
        pad = 3 if extra else 0
        held = torch.full((m, n + pad), 9.0, dtype=DT[dtype], device="cuda")
        res = torch.randn((m, n), generator=g).to(DT[dtype]).cuda() if resid else None
        want = _expected(a, sa, b, sb, bias, res, dtype)
        work = E.i8_gemm_workspace(a, b)
        work.fill_(0xA5)
        E.op_i8_gemm(a, sa, b, sb, held[:, :n], bias=bias, residual=res, workspace=work)
        assert _same(held[:, :n], want), f"{dtype} {extra}"
        assert (held[:, n:] == 9).all()
        if resid:   # in place
            E.op_i8_gemm(a, sa, b, sb, res, bias=bias, residual=res, workspace=work)
            assert _same(res, want)


def _reaching():
    """The smallest of many shapes for each kernel and tile that the plan has."""
    r, found = random.Random(0), {}

    def size(lo, hi):
        return int(math.exp(r.uniform(math.log(lo), math.log(hi))))
    for _ in range(20000):
        m, n, k = size(1, 11000), size(1, 23000), 16 * size(1, 700)
        p = E.i8_gemm_plan(m, n, k)
        key = (p["kernel"], p["rows"], p["cols"], p["splits"] > 1, p["cut"], p["workgroups"] == 256,
               p["kernel"] == "decode" and m > p["rows"])
        if key not in found or m * n * k < math.prod(found[key]):
            found[key] = (m, n, k)
    return found


@gpu
def test_products_of_every_kernel():
    """Bit for bit, at odd sizes, with a bias and a residual in turn, outputs and floats of any alignment."""
    g = torch.Generator().manual_seed(1)
    found = _reaching()
    assert {k[0] for k in found} == {"large", "ring", "decode"} and len(found) > 40
    for i, (key, (m, n, k)) in enumerate(sorted(found.items(), key=str)):
        a, sa = _operand(m, k, g, k + 16 * (i % 3))
        b, sb = _operand(n, k, g)
        for dtype, shift in (("fp32", 0), ("bf16", 1)):
            bias = torch.randn(n + shift, generator=g).cuda()[shift:] if i % 2 == shift else None
            res = torch.randn((m, n), generator=g).to(DT[dtype]).cuda() if i % 4 < 2 else None
            sb2 = torch.cat([sb[:shift], sb])[shift:]
            held = torch.full((m * n + 8,), 3.0, dtype=DT[dtype], device="cuda")
            out = held[shift:shift + m * n].view(m, n)
            E.op_i8_gemm(a, sa, b, sb2, out, bias=bias, residual=res)
            assert _same(out, _expected(a, sa, b, sb2, bias, res, dtype)), f"{key} {m} x {n} x {k} {dtype}"
            assert (held[:shift] == 3).all() and (held[shift + m * n:] == 3).all()


@gpu
@pytest.mark.parametrize("m,k", [(2085, 512), (591, 1296), (1100, 2064), (4200, 272)])
@pytest.mark.parametrize("n", [4093, 4094, 4095, 4097, 4098, 4099, 4031, 4036, 4161])
def test_edges_of_large_products(m, n, k):
    """Last rows and columns of large tiles: one to three columns behind whole fours, of a wave, of a tile; bit for
    bit, the residual in place, rows of c at any element."""
    assert E.i8_gemm_plan(m, n, k)["kernel"] == "large"
    g = torch.Generator().manual_seed(n + m)
    (a, sa), (b, sb) = _operand(m, k, g), _operand(n, k, g)
    for dtype, resid, shift in (("fp32", True, 1), ("bf16", True, 3), ("fp32", False, 0), ("bf16", False, 1)):
        bias = torch.randn(n, generator=g).cuda() if shift else None
        ld = n + 2 * shift + 1
        held = torch.full((shift + m * ld,), 5.0, dtype=DT[dtype], device="cuda")
        out = held.as_strided((m, n), (ld, 1), shift)
        res = torch.randn((m, n), generator=g).to(DT[dtype]).cuda() if resid else None
        want = _expected(a, sa, b, sb, bias, res, dtype)
        if resid:
            out.copy_(res)
        E.op_i8_gemm(a, sa, b, sb, out, bias=bias, residual=out if resid else None)
        assert _same(out, want), f"{dtype} {resid}"
        assert (held[:shift] == 5).all() and (held[shift:].view(m, ld)[:, n:] == 5).all()
        if resid:   # of another stride
            other = torch.empty((m, n), dtype=DT[dtype], device="cuda")
            E.op_i8_gemm(a, sa, b, sb, other, bias=bias, residual=res)
            assert _same(other, want)


@gpu
@pytest.mark.parametrize("dtype,m,n,ld", [("fp32", 8300, 4100, 4128), ("bf16", 16500, 4099, 4160), ("bf16", 16640, 4352, 4352)])
def test_results_past_the_cache(dtype, m, n, ld):
    """128 MB and more in whole cache lines, with tiles at the edges; then read by the next call."""
    g = torch.Generator().manual_seed(n)
    (a, sa), (b, sb) = _operand(m, 272, g), _operand(n, 272, g)
    held = torch.full((m, ld), 5.0, dtype=DT[dtype], device="cuda")
    want = _expected(a, sa, b, sb, None, None, dtype)
    E.op_i8_gemm(a, sa, b, sb, held[:, :n])
    assert _same(held[:, :n], want) and (held[:, n:] == 5).all()
    codes, scales = E.i8_alloc(m, n)
    E.op_i8_gemm(a, sa, b, sb, held[:, :n], bias=sb)
    E.op_i8_quant(held[:, :n], codes, scales)
    y = _expected(a, sa, b, sb, sb, None, dtype).double()
    assert torch.equal(scales, (y.abs().amax(1) / 127).float().clamp_min(LEAST))
    assert torch.equal(codes[:, :n].double(), torch.round(y / scales.double()[:, None]))


ROUNDS = [(8300, 4099), (9216, 4096), (12544, 4090), (5476, 8192), (16900, 2049), (9216, 8192)]


@gpu
@pytest.mark.parametrize("m,n,k", [(m, n, k) for m, n in ROUNDS for k in (112, 240, 272, 400, 1040) if n > 2049 or k > 112])
def test_rounds_of_large_products(m, n, k):
    """Workgroups with two and three large tiles one after the other, inner ones before inner ones and before the
    last rows' and columns', of one, two, three, four and nine K tiles; results that stay in the caches and, of
    9216 x 8192, that are stored past them; rows of any alignment; the residual in place and apart.  The next tile's loads are in flight behind the results of the one before."""
    assert E.i8_gemm_plan(m, n, k)["kernel"] == "large" and -(-m // 256) * -(-n // 256) >= 512
    g = torch.Generator().manual_seed(m + k)
    (a, sa), (b, sb) = _operand(m, k, g), _operand(n, k, g, k + 16)
    vec, large = torch.randn(n, generator=g).cuda(), torch.Generator("cuda").manual_seed(k)
    for i, (dtype, resid, shift) in enumerate((d, r, s) for d in ("fp32", "bf16") for r in (None, "apart", "in place")
                                              for s in (0, 1)):
        bias = vec if i % 3 == 0 else None
        res = torch.randn((m, n), generator=large, device="cuda").to(DT[dtype]) if resid else None
        # shift: rows that start off an aligned element, so that no result goes past the caches
        held = torch.full((shift + m * (n + shift) + 8,), 5.0, dtype=DT[dtype], device="cuda")
        out = held.as_strided((m, n), (n + shift, 1), shift)
        want = _expected(a, sa, b, sb, bias, res, dtype)
        if resid == "in place":
            out.copy_(res)
            res = out
        E.op_i8_gemm(a, sa, b, sb, out, bias=bias, residual=res)
        assert _same(out, want), f"{dtype} {resid} {shift}"
        assert (held[:shift] == 5).all() and (held[shift + m * (n + shift):] == 5).all()
        if shift:
            assert (held[1:1 + m * (n + 1)].view(m, n + 1)[:, n:] == 5).all()


@gpu
@pytest.mark.parametrize("far", ["a", "b"])
def test_rows_far_apart_on_large_tiles(far):
    """256 rows of a tile, 8 MB apart, of either operand: offsets in a tile up to 2139091072, just below 2^31, and tiles
    4 GB apart."""
    g = torch.Generator().manual_seed(3)
    ld, k, few, many = (1 << 23) - 16, 240, 768, 65536
    held = torch.zeros(ld * (few - 1) + k, dtype=torch.int8, device="cuda")
    spread = held.as_strided((few, k), (ld, 1))
    spread.copy_(torch.randint(-128, 128, (few, k), generator=g, dtype=torch.int8))
    a, b = (spread, _operand(many, k, g)[0]) if far == "a" else (_operand(many, k, g)[0], spread)
    m, n = len(a), len(b)
    plan = E.i8_gemm_plan(m, n, k)
    assert plan["kernel"] == "large" and plan["cut"] == 1
    sa, sb = torch.rand(m, generator=g).cuda(), torch.rand(n, generator=g).cuda()
    out = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    E.op_i8_gemm(a, sa, b, sb, out)
    assert torch.equal(out, _expected(a, sa, b, sb, None, None, "bf16"))


@gpu
def test_rows_far_apart():
    """Rows of operands 8 MB apart: offsets in a tile that pass 31 bits."""
    g = torch.Generator().manual_seed(2)
    ld, k = (1 << 23) - 16, 256
    held = torch.zeros(ld * 299 + k, dtype=torch.int8, device="cuda")
    far = held.as_strided((300, k), (ld, 1))
    far.copy_(torch.randint(-128, 128, (300, k), generator=g, dtype=torch.int8))
    for m, n in ((300, 300), (300, 8192), (8, 300), (2048, 300)):
        a, b = (far if m == 300 else _operand(m, k, g)[0]), (far if n == 300 else _operand(n, k, g)[0])
        sa, sb = torch.ones(m, device="cuda"), torch.ones(n, device="cuda")
        out = torch.empty((m, n), device="cuda")
        E.op_i8_gemm(a, sa, b, sb, out)
        assert torch.equal(out, _sums(a, b).float())
    wide = held.as_strided((256, k), (ld, 1))
    a, sa = _operand(16384, k, g)
    out = torch.empty((16384, 256), device="cuda")
    E.op_i8_gemm(a, sa, wide, torch.ones(256, device="cuda"), out)
    assert torch.equal(out, _expected(a, sa, wide, torch.ones(256, device="cuda"), None, None, "fp32"))


@gpu
def test_sums_at_the_end_of_the_range():
    """-128 times -128 at the longest K: 2^31 - 2^18, exactly; and the most negative sum."""
    k = 131056
    a = torch.full((2, k), -128, dtype=torch.int8, device="cuda")
    b = torch.full((40, k), -128, dtype=torch.int8, device="cuda")
    b[7] = 127
    one = torch.ones(40, device="cuda")
    out = torch.empty((2, 40), device="cuda")
    E.op_i8_gemm(a, one[:2], b, one, out)
    want = torch.full((40,), float(128 * 128 * k), dtype=torch.float64)
    want[7] = -128.0 * 127 * k
    assert (out.cpu().double() == want.float().double()).all()


@gpu
@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (8, 4096, 11008), (64, 1024, 2048), (591, 1003, 1296), (2304, 2048, 1024)])
def test_rows_do_not_depend_on_the_call(m, n, k):
    """A row's outputs are the same in a call of its own, on a few compute units, and on another stream."""
    g = torch.Generator().manual_seed(k)
    a, sa = _operand(m, k, g)
    b, sb = _operand(n, k, g)
    out = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    E.op_i8_gemm(a, sa, b, sb, out)
    i = m // 2
    one = torch.empty((1, n), dtype=torch.bfloat16, device="cuda")
    E.op_i8_gemm(a[i:i + 1], sa[i:i + 1], b, sb, one)
    assert torch.equal(one[0], out[i])
    again = torch.empty_like(out)
    work = E.i8_gemm_workspace(a, b)
    torch.cuda.synchronize()
    s = E.create_cu_masked_stream(0, [0xFFFF] + [0] * 7)
    try:
        E.op_i8_gemm(a, sa, b, sb, again, workspace=work, stream=s)
        torch.cuda.synchronize()
    finally:
        E.destroy_stream(s)
    assert torch.equal(again, out)
    side = torch.cuda.Stream()
    again.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        E.op_i8_gemm(a, sa, b, sb, again, workspace=work)
    side.synchronize()
    assert torch.equal(again, out)


@gpu
@pytest.mark.parametrize("m", [1, 37, 600])
def test_captured_linear_is_replayed(m):
    """Quantised rows and their product in a graph, replayed on new inputs beside eager calls."""
    g = torch.Generator().manual_seed(m)
    k, n = 1024, 1000
    x = torch.randn((m, k), generator=g).cuda()
    b, sb = _operand(n, k, g)
    a, sa = E.i8_alloc(m, k)
    out = torch.empty((m, n), device="cuda")
    work = E.i8_gemm_workspace(a, b)

    def step(to, codes, scales, w):
        E.op_i8_quant(x, codes, scales, norm_eps=1e-6)
        E.op_i8_gemm(codes, scales, b, sb, to, workspace=w)
    step(out, a, sa, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, a, sa, work)
    other, (a2, sa2) = torch.empty_like(out), E.i8_alloc(m, k)
    for i in range(4):
        x.copy_(torch.randn((m, k), generator=g))
        step(other, a2, sa2, None)
        if i == 2:
            torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other) and torch.equal(a, a2)


@gpu
def test_quantised_linear_layer():
    """Weights and rows by op_i8_quant: within the steps' bound of the layer in 64 bits.  Each code is off by
    half a step of its row's scale, so an output by at most sum (|a| sb + |b| sa + sa sb / 2) / 2, and its own
    rounding."""
    g = torch.Generator().manual_seed(5)
    m, n, k = 50, 200, 1000
    x, w = torch.randn((m, k), generator=g).cuda(), torch.randn((n, k), generator=g).cuda()
    a, sa = E.i8_alloc(m, k)
    b, sb = E.i8_alloc(n, k)
    E.op_i8_quant(x, a, sa)
    E.op_i8_quant(w, b, sb)
    out = torch.empty((m, n), device="cuda")
    E.op_i8_gemm(a, sa, b, sb, out)
    xd, wd, s, t = x.double(), w.double(), sa.double()[:, None], sb.double()[None]
    bound = (xd.abs().sum(1)[:, None] * t + wd.abs().sum(1)[None] * s + k * s * t / 2) / 2
    want = xd @ wd.t()
    assert ((out.double() - want).abs() <= bound + want.abs() * 2.0 ** -21 + bound * 2.0 ** -21).all()
