"""Refusals of the 8-bit linear layer's operators, on the CPU: every bad argument is
turned down before a device is touched."""
import ctypes
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20818_amd as prm  # noqa: E402

FAKE = 1 << 20  # never dereferenced: the arguments are refused first
BF = prm.BF16


def refused(name, args, code, word=""):
    L = prm.load()
    rc = getattr(L, name)(*args)
    assert rc == code, (name, rc)
    assert word in L.prm_last_error().decode(), L.prm_last_error()


def changed(base, **kw):
    out = dict(base)
    out.update(kw)
    return list(out.values())


Q = dict(x=FAKE, dtype=BF, rows=4, cols=8, ldx=8, q=FAKE, ldq=8, scale=FAKE, stream=None)
C = dict(x=FAKE, dtype=BF, rows=2000, cols=8, ldx=8, q=FAKE, ldq=2000, scale=FAKE, sum=None, ws=FAKE, nws=1 << 16, stream=None)
M = dict(a=FAKE, lda=8, sa=FAKE, b=FAKE, ldb=8, sb=FAKE, bias=None, dtype=BF, out=FAKE, ldo=6, m=4, n=6, k=8, ws=None, nws=0, stream=None)
N = dict(x=FAKE, ldx=8, res=None, ldres=0, w=FAKE, dtype=BF, rows=4, cols=8, eps=1e-6, h=None, ldh=0, y=FAKE, ldy=8, q=None,
         ldq=0, scale=None, stream=None)
G = dict(gy=FAKE, ldgy=8, gh=None, ldgh=0, h=FAKE, ldh=8, w=FAKE, dtype=BF, rows=4, cols=8, eps=1e-6, dx=FAKE, lddx=8,
         dw=FAKE, ws=FAKE, nws=1 << 16, stream=None)
F = dict(x=FAKE, ldx=8, w=FAKE, ldw=8, bias=None, dtype=BF, y=FAKE, ldy=6, m=4, n=6, k=8, ws=FAKE, nws=1 << 20, stream=None)
B = dict(gy=FAKE, ldgy=6, x=FAKE, ldx=8, w=FAKE, ldw=8, dtype=BF, dx=FAKE, lddx=8, dw=FAKE, lddw=8, db=FAKE, m=4, n=6, k=8, ws=FAKE,
         nws=1 << 20, stream=None)
BASE = {"prm_int8_linear": F, "prm_int8_linear_backward": B, "prm_quantize_rows": Q, "prm_quantize_cols": C, "prm_int8_matmul": M, "prm_rms_norm": N, "prm_rms_norm_backward": G}


@pytest.mark.parametrize("name", sorted(BASE))
def test_unknown_type(name):
    for t in (3, -1):
        refused(name, changed(BASE[name], dtype=t), prm.PRM_EDTYPE, "dtype")


@pytest.mark.parametrize("name,kw", [
    ("prm_quantize_rows", dict(rows=-1)), ("prm_quantize_rows", dict(cols=0)), ("prm_quantize_rows", dict(cols=(1 << 24) + 1)),
    ("prm_quantize_rows", dict(rows=1 << 31)), ("prm_quantize_rows", dict(ldx=7)), ("prm_quantize_rows", dict(ldq=7)),
    ("prm_quantize_rows", dict(x=None)), ("prm_quantize_rows", dict(q=None)), ("prm_quantize_rows", dict(scale=None)),
    ("prm_quantize_cols", dict(rows=0)), ("prm_quantize_cols", dict(rows=(1 << 22) + 1, ldq=1 << 30)),
    ("prm_quantize_cols", dict(ldq=1999)), ("prm_quantize_cols", dict(ldx=7)), ("prm_quantize_cols", dict(nws=8)),
    ("prm_quantize_cols", dict(ws=None)), ("prm_quantize_cols", dict(x=None)),
    ("prm_int8_matmul", dict(k=0)), ("prm_int8_matmul", dict(k=(1 << 20) + 1, lda=1 << 21, ldb=1 << 21)),
    ("prm_int8_matmul", dict(k=131072, lda=131073, ldb=131072)),
    ("prm_int8_matmul", dict(k=131072, lda=131072, ldb=131072)),
    ("prm_int8_matmul", dict(k=131072, lda=131072, ldb=131072, ws=FAKE, nws=255)),
    ("prm_int8_matmul", dict(m=-1)), ("prm_int8_matmul", dict(n=(1 << 24) + 1, ldo=1 << 30)),
    ("prm_int8_matmul", dict(lda=7)), ("prm_int8_matmul", dict(ldb=7)), ("prm_int8_matmul", dict(ldo=5)),
    ("prm_int8_matmul", dict(a=None)), ("prm_int8_matmul", dict(sb=None)), ("prm_int8_matmul", dict(out=None)),
    ("prm_rms_norm", dict(eps=0.0)), ("prm_rms_norm", dict(eps=float("nan"))), ("prm_rms_norm", dict(eps=float("inf"))),
    ("prm_rms_norm", dict(res=FAKE, ldres=8)), ("prm_rms_norm", dict(h=FAKE, ldh=8)),
    ("prm_rms_norm", dict(res=FAKE, ldres=7, h=FAKE, ldh=8)), ("prm_rms_norm", dict(res=FAKE, ldres=8, h=FAKE, ldh=7)),
    ("prm_rms_norm", dict(y=None)), ("prm_rms_norm", dict(q=FAKE, ldq=8)), ("prm_rms_norm", dict(y=None, q=FAKE, ldq=8)),
    ("prm_rms_norm", dict(y=None, q=FAKE, ldq=7, scale=FAKE)), ("prm_rms_norm", dict(ldy=7)), ("prm_rms_norm", dict(cols=0)),
    ("prm_rms_norm", dict(x=None)),
    ("prm_int8_linear", dict(m=-1)), ("prm_int8_linear", dict(n=0)), ("prm_int8_linear", dict(k=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21)),
    ("prm_int8_linear", dict(m=(1 << 20) + 1)), ("prm_int8_linear", dict(ldx=7)), ("prm_int8_linear", dict(ldw=7)), ("prm_int8_linear", dict(ldy=5)),
    ("prm_int8_linear", dict(nws=64)), ("prm_int8_linear", dict(ws=None)), ("prm_int8_linear", dict(w=None)),
    ("prm_int8_linear_backward", dict(m=0)), ("prm_int8_linear_backward", dict(n=(1 << 20) + 1, ldgy=1 << 21)),
    ("prm_int8_linear_backward", dict(ldgy=5)), ("prm_int8_linear_backward", dict(ldx=7)), ("prm_int8_linear_backward", dict(ldw=7)),
    ("prm_int8_linear_backward", dict(lddx=7)), ("prm_int8_linear_backward", dict(lddw=7)), ("prm_int8_linear_backward", dict(nws=64)),
    ("prm_int8_linear_backward", dict(x=None)), ("prm_int8_linear_backward", dict(w=None)), ("prm_int8_linear_backward", dict(gy=None)),
    ("prm_quantize_cols", dict(rows=1 << 22, cols=1 << 16, ldx=1 << 16, ldq=1 << 22, nws=1 << 40)),
    ("prm_rms_norm_backward", dict(eps=-1.0)), ("prm_rms_norm_backward", dict(ldgy=7)),
    ("prm_rms_norm_backward", dict(gh=FAKE, ldgh=7)), ("prm_rms_norm_backward", dict(ldh=7)),
    ("prm_rms_norm_backward", dict(lddx=7)), ("prm_rms_norm_backward", dict(nws=4)),
    ("prm_rms_norm_backward", dict(ws=None)), ("prm_rms_norm_backward", dict(dx=None)),
])
def test_bad_argument(name, kw):
    refused(name, changed(BASE[name], **kw), prm.PRM_EINVAL)


@pytest.mark.parametrize("name,kw", [
    ("prm_quantize_rows", dict(x=FAKE + 1)), ("prm_quantize_rows", dict(scale=FAKE + 2)),
    ("prm_quantize_rows", dict(x=FAKE + 2, dtype=prm.F32)), ("prm_quantize_cols", dict(ws=FAKE + 8)),
    ("prm_int8_matmul", dict(out=FAKE + 1)), ("prm_int8_matmul", dict(sa=FAKE + 2)), ("prm_int8_matmul", dict(bias=FAKE + 1)),
    ("prm_rms_norm", dict(w=FAKE + 1)), ("prm_rms_norm_backward", dict(gy=FAKE + 1)),
])
def test_off_an_elements_boundary(name, kw):
    refused(name, changed(BASE[name], **kw), prm.PRM_EALIGN, "aligned")


def test_nothing_to_do():
    L = prm.load()
    assert L.prm_quantize_rows(*changed(Q, rows=0, x=None, q=None, scale=None)) == prm.PRM_OK
    assert L.prm_int8_matmul(*changed(M, m=0)) == prm.PRM_OK
    assert L.prm_int8_matmul(*changed(M, n=0)) == prm.PRM_OK
    assert L.prm_rms_norm(*changed(N, rows=0)) == prm.PRM_OK
    assert L.prm_rms_norm_backward(*changed(G, rows=0, dw=None)) == prm.PRM_OK
    assert L.prm_int8_linear(*changed(F, m=0, x=None, ws=None)) == prm.PRM_OK
    assert L.prm_int8_linear_backward(*changed(B, dx=None, dw=None, db=None, ws=None)) == prm.PRM_OK


def test_workspace_sizes():
    L = prm.load()
    for f in (L.prm_quantize_cols_workspace, L.prm_rms_norm_backward_workspace):
        assert f(0, 8) == 0 and f(8, 0) == 0 and f(8, (1 << 24) + 1) == 0
        assert f(1, 1) > 0 and f(8192, 4096) >= 4 * 4096
        assert f(8192, 4096) % 4 == 0
    assert L.prm_quantize_cols_workspace((1 << 22) + 1, 8) == 0
    w = L.prm_int8_matmul_workspace
    assert w(FAKE, 4096, FAKE, 4096, 4096, 4096, 4096) == 0  # one piece, rows as they are
    assert w(FAKE, 16000, FAKE, 16000, 40, 200, 16000) >= 2 * 40 * 200 * 4  # split
    # one operand laid out anew, the other, both
    assert w(FAKE, 4097, FAKE, 4096, 4096, 8192, 4096) == 4096 * 4096 and w(FAKE, 4096, FAKE + 8, 4096, 4096, 8192, 4096) == 8192 * 4096
    assert w(FAKE, 4097, FAKE, 4097, 4096, 8192, 4097) == 3 * 4096 * 4224
    assert w(FAKE, 4096, FAKE, 4096, 0, 8, 4096) == 0 and w(FAKE, 8, FAKE, 16, 8, 8, 16) == 0
    for f in (L.prm_int8_linear_workspace, L.prm_int8_linear_backward_workspace):
        assert f(0, 8, 8) == f(8, 0, 8) == f(8, 8, 0) == f((1 << 20) + 1, 8, 8) == 0
        assert f(100, 60, 30) >= 100 * 30 + 60 * 30


def test_16_bit_values_round_right_without_a_check():
    """The quantiser's claim for values of a 16-bit type: rint of u inv, the product unrounded
    (an fma), with inv = 127 / top rounded up, is the nearest whole number of 127 u / top,
    ties to even, for every value u = U 2^-j and top = T whose whole T 127 does not divide."""
    from fractions import Fraction

    import numpy as np
    for bits in (8, 11):  # bf16, fp16: whole numbers of that many bits
        for T in range(1 << (bits - 1), 1 << bits):
            inv = np.float32(127) / np.float32(T)
            if Fraction(float(inv)) * T < 127:
                inv = np.nextafter(inv, np.float32(np.inf))
            if T % 127 == 0:
                continue
            for j in range(9):
                U = np.arange(1 << (bits - 1), min(T << j, (1 << bits) - 1) + 1, dtype=np.int64)
                n = np.rint(U * float(inv) / (1 << j)).astype(np.int64)  # 11 + 24 bits: exact in fp64
                num, den = 254 * U, 2 * (T << j)
                k = num // den
                rest = 2 * (num - k * den)
                assert np.array_equal(n, k + ((rest > den) | ((rest == den) & (k % 2 == 1)))), (bits, T, j)


def test_direct_loads_leave_m0_to_the_compiler(tmp_path):
    # the products' loads into shared memory write M0 in inline assembly, a register that the
    # compiler reserves: sound while it reads M0 nowhere itself
    import subprocess

    from paper_2608_20818_amd import build as b
    from test_abi import _m0_check
    out = tmp_path / "ops.s"
    r = subprocess.run([b.hipcc(), *[f for f in b.FLAGS if f != "-fPIC"], "--cuda-device-only", "-S", os.path.join(b.CSRC, "ops_matmul.hip"),
                        "-o", str(out)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    readers, asm_dma, bad = _m0_check(out.read_text())
    assert asm_dma > 0 and readers == 0 and not bad


def test_the_step_takes_no_fp16():
    with pytest.raises(prm.PRMError) as e:
        prm.plan_workspace_bytes([(4, 8)], prm.config_default(param_dtype=prm.F16))
    assert e.value.code == prm.PRM_EDTYPE


def test_host_tensors_are_refused():
    x, w = torch.zeros(3, 8), torch.zeros(5, 8)
    q, s = torch.zeros(3, 8, dtype=torch.int8), torch.zeros(3)
    for call in (lambda: prm.quantize_rows(x), lambda: prm.quantize_rows(x, transpose=True), lambda: prm.rms_norm(x),
                 lambda: prm.int8_linear(x, w), lambda: prm.int8_matmul(q, s, q, s)):
        with pytest.raises(ValueError, match="device tensor"):
            call()


def test_names_are_public():
    for n in ("quantize_rows", "int8_matmul", "int8_linear", "rms_norm"):
        assert n in prm.__all__ and callable(getattr(prm, n))
    assert ctypes.sizeof(ctypes.c_int32) == 4


@pytest.mark.parametrize("h,w", [((3, 7), (8,)), ((2, 8), (8,)), ((3, 8), (7,)), ((3, 8), None)], ids=str)
def test_saved_norm_inputs_are_checked(h, w):
    # what hooks bring back reaches the gradient's kernel only in the shape and type saved
    from types import SimpleNamespace

    from paper_2608_20818_amd import operators
    t = torch.float16 if w is None else torch.float32
    ctx = SimpleNamespace(saved_tensors=(torch.zeros(h, dtype=t), torch.zeros(w) if w else None), needs_input_grad=(True, w is not None, False, False),
                          eps=1e-6)
    with pytest.raises(ValueError, match="saved (input|weight)"):
        operators._RmsNorm.backward(ctx, torch.zeros(3, 8))
