"""The 8-bit linear layer's operators on the CPU: what is refused, before a device is touched, so
that nothing is lost without a word."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_20818_amd as prm  # noqa: E402

X, W, Q, S = torch.zeros(3, 8), torch.zeros(5, 8), torch.zeros(3, 8, dtype=torch.int8), torch.zeros(3)
CALLS = {"rms_norm": lambda x: prm.rms_norm(x), "residual": lambda x: prm.rms_norm(X, residual=x), "weight": lambda x: prm.rms_norm(X, x[0]),
         "eight bits": lambda x: prm.rms_norm(x, quantize=True)[1], "linear": lambda x: prm.int8_linear(x, W), "bias": lambda x: prm.int8_linear(X, X, x[:, 0])}
UNSEEN = {"rows": lambda x: prm.quantize_rows(x)[1], "columns": lambda x: prm.quantize_rows(x, transpose=True)[1],
          "product": lambda x: prm.int8_matmul(Q, S, Q, S, bias=x[:, 0], dtype=torch.float32)}


@pytest.mark.parametrize("call", sorted(CALLS))
def test_forward_mode_is_refused(call):
    import torch.autograd.forward_ad as fw
    with fw.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            CALLS[call](fw.make_dual(X, torch.ones_like(X)))
    with pytest.raises(RuntimeError, match="forward-mode"):
        torch.func.jvp(CALLS[call], (X,), (torch.ones_like(X),))


@pytest.mark.parametrize("call", sorted(CALLS) + sorted(UNSEEN))
def test_traces_are_refused(call):
    from torch.fx.experimental.proxy_tensor import make_fx
    f = {**CALLS, **UNSEEN}[call]
    with pytest.raises(RuntimeError, match="trace"):
        torch.jit.trace(f, (X,), check_trace=False)
    for mode in ("real", "fake"):
        with pytest.raises(RuntimeError, match="trace"):
            make_fx(f, tracing_mode=mode)(X)


@pytest.mark.parametrize("gone", ["torch", "library"])
def test_import_star_needs_neither_torch_nor_the_library(gone):
    # the step's names need neither; the operators say what they miss when they are called
    import subprocess
    hide = 'sys.modules["torch"] = None' if gone == "torch" else 'import paper_2608_20818_amd as p; p.LIB_PATH = "/nonexistent/libprm.so"'
    code = f"""import sys
{hide}
from paper_2608_20818_amd import *
assert Config and AdamWConfig and F32 == 0 and rms_norm.__name__ == "rms_norm"
try:
    int8_linear(None, None)
except {"ImportError" if gone == "torch" else "PRMError"} as e:
    print("said:", e)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and ("torch" if gone == "torch" else "libprm") in r.stdout.split("said:")[1], r.stderr


FAKE = 1 << 20  # never dereferenced: the arguments are refused first


def test_a_products_limits_are_its_kernels():
    # rows on any byte, 2^18 x 64 tiles of 64: past a grid's 2^24, so another kernel's, which lays both
    # operands out anew
    import ctypes
    L = prm.load()
    m, n, k = 1 << 24, 4096, 100
    assert L.prm_int8_matmul_workspace(FAKE, k, FAKE, k, m, n, k) == (m + n) * 128
    # each kernel refuses a grid too large for its own tiles before it looks at a pointer
    P, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    f = L.prm_internal_int8_matmul
    f.argtypes = [P, i64, P, P, i64, P, P, i32, P, i64, i64, i64, i64, P, ctypes.c_uint64, P, i32, i32, i32]

    def refused(m, n, k, kind, splits=1, pack=0, ld=1 << 20):
        rc = f(FAKE, ld, FAKE, FAKE, ld, FAKE, None, prm.F32, FAKE, n, m, n, k, FAKE, 1 << 62, None, kind, splits, pack)
        assert rc in (prm.PRM_EINVAL, prm.PRM_EHIP)  # here or at the pointers: no memory of a device, or no device
        return "does not take" in L.prm_last_error().decode()

    for kind, tile in ((2, 64), (3, 128), (4, 64), (5, 128), (6, 128), (7, 256)):
        rows = min(1 << 24, (1 << 12) * tile)
        cols = (1 << 24) // (rows // tile) * tile
        assert refused(rows, cols, 128, kind) and not refused(rows, cols - tile, 128, kind)
    assert refused(1 << 18, 1 << 17, 256, 4, 2) and not refused(1 << 18, (1 << 17) - 8, 256, 4, 2)  # the sums joined
    assert refused(1 << 22, 64, 1 << 14, 4, 1, 1) and not refused((1 << 22) - 1, 64, 1 << 14, 4, 1, 1)  # the operand laid out anew
    # with no kernel left: said so, and not of the workspace
    assert L.prm_int8_matmul(FAKE, 128, FAKE, FAKE, 128, FAKE, None, prm.F32, FAKE, 1 << 24, 1 << 24, 1 << 24, 128, None, 0, None) == prm.PRM_EINVAL
    assert "too large" in L.prm_last_error().decode()
    assert L.prm_int8_matmul_workspace(FAKE, 128, FAKE, 128, 1 << 24, 1 << 24, 128) == 0


def test_a_layers_limits_come_before_its_first_launch():
    L, big = prm.load(), 1 << 20
    room = 1 << 62
    rc = L.prm_int8_linear(FAKE, big, FAKE, big, None, prm.BF16, FAKE, big, big, big, 16, FAKE, room, None)
    assert rc == prm.PRM_EINVAL and "too large" in L.prm_last_error().decode()
    # dx (m x k), dw (n x k), and the columns of gy and x in one launch
    for m, n, k, dx, dw, db in ((big, 16, big, FAKE, None, None), (16, big, big, None, FAKE, None), (big, big, 16, None, None, FAKE)):
        rc = L.prm_int8_linear_backward(FAKE, big, FAKE, big, FAKE, big, prm.BF16, dx, big, dw, big, db, m, n, k, FAKE, room, None)
        assert rc == prm.PRM_EINVAL and "too large" in L.prm_last_error().decode(), (m, n, k)
