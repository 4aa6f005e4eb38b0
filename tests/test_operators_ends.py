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
