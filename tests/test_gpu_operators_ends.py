"""The 8-bit linear layer's operators at the ends of their ranges, on the GPU, against plain
implementations in 64 bits on the CPU: magnitudes where fp32 ends, many rows and tokens, what
autograd and tensors' views may hand them.

Tolerances count roundings as in test_gpu_operators.py: u = 2^-24 for each of fp32 arithmetic,
half a step for the one to the output's type.  With S roundings of a row's sums, r of the norm
has S / 2 + 4.  In dx = r (g - n mean(g n)) the last term has r three times, the sum of g h once
(S + 3) and five more: 2.5 S + 20 u of r (|g| + |n| mean|g n|) + |gh|.
"""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20818_amd as prm  # noqa: E402
from paper_2608_20818_amd import operators  # noqa: E402
from test_gpu_operators import TYPES, NAMES, U, check, check_product, check_scale, eight, half, low, norm64, rand, sums  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    """Both ways a call can take: native code, and Python where that is not built."""
    if request.param == "python":
        monkeypatch.setattr(operators, "_native", type("none", (), {n: staticmethod(lambda *a: None) for n in (
            "quantize_rows", "quantize_cols", "int8_matmul", "int8_linear", "rms_norm")}))
    return request.param


# ---------------------------------------------------------------- magnitudes
def tall_rows(t):
    # largest values 254 2^n, a multiple of 127, up to the end of the range: every odd multiple of
    # 2^n is a border of two whole numbers there
    v = torch.tensor([254, -254, 150, 250, 253, -251, 127, 1, -3, 0, 129, 75], dtype=torch.float64)
    return torch.stack([v * s * 2.0 ** n for n in range(108, 121) for s in (1, -1)]).to(t)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32], ids=NAMES.get)
def test_quantize_rows_near_the_ranges_end(t):
    x = tall_rows(t)
    assert torch.isfinite(x).all()
    qe, se = eight(x.double())
    for q, s in (prm.quantize_rows(x.cuda()), prm.quantize_rows(x.t().contiguous().cuda(), transpose=True)):
        assert torch.equal(q.cpu().double(), qe)
        check_scale(s, se)
    # the layer's own quantiser of rows; one-hot weights give back the values that q stands for, of
    # which a scale has 2 u and the product 4
    w = torch.eye(12, dtype=t)
    y = prm.int8_linear(x.cuda(), w.cuda()).double().cpu()
    want = qe * se[:, None]
    ok = (want * 127).abs() < 3.4e38  # the sum times the first scale, before the weight's 1 / 127, in fp32's range
    assert ok.any() and ((y - want).abs() <= 8 * U * want.abs() + half(t) * want.abs() * (1 + 1e-3))[ok].all()


def test_norm_eight_bits_of_large_products():
    # h w past 2^120 in fp32, on borders of two whole numbers; the squares of h stay in its range
    v = torch.tensor([254, 253, -251, 127, 1, -3, 0, 129, 75, -254, 249, 5], dtype=torch.float64)
    x, w = (torch.stack([v * 2.0 ** 52, v.flip(0) * 2.0 ** 50])).to(torch.bfloat16), torch.full((12,), 2.0 ** 63, dtype=torch.bfloat16)
    q, s = prm.rms_norm(x.cuda(), w.cuda(), quantize=True)
    _, r, _ = norm64(x, None, w, 1e-6, torch.bfloat16)
    qe, se = eight(x.double() * w.double())
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se * r[:, 0], (sums(12) / 2 + 6) * U)


WIDE = [(1, 40), (3, 513), (5, 1001), (600, 2050), (2, 4100), (2, 12289), (2, 33000)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32], ids=NAMES.get)
@pytest.mark.parametrize("shape", WIDE, ids=str)
def test_norm_past_the_range_of_squares(shape, t):
    # rows whose squares leave fp32's range beside ordinary ones, plain and in 8 bits, with products
    # h w that leave it at either end too
    x, res = rand(shape, t, 1), rand(shape, t, 2)
    up = torch.tensor([2.0 ** e for e in (125, 0, 70, 100, 120, 63)], dtype=torch.float64)
    by = up[torch.arange(shape[0]) % 6][:, None]
    x, res = (x.double() * by).to(t), (res.double() * by).to(t)
    for scale in (1.0, 2.0 ** 60, 2.0 ** -120):
        w = rand(shape[1:], t, 3, scale)
        for rs in (None, res):
            h, r, y = norm64(x, rs, w, 1e-6, t)
            got = prm.rms_norm(x.cuda(), w.cuda(), None if rs is None else rs.cuda())
            got8 = prm.rms_norm(x.cuda(), w.cuda(), None if rs is None else rs.cuda(), quantize=True)
            if rs is not None:
                assert torch.equal(got[1], got8[2])
                h, r, y = norm64(got[1].cpu(), None, w, 1e-6, t)
                got = got[0]
            check(got, y, ((sums(shape[1]) / 2 + 6) * U + half(t)) * y.abs() * (1 + half(t)) + low(t))
            qe, se = eight(h * w.double())
            assert torch.equal(got8[0].cpu().double(), qe)
            check_scale(got8[1], se * r[:, 0], (sums(shape[1]) / 2 + 6) * U)


def test_norm_eight_bits_of_small_products():
    # h w below fp32's normal range: q is decided on the exact products all the same
    t = torch.bfloat16
    x, w = rand((4, 300), t, 4), rand((300,), t, 5, 2.0 ** -60)
    x = (x.double() * torch.tensor([2.0 ** -60, 2.0 ** -70, 2.0 ** -80, 1.0], dtype=torch.float64)[:, None]).to(t)
    q, s = prm.rms_norm(x.cuda(), w.cuda(), eps=1e-30, quantize=True)
    qe, se = eight(x.double() * w.double())
    r = 1 / torch.sqrt(x.double().square().mean(1) + float(torch.tensor(1e-30)))
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se * r, (sums(300) / 2 + 6) * U)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32], ids=NAMES.get)
def test_norm_of_rows_that_are_not_finite_beside_large_ones(t):
    x, w = rand((6, 700), t, 6), rand((700,), t, 7)
    x[0] *= 2.0 ** 80
    x[1] *= 2.0 ** 80
    x[1, 5] = float("nan")
    x[2] *= 2.0 ** 80
    x[2, 699] = float("-inf")
    x[3] = 0
    x[4, 7] = 2.0 ** 120
    y, (q, s) = prm.rms_norm(x.cuda(), w.cuda()).cpu(), (v.cpu() for v in prm.rms_norm(x.cuda(), w.cuda(), quantize=True))
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 699]) and (y[2, :699] == 0).all() and (y[3] == 0).all()
    assert torch.isnan(s[1:3]).all() and (q[1:4] == 0).all() and s[3] == 0
    rows = [0, 4, 5]
    _, r, want = norm64(x[rows], None, w, 1e-6, t)
    check(y[rows], want, ((sums(700) / 2 + 6) * U + half(t)) * want.abs() * (1 + half(t)) + low(t))
    qe, se = eight(x[rows].double() * w.double())
    assert torch.equal(q[rows].double(), qe)
    check_scale(s[rows], se * r[:, 0], (sums(700) / 2 + 6) * U)


def additions(rows, cols, t):
    # of dw, by the kernel's rule: a thread's rows one after the other, the four waves of a block of
    # short rows, each 32nd of the blocks' sums, and 32 of those
    groups = -(-rows // 4) if cols <= 512 else rows
    most = 256 if cols > 4096 else 512 if cols > 2048 and t == torch.float32 else 1024
    blocks = min(groups, most)
    return -(-groups // blocks) + 4 + -(-blocks // 32) + 32


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32], ids=NAMES.get)
@pytest.mark.parametrize("shape", WIDE, ids=str)
def test_norm_gradients_past_the_range_of_squares(shape, t):
    # the rows as above; gradients of about the norm's own size, so that r g stays a normal number.
    # A value below 2^-46 of a row scaled by 2^-80 may round in fp32's lowest range, by 2^-150, in n
    # times r 2^80, where r is at most 2^-52 (2^24 squares past 2^128): below 2^-122
    x = rand(shape, t, 8)
    up = torch.tensor([2.0 ** e for e in (125, 0, 70, 100, 120, 63)], dtype=torch.float64)
    by = up[torch.arange(shape[0]) % 6][:, None]
    x, w, gy, gh = (x.double() * by).to(t), rand(shape[1:], t, 9), rand(shape, t, 10), rand(shape, t, 11)
    for kept in (False, True):
        xg, wg, rg = x.cuda().requires_grad_(), w.cuda().requires_grad_(), torch.zeros_like(x).cuda()
        if kept:
            got = torch.autograd.grad(prm.rms_norm(xg, wg, rg), (xg, wg), (gy.cuda(), gh.cuda()))
        else:
            got = torch.autograd.grad(prm.rms_norm(xg, wg), (xg, wg), gy.cuda())
        h = x.double()
        r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
        g, n = gy.double() * w.double(), h * r
        dx = r * (g - n * (g * n).mean(1, keepdim=True))
        size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
        if kept:
            dx, size = dx + gh.double(), size + gh.double().abs()
        s = sums(shape[1])
        check(got[0], dx, (2.5 * s + 20) * U * size + half(t) * dx.abs() * (1 + 1e-3) + low(t))
        dw, size = (gy.double() * n).sum(0), (gy.double() * n).abs().sum(0)
        check(got[1], dw, (s / 2 + 6 + additions(*shape, t)) * U * size + half(t) * dw.abs() * (1 + 1e-3) + low(t)
              + 2.0 ** -122 * gy.double().abs().sum(0))


@pytest.mark.parametrize("shape", [(7, 40), (1030, 2050), (300, 4100), (5, 33000)], ids=str)
def test_norm_gradients_past_the_range_of_g_h(shape):
    # squares in fp32's range, sums of g h not (and none of the share of dw twice); rows that are
    # not finite keep to themselves
    t, rows = torch.float32, shape[0]
    x, w, gy = rand(shape, t, 12), rand(shape[1:], t, 13), rand(shape, t, 14)
    x[1] *= 2.0 ** 55
    gy[1] *= 2.0 ** 90
    for bad in (None, float("inf"), float("nan")):
        xb, gb = x.clone(), gy.clone()
        if bad is not None:
            gb[rows - 2, 3], xb[rows - 3, 5] = bad, bad
        xg, wg = xb.cuda().requires_grad_(), w.cuda().requires_grad_()
        got = torch.autograd.grad(prm.rms_norm(xg, wg), (xg, wg), gb.cuda())
        h = x.double()
        r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
        g, n = gy.double() * w.double(), h * r
        dx = r * (g - n * (g * n).mean(1, keepdim=True))
        size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
        s = sums(shape[1])
        ok = torch.ones(rows, dtype=torch.bool)
        if bad is not None:
            ok[[rows - 2, rows - 3]] = False
            assert not torch.isfinite(got[0][rows - 2]).any() and torch.isnan(got[0][rows - 3, 5])
            assert not torch.isfinite(got[1][3]) and not torch.isfinite(got[1][5])
        else:
            size_w = (gy.double() * n).abs().sum(0)
            check(got[1], (gy.double() * n).sum(0), (s / 2 + 6 + additions(*shape, t)) * U * size_w + half(t) * size_w + low(t))
        check(got[0].cpu()[ok], dx[ok], ((2.5 * s + 20) * U * size + half(t) * dx.abs() * (1 + 1e-3) + low(t))[ok])


# ---------------------------------------------------------------- what autograd may hand over
def test_forward_mode_and_tracing_are_refused(path):
    # no tangent is dropped, and no trace records the outputs' allocation alone
    import torch.autograd.forward_ad as fw
    from torch.fx.experimental.proxy_tensor import make_fx
    x, w, nw = rand((4, 16), torch.float32, 20).cuda(), rand((8, 16), torch.float32, 21).cuda(), rand((16,), torch.float32, 22).cuda()
    q, s = prm.quantize_rows(x)
    calls = [lambda v: prm.rms_norm(v, nw), lambda v: prm.rms_norm(x, nw, residual=v), lambda v: prm.rms_norm(v, quantize=True)[1],
             lambda v: prm.int8_linear(v, w), lambda v: prm.int8_linear(w, v)]
    with fw.dual_level():
        d = fw.make_dual(x, torch.ones_like(x))
        for f in calls:
            with pytest.raises(RuntimeError, match="forward-mode"):
                f(d)
    for f in calls[:2] + calls[3:]:
        with pytest.raises(RuntimeError, match="forward-mode"):
            torch.func.jvp(f, (x,), (torch.ones_like(x),))
    for f in calls + [lambda v: prm.quantize_rows(v)[1], lambda v: prm.quantize_rows(v, transpose=True)[1],
                      lambda v: prm.int8_matmul(q, s, q, s, bias=v[:, 0], dtype=torch.float32)]:
        with pytest.raises(RuntimeError, match="trace"):
            torch.jit.trace(f, (x,), check_trace=False)
        with pytest.raises(RuntimeError, match="trace"):
            make_fx(f)(x)


def test_layer_of_more_tokens_than_a_sum_holds(path):
    # tokens are the sum of the weight's gradient alone: the output, the inputs' gradient and the
    # bias's take more than 2^20
    t, m, n, k = torch.bfloat16, (1 << 20) + 77, 8, 16
    x, w, b, gy = rand((m, k), t, 30).cuda(), rand((n, k), t, 31).cuda(), rand((n,), t, 32).cuda(), rand((m, n), t, 33).cuda()
    with torch.no_grad():
        y = prm.int8_linear(x, w, b)
    assert torch.equal(y[-100:], prm.int8_linear(x[-100:], w, b)) and torch.equal(y[:100], prm.int8_linear(x[:100], w, b))
    xg, bg, wg = (v.clone().requires_grad_() for v in (x, b, w))
    gx, gb = torch.autograd.grad(prm.int8_linear(xg, w, bg), (xg, bg), gy)
    assert torch.equal(gx[-100:], prm.int8_matmul(*prm.quantize_rows(gy[-100:]), *prm.quantize_rows(w, transpose=True), dtype=t))
    # at most 64 row blocks, rows 8 apart, then the blocks' sums
    g = gy.double().cpu()
    check(gb, g.sum(0), (m / 64 / 8 + 8 + 64) * U * g.abs().sum(0) + half(t) * g.sum(0).abs() * (1 + 1e-3) + low(t))
    with pytest.raises(RuntimeError, match="1048576"):
        torch.autograd.grad(prm.int8_linear(x, wg), wg, gy)


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_views_that_stand_for_the_negative(path, t):
    # contiguous views whose values are the memory's negated (what conj().imag gives of one column)
    x, r, nw, w, gy = (rand(s, t, 40 + i).cuda() for i, s in enumerate([(6, 24), (6, 24), (24,), (10, 24), (6, 10)]))
    n = torch._neg_view
    calls = [(lambda a, b, c: torch.cat(list(prm.rms_norm(a, c, b))), (x, r, nw)),
             (lambda a, b, c: torch.mul(*[v if v.dim() > 1 else v[:, None] for v in prm.rms_norm(a, c, b, quantize=True)[:2]]), (x, r, nw)),
             (lambda a: prm.quantize_rows(a)[0], (x,)), (lambda a: prm.quantize_rows(a, transpose=True)[0], (x,)),
             (lambda a, b, c: prm.int8_linear(a, b, c), (x, w, gy[0])),
             (lambda a, b, c: prm.int8_matmul(*prm.quantize_rows(x), *prm.quantize_rows(w), bias=c, dtype=t), (x, w, gy[0]))]
    for f, args in calls:
        assert torch.equal(f(*[n(a) for a in args]), f(*[-a for a in args]))
    xg, wg, ng = (v.clone().requires_grad_() for v in (x, w, nw))
    for f, to, g in ((lambda: prm.int8_linear(xg, wg), (xg, wg), gy), (lambda: prm.rms_norm(xg, ng), (xg, ng), x)):
        got, want = torch.autograd.grad(f(), to, n(g)), torch.autograd.grad(f(), to, -g)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_errors_keep_their_type(path):
    # an allocation that fails, and a hook that raises
    x, w, nw = (rand(s, torch.float32, 50 + i).cuda().requires_grad_() for i, s in enumerate([(4, 16), (8, 16), (16,)]))
    q, s = torch.zeros(1 << 20, 16, dtype=torch.int8, device="cuda"), torch.zeros(1 << 20, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):  # 4 TiB of outputs
        prm.int8_matmul(q, s, q, s, dtype=torch.float32)

    class Told(Exception):
        pass

    def hook(t):
        raise Told("no room")

    for f in (lambda: prm.int8_linear(x, w), lambda: prm.rms_norm(x, nw)):
        with torch.autograd.graph.saved_tensors_hooks(hook, lambda t: t):
            with pytest.raises(Told, match="no room"):
                f()


def test_frozen_parts_of_a_layer_keep_nothing(path):
    # x serves the weight's gradient alone, the weight the input's: what no gradient needs is not
    # kept, and may change
    x, w, b = (rand(s, torch.float32, 60 + i).cuda() for i, s in enumerate([(40, 64), (32, 64), (32,)]))
    gy = rand((40, 32), torch.float32, 63).cuda()
    for frozen, leaf in ((w, x), (x, w)):
        leaf.requires_grad_()
        want = torch.autograd.grad(prm.int8_linear(x, w, b), leaf, gy)[0]
        kept = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(tuple(t.shape)) or t, lambda t: t):
            y = prm.int8_linear(x, w, b)
        assert kept == [tuple(frozen.shape)]
        with torch.no_grad():
            leaf.add_(1)
        assert torch.equal(torch.autograd.grad(y, leaf, gy)[0], want)
        leaf.requires_grad_(False)
    b.requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t), lambda t: t):
        kept.clear()
        y = prm.int8_linear(x, w, b)
    assert not kept and torch.equal(torch.autograd.grad(y, b, torch.ones_like(y))[0], torch.full_like(b, 40))


def test_gradients_take_the_memory_of_what_is_asked_for():
    m, n, k, t = 4096, 2048, 1024, torch.bfloat16
    x, w = rand((m, k), t, 64).cuda(), rand((n, k), t, 65).cuda()
    gy = rand((m, n), t, 66).cuda()

    def peak(*leaves):
        for v in (x, w):
            v.requires_grad_(any(v is u for u in leaves))
        y = prm.int8_linear(x, w)
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        g = torch.autograd.grad(y, leaves, gy)
        out = sum(v.numel() * v.element_size() for v in g)
        return torch.cuda.max_memory_allocated() - before - out

    both, dx, dw = peak(x, w), peak(x), peak(w)
    # 8-bit operands: gy and w of one, both transposed of the other; a twentieth for scales and statistics
    assert dx <= 1.05 * (m * n + n * k) + (1 << 20) and dw <= 1.05 * (m * n + m * k) + (3 << 20) and both >= dx


def test_saved_tensors_of_a_layer_are_checked(path):
    # what hooks bring back is what was saved, whichever gradient is asked for
    x, w = rand((12, 40), torch.float32, 67).cuda(), rand((20, 40), torch.float32, 68).cuda()
    for wrong in (lambda t: t.half(), lambda t: t.cpu(), lambda t: t[:, :-1], lambda t: t[:-1]):
        for leaf in (x, w):
            leaf.requires_grad_()
            with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wrong):
                y = prm.int8_linear(x, w)
            with pytest.raises((RuntimeError, ValueError), match="saved "):
                torch.autograd.grad(y.sum(), leaf)
            leaf.requires_grad_(False)


def test_gradient_of_the_kept_sum_alone(path):
    # the weight takes no part in the kept sum, so it has no gradient, not one of zeros that a step
    # with weight decay would take
    x, w, r = (rand(s, torch.float32, 70 + i).cuda().requires_grad_() for i, s in enumerate([(7, 33), (33,), (7, 33)]))
    prm.rms_norm(x, w, r)[1].sum().backward()
    assert w.grad is None and (x.grad == 1).all() and (r.grad == 1).all()


# ---------------------------------------------------------------- many rows
@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", [(9000, 64), (2100, 600), (1100, 2056), (2300, 4090), (700, 4104), (600, 9000), (600, 17000), (600, 33000)], ids=str)
def test_norm_gradients_of_several_rows_a_block(shape, t):
    # on the GPU in 64 bits, as these are too many for the host
    x, w, gy, gh = (rand(s, t, 80 + i).cuda() for i, s in enumerate([shape, shape[1:], shape, shape]))
    for kept, need_w in ((True, True), (False, True), (True, False)):
        xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_(need_w)
        to = (xg, wg) if need_w else (xg,)
        if kept:
            got = torch.autograd.grad(prm.rms_norm(xg, wg, torch.zeros_like(x)), to, (gy, gh))
        else:
            got = torch.autograd.grad(prm.rms_norm(xg, wg), to, gy)
        h = x.double()
        r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
        g, n = gy.double() * w.double(), h * r
        dx = r * (g - n * (g * n).mean(1, keepdim=True))
        size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
        if kept:
            dx, size = dx + gh.double(), size + gh.double().abs()
        s = sums(shape[1])
        check(got[0], dx.cpu(), ((2.5 * s + 20) * U * size + half(t) * dx.abs() * (1 + 1e-3) + low(t)).cpu())
        if need_w:
            dw, size = (gy.double() * n).sum(0), (gy.double() * n).abs().sum(0)
            check(got[1], dw.cpu(), ((s / 2 + 6 + additions(*shape, t)) * U * size + half(t) * dw.abs() * (1 + 1e-3) + low(t)).cpu())


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("mnk", [(2500, 600, 1000), (2100, 40, 5000), (3001, 2100, 520), (2300, 24, 17000), (9001, 513, 48)], ids=str)
def test_linear_of_several_rows_a_block(mnk, t):
    # one call of the layer takes rows in turn where they are many: the bits of its parts, and the
    # parts those of the definition
    m, n, k = mnk
    x, w, gy = rand((m, k), t, 90).cuda(), rand((n, k), t, 91, 0.02).cuda(), rand((m, n), t, 92, 1e-2).cuda()
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    y = prm.int8_linear(xg, wg)
    gx, gw = torch.autograd.grad(y, (xg, wg), gy)
    assert torch.equal(y, prm.int8_matmul(*prm.quantize_rows(x), *prm.quantize_rows(w), dtype=t))
    assert torch.equal(gx, prm.int8_matmul(*prm.quantize_rows(gy), *prm.quantize_rows(w, transpose=True), dtype=t))
    assert torch.equal(gw, prm.int8_matmul(*prm.quantize_rows(gy, transpose=True), *prm.quantize_rows(x, transpose=True), dtype=t))
    for v in (x, gy):
        for a, b in ((prm.quantize_rows(v), eight(v.double().cpu())), (prm.quantize_rows(v, transpose=True), eight(v.double().cpu().t()))):
            assert torch.equal(a[0].cpu().double(), b[0])
            check_scale(a[1], b[1])


def test_rows_of_more_than_one_launch():
    # over 2^21 rows a kernel runs in slices
    t, rows, cols = torch.bfloat16, (1 << 21) + 4099, 24
    x, r, w = rand((rows, cols), t, 100).cuda(), rand((rows, cols), t, 101).cuda(), rand((cols,), t, 102).cuda()
    q, s = prm.quantize_rows(x)
    y, h = prm.rms_norm(x, w, r)
    q8, s8, h8 = prm.rms_norm(x, w, r, quantize=True)
    assert torch.equal(h, h8) and torch.equal(h, (x.float() + r.float()).to(t))
    for at in (slice(0, 300), slice((1 << 21) - 300, (1 << 21) + 300), slice(rows - 300, rows)):
        for a, b in ((q, s), (q8, s8)):
            assert a.shape == (rows, cols) and b.shape == (rows,)
        assert all(torch.equal(a, b) for a, b in zip((q[at], s[at]), prm.quantize_rows(x[at])))
        assert all(torch.equal(a, b) for a, b in zip((y[at], h[at]), prm.rms_norm(x[at], w, r[at])))
        assert all(torch.equal(a, b) for a, b in zip((q8[at], s8[at], h8[at]), prm.rms_norm(x[at], w, r[at], quantize=True)))
    qe, se = eight(x.double().cpu())
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se)
