"""The 8-bit linear layer's operators on the GPU against plain implementations in 64
bits on the CPU.

Tolerances count roundings, u = 2^-24 each for fp32 arithmetic and half a step,
finfo(type).eps / 2, for the one to the output's type (below its normal range: of the
range's fixed step):

* 8-bit values are exact, and so are sums of their products; a scale has at most 2 u
  (the quotient's rounding; for the norm also those of r, below).
* product: conversion, two factors and the bias: 4 u of |product| + |bias|.
* norm: a thread adds up to 8 ceil(cols / 512) squares one after the other (cols / 128 + 8
  for the rows that are swept), then 6 steps of a wave and at most 16 waves: S = that + 24
  roundings of the sum, so r has S / 2 + 4, y S / 2 + 6.
* its gradient: the same for r, and S for mean(g n): S + 12 u of
  r (|g| + |n| mean|g n|) + |gh|; dw: (S / 2 + 4 + 2) u for each term, and the additions:
  rows / parts + parts / 8 + 16, with parts of at least 1 and at most 2048 rows.
"""
import ctypes
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_20818_amd as prm  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}


def half(t):
    return torch.finfo(t).eps / 2


def low(t):
    # below the smallest normal number 2^e values lie 2^e eps apart, so rounding to one is
    # off by up to half of that (fp16: 2^-25), however small the value
    return torch.finfo(t).smallest_normal * half(t)


def rand(shape, t, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=g)).to(t)


def on_gpu(x, stride=None, offset=0):
    """x on the GPU as a view whose rows lie `stride` elements apart and start `offset`
    elements into an allocation, with NaN (for 8 bits: 99) around them."""
    if stride is None:
        return x.cuda()
    fill = 99 if x.dtype == torch.int8 else float("nan")
    flat = torch.full((offset + x.shape[0] * stride + 8,), fill, dtype=x.dtype, device="cuda")
    v = flat[offset:offset + x.shape[0] * stride].view(x.shape[0], stride)[:, :x.shape[1]]
    v.copy_(x)
    return v


def eight(v):
    """Rows of a 64-bit matrix in 8 bits, from the definition."""
    top = v.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(127 * v / top), torch.zeros_like(v))
    s = top[:, 0] / 127
    bad = ~torch.isfinite(v).all(1)
    q[bad], s[bad] = 0, float("nan")
    return q, s


def check_scale(got, want, rel=2 * U):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    # below fp32's normal range: half its smallest step
    assert ((got - want)[ok].abs() <= rel * want[ok].abs() + 2.0 ** -150).all()


def check(got, want, tol):
    err = (got.double().cpu() - want).abs()
    assert torch.isfinite(want).all() and (err <= tol).all(), f"worst {(err / tol.clamp_min(1e-300)).max():.3f} of the tolerance"


# ---------------------------------------------------------------- quantiser
ROWS = [(1, 1), (1, 7), (5, 8), (3, 64), (2, 511), (4, 513), (9, 1001), (2, 2048), (3, 4100), (1, 8192), (2, 12289), (2, 33000),
        (2100, 1000), (2049, 300), (600, 5000)]


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", ROWS, ids=str)
def test_quantize_rows(shape, t):
    x = rand(shape, t, 1)
    x[0, 0] = 3.0
    q, s = prm.quantize_rows(x.cuda())
    qe, se = eight(x.double())
    assert q.dtype == torch.int8 and tuple(q.shape) == shape and s.dtype == torch.float32
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se)


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", [(1, 1), (7, 1), (1, 9), (128, 64), (127, 65), (129, 63), (1000, 77), (77, 1000), (5000, 300), (64, 2050)],
                         ids=str)
def test_quantize_transposed(shape, t):
    x = rand(shape, t, 2)
    q, s = prm.quantize_rows(x.cuda(), transpose=True)
    qe, se = eight(x.double().t())
    assert tuple(q.shape) == shape[::-1]
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se)


def borders(t):
    """Rows with every border of two whole numbers: (k + 1/2) / 127 of the largest, and the
    values of the type next to it on both sides; largest values that leave the quotient
    exact and ones that do not."""
    rows = []
    for top in (127.0, 1.0, 254.0, 0.7, 3.14159, 96.5):
        top = torch.tensor(top, dtype=t).double()
        b = ((torch.arange(127).double() + 0.5) * top / 127).to(t)
        up = torch.nextafter(b.float(), torch.tensor(1e30)) if t == torch.float32 else (b.view(torch.int16) + 1).view(t)
        down = torch.nextafter(b.float(), torch.tensor(-1e30)) if t == torch.float32 else (b.view(torch.int16) - 1).view(t)
        v = torch.cat([b, up.to(t), -down.to(t), -b, top.to(t)[None]])
        rows.append(torch.minimum(torch.maximum(v, -top.to(t)), top.to(t)))
    return torch.stack(rows)


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_quantize_borders(t):
    x = borders(t)
    qe, se = eight(x.double())
    for got, want in ((prm.quantize_rows(x.cuda()), (qe, se)),
                      (prm.quantize_rows(x.t().contiguous().cuda(), transpose=True), (qe, se))):
        assert torch.equal(got[0].cpu().double(), want[0])
        check_scale(got[1], want[1])


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_quantize_special_rows(t):
    x = rand((8, 40), t, 3)
    x[0] = 0
    x[1] = 0
    x[1, 39] = -2
    x[2, 5] = float("inf")
    x[3, 0] = float("nan")
    x[4, 7], x[4, 8] = float("nan"), float("-inf")
    x[5] = x[5] * 1e-6
    x[6] = torch.finfo(t).max * torch.sign(x[6])
    x[7] = torch.finfo(t).tiny * torch.round(4 * x[7].float()).to(t)  # smallest normal numbers
    qe, se = eight(x.double())
    for got in (prm.quantize_rows(x.cuda()), prm.quantize_rows(x.t().contiguous().cuda(), transpose=True)):
        assert torch.equal(got[0].cpu().double(), qe)
        check_scale(got[1], se)


def test_quantize_subnormal_rows():
    x = torch.tensor([[1e-45, -3e-45, 0.0, 2.8e-45], [1e-40, 5e-39, -1.1e-38, 0.0]])
    q, s = prm.quantize_rows(x.cuda())
    qe, se = eight(x.double())
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se)


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_quantize_strides(t):
    x = rand((37, 101), t, 4)
    qe, se = eight(x.double())
    for stride, offset in ((101, 0), (104, 1), (113, 3)):
        v = on_gpu(x, stride, offset)
        q, s = prm.quantize_rows(v)
        assert torch.equal(q.cpu().double(), qe)
        check_scale(s, se)
        q, s = prm.quantize_rows(v, transpose=True)
        qc, sc = eight(x.double().t())
        assert torch.equal(q.cpu().double(), qc)
        check_scale(s, sc)
    # a transposed view, a row broadcast to many, more dimensions, a vector
    q, s = prm.quantize_rows(x.cuda().t())
    assert torch.equal(q.cpu().double(), eight(x.double().t())[0])
    q, s = prm.quantize_rows(x[:1].cuda().expand(6, 101))
    assert torch.equal(q.cpu().double(), qe[:1].expand(6, 101))
    q, s = prm.quantize_rows(x[:36].view(3, 12, 101).cuda())
    assert tuple(q.shape) == (3, 12, 101) and tuple(s.shape) == (3, 12)
    assert torch.equal(q.cpu().double().reshape(36, 101), qe[:36])
    q, s = prm.quantize_rows(x[5].cuda())
    assert tuple(s.shape) == () and torch.equal(q.cpu().double(), qe[5])
    q, s = prm.quantize_rows(x[:0].cuda())
    assert tuple(q.shape) == (0, 101) and tuple(s.shape) == (0,)


def test_quantize_writes_its_rows_only():
    # the C entry with a wide leading dimension: what lies between rows stays
    x = rand((5, 21), torch.float32, 5).cuda()
    q = torch.full((7, 40), 55, dtype=torch.int8, device="cuda")
    s = torch.full((9,), 8.0, device="cuda")
    L = prm.load()
    st = torch.cuda.current_stream().cuda_stream
    assert L.prm_quantize_rows(x.data_ptr(), prm.F32, 5, 21, 21, q[1].data_ptr() + 3, 40, s[2:].data_ptr(), st) == prm.PRM_OK
    want = torch.full((7, 40), 55.0, dtype=torch.float64)
    want.view(-1)[43:43 + 200].view(5, 40)[:, :21] = eight(x.double().cpu())[0]
    assert torch.equal(q.double().cpu(), want)
    assert (s[:2] == 8).all() and (s[7:] == 8).all()
    q = torch.full((23, 16), 55, dtype=torch.int8, device="cuda")
    ws = torch.empty(L.prm_quantize_cols_workspace(5, 21), dtype=torch.uint8, device="cuda")
    total = torch.full((22,), 8.0, device="cuda")
    s = torch.full((22,), 8.0, device="cuda")
    assert L.prm_quantize_cols(x.data_ptr(), prm.F32, 5, 21, 21, q[1].data_ptr() + 1, 16, s.data_ptr(), total.data_ptr(),
                               ws.data_ptr(), ws.numel(), st) == prm.PRM_OK
    want = torch.full((23, 16), 55.0, dtype=torch.float64)
    want.view(-1)[17:17 + 336].view(21, 16)[:, :5] = eight(x.double().cpu().t())[0]
    assert torch.equal(q.double().cpu(), want)
    assert s[21] == 8 and total[21] == 8
    check(total[:21], x.double().cpu().sum(0), 5 * U * x.double().cpu().abs().sum(0))


# ---------------------------------------------------------------- product
def int8s(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-128, 128, shape, generator=g, dtype=torch.int8)


def scales(n, seed):
    g = torch.Generator().manual_seed(seed)
    return 0.01 * torch.rand(n, generator=g) + 1e-4


def product64(a, sa, b, sb, bias=None):
    y = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    return y if bias is None else y + bias.double()


def check_product(got, a, sa, b, sb, bias, t):
    p = product64(a, sa, b, sb)
    y = p if bias is None else p + bias.double()
    add = torch.zeros_like(p) if bias is None else bias.double().abs().expand_as(p)
    check(got, y, 4 * U * (p.abs() + add) * (1 + half(t)) + half(t) * y.abs() + low(t))


PRODUCTS = [(1, 1, 1), (1, 16, 64), (1, 1000, 515), (3, 17, 33), (7, 130, 256), (16, 64, 129), (17, 100, 1000), (31, 33, 31), (32, 48, 4096),
            (33, 15, 700), (64, 200, 640), (65, 64, 128), (65, 63, 127), (128, 128, 128), (129, 130, 257), (200, 1, 100), (255, 257, 1024),
            (300, 700, 391), (2049, 2047, 160), (2305, 2304, 384), (512, 4096, 144),
            (1500, 1501, 2049), (40, 5000, 9001)]


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("mnk", PRODUCTS, ids=str)
def test_product(mnk, t):
    m, n, k = mnk
    a, b, sa, sb = int8s((m, k), 6), int8s((n, k), 7), scales(m, 8), scales(n, 9)
    bias = rand((n,), t, 10) if (m + n + k) % 2 else None
    got = prm.int8_matmul(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), bias=None if bias is None else bias.cuda(), dtype=t)
    assert got.dtype == t and tuple(got.shape) == (m, n)
    check_product(got, a, sa, b, sb, bias, t)


@pytest.mark.parametrize("m", [1, 20, 40, 64, 65, 140, 600])
def test_product_strides(m):
    n, k, t = 75, 203, torch.float32
    a, b, sa, sb = int8s((m, k), 11), int8s((n, k), 12), scales(m, 13), scales(n, 14)
    for lda, ldb, oa, ob in ((208, 208, 0, 0), (204, 207, 1, 3), (256, 203, 16, 0), (240, 224, 16, 32)):
        got = prm.int8_matmul(on_gpu(a, lda, oa), sa.cuda(), on_gpu(b, ldb, ob), sb.cuda(), dtype=t)
        check_product(got, a, sa, b, sb, None, t)
    got = prm.int8_matmul(a.t().contiguous().cuda().t(), sa.cuda(), b.cuda(), sb.cuda(), dtype=t)
    check_product(got, a, sa, b, sb, None, t)


# kernels by number (1: few tokens, 2 and 3: rows on any byte, tiles of 64 and 128, 4 to 6: 64,
# 128, 128 with two buffers, 7: 256), in how many pieces k is split, and which operands are
# laid out anew (1: a, 2: b)
KERNELS = [(1, 1, 0), (2, 1, 0), (3, 1, 0), (4, 1, 0), (5, 1, 0), (6, 1, 0), (7, 1, 0), (4, 2, 0), (4, 7, 0), (5, 3, 0), (4, 1, 3), (4, 3, 3),
           (5, 1, 1), (5, 2, 2), (6, 1, 3), (7, 1, 1), (7, 1, 2), (7, 1, 3)]
SIZES = [(1, 1, 1), (3, 65, 515), (16, 100, 3000), (65, 64, 16), (70, 50, 128), (129, 257, 400), (300, 300, 1000), (257, 511, 1072), (513, 130, 1152),
         (64, 70, 8192), (520, 900, 2053)]


@pytest.mark.parametrize("kernel", KERNELS, ids=str)
def test_every_kernel(kernel):
    # every kernel at every size that it takes, whatever the rule would choose
    kind, splits, pack = kernel
    P, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    f = prm.load().prm_internal_int8_matmul
    f.argtypes = [P, i64, P, P, i64, P, P, i32, P, i64, i64, i64, i64, P, ctypes.c_uint64, P, i32, i32, i32]
    ran = 0
    for m, n, k in SIZES:
        even, any_ = (k + 15) // 16 * 16, k + k % 2
        lda = any_ if kind <= 3 or pack & 1 else even
        ldb = any_ if kind <= 3 or pack & 2 else even
        a, b, sa, sb, t = int8s((m, k), 22), int8s((n, k), 23), scales(m, 24), scales(n, 25), torch.float32
        ag, bg = on_gpu(a, lda, pack & 1), on_gpu(b, ldb, 3 * (pack & 2))
        bias = rand((n,), t, 26)
        ws = torch.empty(splits * m * (n + 7) * 4 + (m + n) * (k + 127), dtype=torch.uint8, device="cuda")
        out = torch.full((m + 1, n + 3), 7.0, device="cuda")
        sag, sbg, biasg = sa.cuda(), sb.cuda(), bias.cuda()
        rc = f(ag.data_ptr(), lda, sag.data_ptr(), bg.data_ptr(), ldb, sbg.data_ptr(), biasg.data_ptr(), prm.F32, out.data_ptr(), n + 3, m, n, k,
               ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream, kind, splits, pack)
        if rc == prm.PRM_EINVAL and (kind == 1 and m > 16 or splits > k // 128):
            continue
        assert rc == prm.PRM_OK, prm.load().prm_last_error()
        ran += 1
        check_product(out[:m, :n], a, sa, b, sb, bias, t)
        out[:m, :n] = 7
        assert (out == 7).all()
    assert ran >= 3


def test_product_without_its_workspace():
    m, n, k = 40, 200, 16000
    a, b, sa, sb = int8s((m, k), 27).cuda(), int8s((n, k), 28).cuda(), scales(m, 29).cuda(), scales(n, 30).cuda()
    L = prm.load()
    assert L.prm_int8_matmul_workspace(a.data_ptr(), k, b.data_ptr(), k, m, n, k) > 0
    want = prm.int8_matmul(a, sa, b, sb, dtype=torch.float32)
    got = torch.empty_like(want)
    for ws, need in ((None, 0), (torch.empty(16, dtype=torch.uint8, device="cuda"), 16)):
        got.zero_()
        assert L.prm_int8_matmul(a.data_ptr(), k, sa.data_ptr(), b.data_ptr(), k, sb.data_ptr(), None, prm.F32, got.data_ptr(), n, m, n, k,
                                 None if ws is None else ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == prm.PRM_OK
        assert torch.equal(got, want)


@pytest.mark.parametrize("m,k", [(1, 131071), (64, 131071), (70, 131071), (300, 131071)])
def test_product_longest_sum(m, k):
    # every term as large as it can be: the sum comes within 2^14 of 2^31
    n = 34
    a = torch.full((m, k), -128, dtype=torch.int8)
    b = torch.full((n, k), -128, dtype=torch.int8)
    one = torch.ones(1)
    got = prm.int8_matmul(a.cuda(), one.expand(m).cuda(), b.cuda(), one.expand(n).cuda(), dtype=torch.float32)
    assert (got.double().cpu() == float(torch.tensor(16384.0 * k, dtype=torch.float32))).all()


@pytest.mark.parametrize("m,k", [(1, 131072), (3, 300000), (200, 262161), (70, 1 << 20)])
def test_product_of_sums_past_32_bits(m, k):
    # split, and joined in 64 bits; each term 2^14, so the sum in fp32 is off by its own rounding
    n, ld = 40, (k + 15) // 16 * 16
    a, b = (torch.full((r, ld), -128, dtype=torch.int8, device="cuda")[:, :k] for r in (m, n))
    one = torch.ones(max(m, n), device="cuda")
    got = prm.int8_matmul(a, one[:m], b, one[:n], dtype=torch.float32)
    assert (got.double() == float(torch.tensor(16384.0 * k, dtype=torch.float32))).all()
    g = torch.Generator(device="cuda").manual_seed(3)
    a.copy_(torch.randint(-128, 128, (m, k), dtype=torch.int8, device="cuda", generator=g))
    b.copy_(torch.randint(-128, 128, (n, k), dtype=torch.int8, device="cuda", generator=g))
    got = prm.int8_matmul(a, one[:m], b, one[:n], dtype=torch.float32)
    assert torch.equal(got, (a.double() @ b.double().t()).float())
    if k % 16:  # rows on any byte
        assert torch.equal(got, prm.int8_matmul(a.contiguous(), one[:m], b, one[:n], dtype=torch.float32))


def test_offsets_past_32_bits():
    # matrices of more than 2^32 bytes, and of more than 2^31 elements: their last rows
    t, rows, cols = torch.bfloat16, 70000, 32768
    x = torch.zeros(rows, cols, dtype=t, device="cuda")
    end = rand((40, cols), t, 150)
    x[-40:] = end.cuda()
    w = rand((cols,), t, 151)
    qe, se = eight(end.double())
    q, s = prm.quantize_rows(x)
    assert torch.equal(q[-40:].cpu().double(), qe) and (q[:-40] == 0).all() and (s[:-40] == 0).all()
    check_scale(s[-40:], se)
    y = prm.rms_norm(x, w.cuda())
    assert torch.equal(y[-40:], prm.rms_norm(end.cuda(), w.cuda()))
    del y
    a, sa = int8s((20, cols), 152).cuda(), scales(20, 153).cuda()
    out = prm.int8_matmul(a, sa, q, s, dtype=torch.float32)
    assert torch.equal(out[:, -40:], prm.int8_matmul(a, sa, q[-40:].clone(), s[-40:].clone(), dtype=torch.float32))
    assert (out[:, :-40] == 0).all()
    out = prm.int8_matmul(q, s, a, sa, dtype=t)
    assert torch.equal(out[-40:], prm.int8_matmul(q[-40:].clone(), s[-40:].clone(), a, sa, dtype=t))
    del q, s, out
    qt, st = prm.quantize_rows(x, transpose=True)
    want, sw = eight(end.double().t())
    assert torch.equal(qt[-1].cpu().double()[-40:], want[-1]) and torch.equal(qt[:, -40:].cpu().double(), want)
    check_scale(st, sw)


def test_layer_of_many_tokens():
    # more tokens than one piece of the weight's gradient holds
    t, m, n, k = torch.bfloat16, 140000, 24, 40
    x, w, gy = rand((m, k), t, 154).cuda().requires_grad_(), rand((n, k), t, 155).cuda().requires_grad_(), rand((m, n), t, 156).cuda()
    y = prm.int8_linear(x, w)
    gx, gw = torch.autograd.grad(y, (x, w), gy)
    (gq, gs), (xq, xs) = (eight(v.detach().cpu().double().t()) for v in (gy, x))
    want = product64(gq, gs, xq, xs)
    check(gw, want, 8 * U * want.abs() + half(t) * want.abs() * (1 + 1e-3) + low(t))
    assert torch.equal(y[-100:], prm.int8_linear(x[-100:].detach(), w.detach()))
    assert torch.equal(gx[-100:], prm.int8_matmul(*prm.quantize_rows(gy[-100:]), *prm.quantize_rows(w.detach(), transpose=True), dtype=t))


def test_product_leaves_what_is_around():
    m, n, k = 70, 35, 50
    a, b, sa, sb = int8s((m, k), 15), int8s((n, k), 16), scales(m, 17), scales(n, 18)
    L, st = prm.load(), torch.cuda.current_stream().cuda_stream
    ag, bg, sag, sbg = a.cuda(), b.cuda(), sa.cuda(), sb.cuda()
    for mm in (5, 70):
        out = torch.full((mm + 2, 48), 7.0, device="cuda")
        assert L.prm_int8_matmul(ag.data_ptr(), k, sag.data_ptr(), bg.data_ptr(), k, sbg.data_ptr(), None, prm.F32, out[1].data_ptr() + 4,
                                 48, mm, n, k, None, 0, st) == prm.PRM_OK
        check_product(out[1:mm + 1, 1:n + 1], a[:mm], sa[:mm], b, sb, None, torch.float32)
        out[1:mm + 1, 1:n + 1] = 7
        assert (out == 7).all()


def test_product_shapes_and_poisoned_rows():
    a, b, sa, sb = int8s((2, 3, 40), 19), int8s((9, 40), 20), scales(6, 21).view(2, 3), scales(9, 22)
    sa[1, 1] = float("nan")
    got = prm.int8_matmul(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), dtype=torch.float32)
    assert tuple(got.shape) == (2, 3, 9)
    assert torch.isnan(got[1, 1]).all() and torch.isfinite(got[0]).all() and torch.isfinite(got[1, 0]).all()
    one = prm.int8_matmul(a[0, 0].cuda(), sa[0, 0].cuda(), b.cuda(), sb.cuda(), dtype=torch.float32)
    assert tuple(one.shape) == (9,) and torch.equal(one, got[0, 0])
    none = prm.int8_matmul(a[:0].cuda(), sa[:0].cuda(), b.cuda(), sb.cuda())
    assert tuple(none.shape) == (0, 3, 9)


def test_refusals():
    a, s = int8s((4, 16), 1).cuda(), scales(4, 1).cuda()
    x = rand((4, 16), torch.bfloat16, 1).cuda()
    bad = [lambda: prm.int8_matmul(a, s, a[:, :8], s), lambda: prm.int8_matmul(a, s[:3], a, s), lambda: prm.int8_matmul(a, s.half(), a, s),
           lambda: prm.int8_matmul(x, s, a, s), lambda: prm.int8_matmul(a, s, a, s, bias=s), lambda: prm.int8_matmul(a, s, a, s.cpu()),
           lambda: prm.int8_matmul(a, s, a, s, dtype=torch.float64), lambda: prm.int8_matmul(a, s, a.view(2, 2, 16), s),
           lambda: prm.quantize_rows(x.double()), lambda: prm.quantize_rows(x.view(2, 2, 16), transpose=True),
           lambda: prm.quantize_rows(a), lambda: prm.quantize_rows(x[:, :0]),
           lambda: prm.rms_norm(x, x[0].float()), lambda: prm.rms_norm(x, x[0, :8]), lambda: prm.rms_norm(x, residual=x[:2]),
           lambda: prm.rms_norm(x, residual=x.float()), lambda: prm.rms_norm(x.clone().requires_grad_(), quantize=True),
           lambda: prm.int8_linear(x, x[:, :8]), lambda: prm.int8_linear(x, x.float()), lambda: prm.int8_linear(x, x, x[0]), lambda: prm.int8_linear(x, x[:0])]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused:", i)
    for f in (lambda: prm.rms_norm(x, eps=0.0), lambda: prm.quantize_rows(x[:0], transpose=True)):
        with pytest.raises(prm.PRMError):
            f()
    host = torch.zeros(64, dtype=torch.bfloat16)
    q, sc = torch.empty(64, dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
    rc = prm.load().prm_quantize_rows(host.data_ptr(), prm.BF16, 8, 8, 8, q.data_ptr(), 8, sc.data_ptr(), None)
    assert rc == prm.PRM_EINVAL and "device memory" in prm.load().prm_last_error().decode()


# ---------------------------------------------------------------- norm
def norm64(x, res, w, eps, t):
    h = x.double() if res is None else (x.double() + res.double()).to(t).double()
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, r, h * r * (w.double() if w is not None else 1.0)


def sums(cols):
    return max(8 * -(-cols // 512), cols // 128 + 8) + 24


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", ROWS, ids=str)
def test_norm(shape, t):
    x, res, w = rand(shape, t, 23), rand(shape, t, 24, 3.0), rand(shape[1:], t, 25)
    for rs, wt in ((None, w), (res, w), (res, None)):
        h, _, y = norm64(x, rs, wt, 1e-6, t)
        got = prm.rms_norm(x.cuda(), None if wt is None else wt.cuda(), None if rs is None else rs.cuda())
        if rs is not None:
            got, kept = got
            # fp32 addition of two values of the type, rounded once: as torch's
            assert torch.equal(kept.cpu(), (x.float() + res.float()).to(t))
            h2 = kept.cpu().double()
            assert torch.equal(h2, h) or t == torch.float32
            h, _, y = norm64(kept.cpu(), None, wt, 1e-6, t)
        check(got, y, ((sums(shape[1]) / 2 + 6) * U + half(t)) * y.abs() * (1 + half(t)) + low(t))


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", ROWS, ids=str)
def test_norm_eight_bits(shape, t):
    x, res, w = rand(shape, t, 26), rand(shape, t, 27, 3.0), rand(shape[1:], t, 28)
    for rs, wt in ((None, w), (res, w), (res, None)):
        got = prm.rms_norm(x.cuda(), None if wt is None else wt.cuda(), None if rs is None else rs.cuda(), quantize=True)
        h = x
        if rs is not None:
            h = got[2].cpu()
            assert torch.equal(h, (x.float() + res.float()).to(t))
        _, r, _ = norm64(h, None, wt, 1e-6, t)
        u = h.double() * (wt.double() if wt is not None else 1.0)
        qe, se = eight(u)  # r cancels from q
        assert torch.equal(got[0].cpu().double(), qe)
        check_scale(got[1], se * r[:, 0], (sums(shape[1]) / 2 + 6) * U)


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_norm_special_rows(t):
    x, w = rand((5, 100), t, 29), rand((100,), t, 30)
    x[0] = 0
    x[1] = 0
    x[1, 99] = 1e-3
    x[2, 3] = float("nan")
    x[3, 4] = float("inf")
    q, s = prm.rms_norm(x.cuda(), w.cuda(), quantize=True)
    y = prm.rms_norm(x.cuda(), w.cuda())
    assert (q[0] == 0).all() and s[0] == 0 and (y[0] == 0).all()
    assert abs(int(q[1, 99])) == 127 and (q[1, :99] == 0).all()
    for i in (2, 3):
        assert torch.isnan(s[i]) and (q[i] == 0).all()
    assert torch.isnan(y[2]).all() and torch.isnan(y[3, 4])
    _, _, y4 = norm64(x[4:], None, w, 1e-6, t)
    check(y[4:], y4, ((sums(100) / 2 + 6) * U + half(t)) * y4.abs() * (1 + half(t)) + low(t))
    wn = w.clone()
    wn[5] = float("nan")
    q, s = prm.rms_norm(x.cuda(), wn.cuda(), quantize=True)
    assert torch.isnan(s[4]) and (q[4] == 0).all()


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_norm_strides(t):
    x, res, w = rand((12, 75), t, 31), rand((12, 75), t, 32), rand((75,), t, 33)
    want = prm.rms_norm(x.cuda(), w.cuda(), res.cuda())
    for sx, ox, sr, orr in ((75, 1, 77, 2), (80, 3, 91, 0)):
        got = prm.rms_norm(on_gpu(x, sx, ox), on_gpu(w[None], 75, 1)[0], on_gpu(res, sr, orr))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got8, want8 = (prm.rms_norm(a, w.cuda(), b, quantize=True) for a, b in ((on_gpu(x, sx, ox), on_gpu(res, sr, orr)), (x.cuda(), res.cuda())))
        assert all(torch.equal(a, b) for a, b in zip(got8, want8))
    y, h = prm.rms_norm(x.cuda().view(3, 4, 75), w.cuda(), res.cuda().view(3, 4, 75))
    assert torch.equal(y.view(12, 75), want[0]) and torch.equal(h.view(12, 75), want[1])
    y = prm.rms_norm(x[:0].cuda(), w.cuda())
    assert tuple(y.shape) == (0, 75)
    # a weight with a stride, the same tensor as input and residual
    w2 = torch.stack([w, w], 1).cuda()[:, 0]
    assert torch.equal(prm.rms_norm(x.cuda(), w2, res.cuda())[0], want[0])
    a = x.cuda()
    y, h = prm.rms_norm(a, w.cuda(), a)
    assert torch.equal(h, a + a)


GRADS = [(1, 1), (1, 9), (3, 64), (5, 511), (9, 513), (4, 1001), (3, 2049), (2, 4096), (2, 4100), (2, 12289), (3, 33000), (1500, 72), (2600, 515),
         (5001, 16)]


def parts(rows):
    return max(1, rows // 2048) + min(rows, 2048) // 8 + 32


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("shape", GRADS, ids=str)
def test_norm_gradients(shape, t):
    x, res, w = rand(shape, t, 34), rand(shape, t, 35), rand(shape[1:], t, 36)
    gy, gh = rand(shape, t, 37), rand(shape, t, 38)
    for rs, wt, ghh in ((None, w, None), (res, w, gh), (res, None, gh), (res, w, None)):
        leaves = [v.cuda().requires_grad_() for v in (x, rs, wt) if v is not None]
        it = iter(leaves)
        xg = next(it)
        rg = next(it) if rs is not None else None
        wg = next(it) if wt is not None else None
        out = prm.rms_norm(xg, wg, rg)
        if rs is None:
            got, h = torch.autograd.grad(out, leaves, gy.cuda()), x.double()
        elif ghh is None:
            got, h = torch.autograd.grad(out[0], leaves, gy.cuda()), out[1].detach().cpu().double()
        else:
            got, h = torch.autograd.grad(out, leaves, (gy.cuda(), gh.cuda())), out[1].detach().cpu().double()
        f = wt.double() if wt is not None else torch.ones(shape[1], dtype=torch.float64)
        cols = shape[1]
        r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
        g, n = gy.double() * f, h * r
        dx = r * (g - n * (g * n).mean(1, keepdim=True))
        size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
        if ghh is not None:
            dx, size = dx + gh.double(), size + gh.double().abs()
        s = sums(cols)
        check(got[0], dx, 2 * (s + 12) * U * size + half(t) * dx.abs() * (1 + 1e-3) + low(t))
        if rs is not None:
            assert torch.equal(got[0], got[1])
        if wt is not None:
            dw = (gy.double() * n).sum(0)
            size = (gy.double() * n).abs().sum(0)
            check(got[-1], dw, (s / 2 + 6 + parts(shape[0])) * U * size + half(t) * dw.abs() * (1 + 1e-3) + low(t))


def test_norm_gradients_against_differences():
    # y . gy along a direction, from the kernel itself: central differences of step e are off
    # by e^2 / 6 of the third derivative and, as each value has about 2^-22 relative, by
    # 2^-22 sum |y gy| / e
    shape, t = (6, 50), torch.float32
    x, w, gy = rand(shape, t, 39).cuda(), rand((50,), t, 40).cuda(), rand(shape, t, 41).cuda()
    dx, dw = rand(shape, t, 42).cuda(), rand((50,), t, 43).cuda()
    xg, wg = x.clone().requires_grad_(), w.clone().requires_grad_()
    y = prm.rms_norm(xg, wg)
    gx, gw = torch.autograd.grad(y, (xg, wg), gy)
    e = 2.0 ** -8
    f = lambda a, b: (prm.rms_norm(a, b).double() * gy.double()).sum().item()  # noqa: E731
    noise = 2.0 ** -22 * (y.detach().abs().double() * gy.abs().double()).sum().item() / e
    for got, lo, hi in (((gx * dx).double().sum().item(), f(x - e * dx, w), f(x + e * dx, w)),
                        ((gw * dw).double().sum().item(), f(x, w - e * dw), f(x, w + e * dw))):
        assert abs(got - (hi - lo) / (2 * e)) <= noise + 40 * e * e * 6


def test_norm_gradients_of_layouts():
    # a broadcast gradient (from a sum), one with another stride, only the kept sum's, none of the weight's
    x, res, w = (rand(s, torch.float32, 44 + i).cuda().requires_grad_() for i, s in enumerate(((7, 33), (7, 33), (33,))))
    y, h = prm.rms_norm(x, w, res)
    a = torch.autograd.grad(y.sum(), (x, w), retain_graph=True)
    b = torch.autograd.grad(y, (x, w), torch.ones(7, 33, device="cuda"), retain_graph=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    g = rand((33, 7), torch.float32, 50).cuda()
    a = torch.autograd.grad(y, (x, w), g.t(), retain_graph=True)
    b = torch.autograd.grad(y, (x, w), g.t().contiguous(), retain_graph=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    a = torch.autograd.grad(h, (x, res, w), g.t(), retain_graph=True, allow_unused=True)
    assert torch.equal(a[0], g.t()) and torch.equal(a[1], g.t()) and (a[2] is None or (a[2] == 0).all())
    a = torch.autograd.grad(y, x, g.t())[0]
    assert torch.equal(a, b[0])
    x0 = torch.zeros(0, 33, device="cuda", requires_grad=True)
    gx, gw = torch.autograd.grad(prm.rms_norm(x0, w).sum(), (x0, w))
    assert tuple(gx.shape) == (0, 33) and (gw == 0).all()


# ---------------------------------------------------------------- layer
@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("mnk", [(1, 1, 1), (1, 40, 100), (7, 33, 65), (64, 48, 96), (100, 130, 257), (300, 259, 129)], ids=str)
def test_linear(mnk, t):
    m, n, k = mnk
    x, w, b = rand((m, k), t, 51), rand((n, k), t, 52, 0.02), rand((n,), t, 53)
    gy = rand((m, n), t, 54, 1e-2)
    leaves = [v.cuda().requires_grad_() for v in (x, w, b)]
    y = prm.int8_linear(*leaves)
    got = torch.autograd.grad(y, leaves, gy.cuda())

    def scaled(v):
        q, s = eight(v.double())
        return q, s.float()

    check_product(y.detach(), *scaled(x), *scaled(w), b, t)
    # a scale's own rounding: 2 u of it on both sides
    for out, p, q in ((got[0], scaled(gy), scaled(w.t())), (got[1], scaled(gy.t()), scaled(x.t()))):
        want = product64(*p, *q)
        check(out, want, 8 * U * want.abs() + half(t) * want.abs() * (1 + 1e-3) + low(t))
    db = gy.double().sum(0)
    check(got[2], db, (m / 8 + 24) * U * gy.double().abs().sum(0) + half(t) * db.abs() * (1 + 1e-3) + low(t))


def test_linear_gradients_against_the_unquantised_layer():
    # each operand of a product is off by at most half of 1/127 of its row's largest value, so
    # |Q(A) Q(B)^T - A B^T| <= sum_k (|A| eb + |B| ea + ea eb); and the same bound holds for
    # differences of the unquantised layer, which is linear: its gradients are their limits
    m, n, k, t = 96, 80, 112, torch.float32
    x, w, gy = rand((m, k), t, 55), rand((n, k), t, 56), rand((m, n), t, 57)
    leaves = [v.cuda().requires_grad_() for v in (x, w)]
    y = prm.int8_linear(*leaves)
    got = torch.autograd.grad(y, leaves, gy.cuda())
    for out, a, b in ((y.detach(), x, w), (got[0], gy, w.t()), (got[1], gy.t(), x.t())):
        a, b = a.double(), b.double()
        ea, eb = (v.abs().amax(1, keepdim=True).expand_as(v) / 254 * (1 + 4 * U) for v in (a, b))
        bound = a.abs() @ eb.t() + ea @ b.abs().t() + ea @ eb.t()
        check(out, a @ b.t(), bound + 1e-5)


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("mnk", [(1, 1, 1), (5, 700, 33), (130, 513, 600), (64, 96, 2049), (33, 5000, 70), (40, 17, 20000), (3000, 24, 40)], ids=str)
def test_linear_is_its_parts(mnk, t):
    # one call of the layer, and the quantisers and products that it is made of: the same bits
    m, n, k = mnk
    x, w, b = rand((m, k), t, 111).cuda(), rand((n, k), t, 112, 0.02).cuda(), rand((n,), t, 113).cuda()
    gy = rand((m, n), t, 114, 1e-2).cuda()
    leaves = [v.requires_grad_() for v in (x, w, b)]
    y = prm.int8_linear(*leaves)
    got = torch.autograd.grad(y, leaves, gy)
    with torch.no_grad():
        assert torch.equal(y, prm.int8_matmul(*prm.quantize_rows(x), *prm.quantize_rows(w), bias=b, dtype=t))
        assert torch.equal(y, prm.int8_linear(x, w, b))
        assert torch.equal(got[0], prm.int8_matmul(*prm.quantize_rows(gy), *prm.quantize_rows(w, transpose=True), dtype=t))
        assert torch.equal(got[1], prm.int8_matmul(*prm.quantize_rows(gy, transpose=True), *prm.quantize_rows(x, transpose=True), dtype=t))


@pytest.mark.parametrize("t", TYPES, ids=NAMES.get)
def test_python_path_is_the_native_one(t, monkeypatch):
    # the calls that native code leaves to Python, and all of them where it is not built
    from paper_2608_20818_amd import operators
    x, res, w = (rand(s, t, 120 + i).cuda().requires_grad_() for i, s in enumerate([(9, 70), (9, 70), (70,)]))
    wl, b = rand((20, 70), t, 123).cuda().requires_grad_(), rand((20,), t, 124).cuda().requires_grad_()
    gy = rand((9, 20), t, 125).cuda()

    def run():
        y, h = prm.rms_norm(x, w, res)
        z = prm.int8_linear(y, wl, b)
        out = [y, h, z, *torch.autograd.grad((z, h), (x, res, w, wl, b), (gy, torch.ones_like(h)))]
        with torch.no_grad():
            q, s, h8 = prm.rms_norm(x, w, res, quantize=True)
            out += [q, s, h8, *prm.quantize_rows(wl), *prm.quantize_rows(wl, transpose=True), prm.rms_norm(x),
                    prm.int8_matmul(q, s, *prm.quantize_rows(wl), bias=b, dtype=t)]
        return [v.detach() for v in out]

    native = run()
    monkeypatch.setattr(operators, "_native", type("none", (), {n: staticmethod(lambda *a: None) for n in (
        "quantize_rows", "quantize_cols", "int8_matmul", "int8_linear", "rms_norm")}))
    assert all(torch.equal(a, c) for a, c in zip(native, run()))


def test_gradients_once():
    # gradients of gradients are refused, and not before they are asked for
    for native in (True, False):
        x, w, wl = (rand(s, torch.float32, 130 + i).cuda().requires_grad_() for i, s in enumerate([(4, 16), (16,), (8, 16)]))
        xv = x if native else x.as_subclass(type("Sub", (torch.Tensor,), {}))
        for y, v in ((prm.rms_norm(xv, w), w), (prm.int8_linear(xv, wl), wl)):
            gx, gv = torch.autograd.grad(y.sum(), (x, v), create_graph=True)
            assert torch.isfinite(gx).all() and torch.isfinite(gv).all()
            with pytest.raises(RuntimeError, match="differentia"):
                torch.autograd.grad(gx.square().sum(), x)


def test_saved_tensor_hooks():
    # saved on the host and brought back: the same gradients; brought back wrong: refused
    x, w, wl, r = (rand(s, torch.float32, 160 + i).cuda().requires_grad_() for i, s in enumerate([(12, 40), (40,), (20, 40), (12, 40)]))

    def run():
        y, h = prm.rms_norm(x, w, r)
        z = prm.int8_linear(y, wl)
        return torch.autograd.grad(z.sum() + h.sum(), (x, w, wl, r))

    want = run()
    with torch.autograd.graph.save_on_cpu():
        assert all(torch.equal(a, b) for a, b in zip(want, run()))
    back = lambda t: t.t().contiguous().t() if t.dim() == 2 else t  # noqa: E731  (other strides)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, back):
        assert all(torch.equal(a, b) for a, b in zip(want, run()))
    for wrong in (lambda t: t.half(), lambda t: t.cpu(), lambda t: t[..., :-1]):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wrong):
            with pytest.raises(RuntimeError, match="saved tensor|invalid gradient"):  # or by autograd: both cut alike
                torch.autograd.grad(prm.int8_linear(x, wl).sum(), wl)
            with pytest.raises(RuntimeError, match="saved tensor"):
                torch.autograd.grad(prm.rms_norm(x, w).sum(), w)


def test_saved_tensors_changed_in_place():
    x, wl = rand((4, 16), torch.float32, 140).cuda().requires_grad_(), rand((8, 16), torch.float32, 141).cuda().requires_grad_()
    for f in (lambda: prm.int8_linear(x, wl), lambda: prm.rms_norm(x)):
        y = f()
        with torch.no_grad():
            x.add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            torch.autograd.grad(y.sum(), x)


def test_accumulates_into_leaves():
    # .backward() twice adds, through a parameter used by two layers
    x, p = rand((6, 32), torch.float32, 142).cuda(), torch.nn.Parameter(rand((32, 32), torch.float32, 143).cuda())
    y = prm.int8_linear(prm.int8_linear(x, p), p)
    y.sum().backward()
    once = p.grad.clone()
    prm.int8_linear(prm.int8_linear(x, p), p).sum().backward()
    assert torch.equal(p.grad, once + once)


def test_linear_layouts():
    t = torch.bfloat16
    x, w, b = rand((2, 5, 48), t, 58).cuda(), rand((31, 48), t, 59).cuda(), rand((31,), t, 60).cuda()
    leaves = [v.requires_grad_() for v in (x, w, b)]
    y = prm.int8_linear(*leaves)
    assert tuple(y.shape) == (2, 5, 31)
    got = torch.autograd.grad(y.sum(), leaves)
    flat = prm.int8_linear(x.detach().view(10, 48), w.detach(), b.detach())
    assert torch.equal(flat, y.detach().view(10, 31))
    assert [tuple(g.shape) for g in got] == [(2, 5, 48), (31, 48), (31,)]
    assert (got[2] == 10).all()
    only = torch.autograd.grad(prm.int8_linear(x.detach(), w.detach(), b).sum(), b)[0]
    assert (only == 10).all()
    x0 = torch.zeros(0, 48, dtype=t, device="cuda", requires_grad=True)
    got = torch.autograd.grad(prm.int8_linear(x0, w, b).sum(), (x0, w, b))
    assert tuple(got[0].shape) == (0, 48) and (got[1] == 0).all() and (got[2] == 0).all()


# ---------------------------------------------------------------- together
def test_serving_chain_other_stream_and_graph():
    t = torch.bfloat16
    x, res, w = rand((3, 264), t, 61).cuda(), rand((3, 264), t, 62).cuda(), rand((264,), t, 63).cuda()
    wq, ws = prm.quantize_rows(rand((500, 264), t, 64, 0.02).cuda())

    def chain():
        q, s, h = prm.rms_norm(x, w, residual=res, quantize=True)
        return prm.int8_matmul(q, s, wq, ws, dtype=t), h

    want = chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        kept = chain()
    for i in range(4):
        x.copy_(rand((3, 264), t, 70 + i))
        want = chain()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)), i


def test_captured_gradients_and_two_graphs():
    # forward and backward captured, twice: the graphs share no workspace
    t = torch.float32
    x, w = rand((40, 96), t, 80).cuda().requires_grad_(), rand((96,), t, 81).cuda().requires_grad_()
    wl = rand((50, 96), t, 82).cuda().requires_grad_()
    gy = rand((40, 50), t, 83).cuda()

    def step():
        y = prm.int8_linear(prm.rms_norm(x, w), wl)
        return (y.detach(), *torch.autograd.grad(y, (x, w, wl), gy))

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for i in range(4):
        with torch.no_grad():
            x.copy_(rand((40, 96), t, 90 + i))
        want = step()
        torch.cuda.synchronize()
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_trains_with_the_step():
    # the layer's gradients through the optimizer step: norm, 8-bit layer and update run together;
    # the weights move as they do on the gradients handed to the step directly
    torch.manual_seed(0)
    x = rand((64, 128), torch.float32, 100).cuda()
    ps = [rand(s, torch.float32, 101 + i, 0.1).cuda() for i, s in enumerate([(128,), (256, 128), (256,)])]
    ps = [torch.nn.Parameter(p) for p in ps]
    twin = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    opt, opt2 = (prm.PRMOptimizer(q, lr=0.01, K=2) for q in (ps, twin))
    for _ in range(3):
        h = prm.rms_norm(x, ps[0])
        y = prm.int8_linear(h, ps[1], ps[2])
        loss = y.square().mean()
        loss.backward()
        gy = 2 * y.detach() / y.numel()
        with torch.no_grad():
            dh = prm.int8_matmul(*prm.quantize_rows(gy), *prm.quantize_rows(ps[1], transpose=True), dtype=torch.float32)
            dw = prm.int8_matmul(*prm.quantize_rows(gy, transpose=True), *prm.quantize_rows(h, transpose=True), dtype=torch.float32)
        assert torch.equal(ps[1].grad, dw)
        nw = torch.nn.Parameter(ps[0].detach().clone())
        prm.rms_norm(x, nw).backward(dh)
        assert torch.equal(ps[0].grad, nw.grad)
        for a, b in zip(twin, ps):
            a.grad = b.grad.clone()
        opt.step()
        opt2.step()
        opt.zero_grad()
        assert all(torch.equal(a, b) for a, b in zip(ps, twin))
        assert all(torch.isfinite(p).all() for p in ps)
