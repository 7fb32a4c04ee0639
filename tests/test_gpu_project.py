"""Rows in 8 bits and their products against the definition (oracle/few_bits.py).

Codes are whole numbers and have to be equal.  Sums of codes are exact; a result is off by the roundings of a scale, of the sum as float32, of two products and
of the bias: 4 w of the product and w of the result, w = 2^-24, and by that of its type.
"""
import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import few_bits as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
W = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def up16(n):
    return -(-n // 16) * 16


def make(rows, cols, outs, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)
    w = torch.zeros(outs, up16(cols), dtype=torch.int8)
    w[:, :cols] = torch.randint(-128, 128, (outs, cols), generator=g)
    return x, w, torch.rand(outs, generator=g) * 0.01 + 1e-4, torch.randn(outs, generator=g)


def want_of(codes, scales, w, ws, bias):
    return (codes.astype(np.float64) @ f64(w)[:, :codes.shape[1]].T) * scales[:, None] * f64(ws)[None], 0.0 if bias is None else f64(bias)[None]


def check(got, codes, scales, w, ws, bias, dtype):
    product, b = want_of(codes, scales, w, ws, bias)
    want = product + b
    bound = 4 * W * np.abs(product) + (W + torch.finfo(dtype).eps / 2) * np.abs(want) + 1e-37
    got = f64(got)
    over = np.abs(got - want) / bound
    assert got.shape == want.shape and np.all(np.isfinite(got)) and over.max(initial=0) <= 1, f"{over.max():.3g} at {np.unravel_index(over.argmax(), over.shape)}"


SHAPES = [(1, 1, 1), (1, 4096, 257), (3, 16, 17), (16, 130, 16), (17, 64, 100), (33, 1000, 33), (64, 2048, 512), (65, 129, 130), (128, 256, 128), (200, 80, 300), (300, 1500, 260), (513, 17, 65),
          (129, 8192, 40), (2, 65536, 3), (1030, 520, 1030)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols,outs", SHAPES)
def test_products(rows, cols, outs, dtype):
    """One row to many, sizes that fill no tile and no 16 bytes."""
    x, w, ws, bias = make(rows, cols, outs, dtype, seed=rows + cols)
    codes, scales = oracle.quantize_rows(f64(x))
    got_codes, got_scales = idf.quantize_rows(x.to(DEV))
    assert got_codes.shape == (rows, up16(cols)) and np.array_equal(got_codes[:, :cols].cpu().numpy(), codes) and not got_codes[:, cols:].any()
    assert np.all(np.abs(f64(got_scales) - scales) <= W * scales)
    for b in (None, bias):
        got = idf.project_rows(x.to(DEV), w.to(DEV), ws.to(DEV), bias=None if b is None else b.to(DEV))
        assert got.dtype == dtype
        check(got, codes, f64(got_scales), w, ws, b, dtype)


@pytest.mark.parametrize("rows", [1, 5, 16, 40, 64, 100, 130, 260, 700, 2100])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_codes_come_from_the_caller(rows, dtype):
    """Codes and scales of the caller's own give the same bits as rows that are taken to them on the way, in any precision of the result."""
    x, w, ws, bias = make(rows, 272, 150, torch.float32, seed=rows)
    codes, scales = idf.quantize_rows(x.to(DEV))
    got = idf.project_rows(codes, w.to(DEV), ws.to(DEV), bias=bias.to(DEV), x_scales=scales, dtype=dtype)
    assert got.dtype == dtype
    check(got, f64(codes).astype(np.int64), f64(scales), w, ws, bias, dtype)
    if dtype == torch.float32:
        assert torch.equal(got, idf.project_rows(x.to(DEV), w.to(DEV), ws.to(DEV), bias=bias.to(DEV)))
    # rows among other columns, from a multiple of 16 on, and from another place, which is copied
    wide = torch.zeros(rows, 400, dtype=torch.int8, device=DEV)
    for at in (16, 5):
        wide[:, at:at + 272] = codes
        assert torch.equal(idf.project_rows(wide[:, at:at + 272], w.to(DEV), ws.to(DEV), bias=bias.to(DEV), x_scales=scales, dtype=dtype), got)


def test_the_largest_sums():
    """All codes at their ends: sums of 65536 products come close to 2^31 and are still exact."""
    codes = torch.full((3, 65536), -128, dtype=torch.int8, device=DEV)
    w = torch.full((20, 65536), -127, dtype=torch.int8, device=DEV)
    w[1] = 127
    one = torch.ones(20, device=DEV)
    got = idf.project_rows(codes, w, one, x_scales=one[:3].contiguous(), dtype=torch.float32)
    total = 65536 * 128 * 127
    assert got[0, 0].item() == float(np.float32(total)) and got[2, 1].item() == -float(np.float32(total))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_middles_between_codes(dtype):
    """Values whose quotient is a middle exactly go to the even code; neighbours in the type to the nearer one."""
    x = torch.zeros(6, 64, dtype=torch.float32)
    for r, most in enumerate((127.0, 254.0, 63.5, 1.0, 3.0, 7.0)):
        x[r, 0] = most
        middles = (torch.arange(0, 30) + 0.5) * most / 127
        x[r, 1:31] = middles
        x[r, 31:61] = -torch.nextafter(middles, torch.full_like(middles, 1e9 if r % 2 else 0.0))
    x = x.to(dtype)
    codes, scales = oracle.quantize_rows(f64(x))
    got, _ = idf.quantize_rows(x.to(DEV))
    assert np.array_equal(got.cpu().numpy(), codes)


@pytest.mark.parametrize("cols", [40, 3000, 20000])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_rows_of_zeros_and_what_is_not_finite(dtype, cols):
    """A row of zeros gives the bias; one with an infinite value or none that is a number gives no number; the others know nothing of it.  Very small
    and very large rows."""
    x, w, ws, bias = make(6, cols, 33, torch.float32, seed=1)
    x[1] = 0
    x[2, cols - 1], x[3, cols // 2] = float("inf"), float("nan")
    x[4] *= 1e-36
    x[5] *= 1e34
    x = x.to(dtype)
    got = idf.project_rows(x.to(DEV), w.to(DEV), ws.to(DEV), bias=bias.to(DEV), dtype=torch.float32)
    codes, scales = oracle.quantize_rows(f64(x))
    assert np.array_equal(idf.quantize_rows(x.to(DEV))[0][:, :cols].cpu().numpy(), codes)
    assert torch.equal(got[1].cpu(), bias) and torch.isnan(got[2:4]).all()
    keep = [0, 1, 5]
    check(got[keep], codes[keep], scales[keep], w, ws, bias, torch.float32)
    assert torch.equal(got[4].cpu(), bias) or (got[4].cpu() - bias).abs().max() <= 1e-6


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_strides(dtype):
    """x among other columns from an odd place on, transposed, repeated rows; an out among other columns, which stay."""
    x, w, ws, bias = make(70, 200, 90, dtype, seed=2)
    x, w, ws = x.to(DEV), w.to(DEV), ws.to(DEV)
    want = idf.project_rows(x, w, ws)
    for at in (0, 1, 8):
        wide = torch.full((70, 240), 5.0, dtype=dtype, device=DEV)
        wide[:, at:at + 200] = x
        to = torch.full((70, 111), 7.0, dtype=dtype, device=DEV)
        got = idf.project_rows(wide[:, at:at + 200], w, ws, out=to[:, at:at + 90])
        assert torch.equal(got, want) and torch.all(to[:, :at] == 7.0) and torch.all(to[:, at + 90:] == 7.0)
    assert torch.equal(idf.project_rows(x.t().contiguous().t(), w, ws), want)
    assert torch.equal(idf.project_rows(x[:1].expand(70, 200), w, ws), want[:1].expand(70, 90))
    assert idf.project_rows(x[:0], w, ws).shape == (0, 90)


def test_rows_do_not_depend_on_their_number():
    """Integer sums: a row gives the same bits whichever kernel its call takes."""
    x, w, ws, bias = (t.to(DEV) for t in make(2000, 320, 700, torch.bfloat16, seed=3))
    want = idf.project_rows(x, w, ws, bias=bias)
    for n in (1, 16, 17, 48, 64, 65, 128, 200, 600):
        assert torch.equal(idf.project_rows(x[:n], w, ws, bias=bias), want[:n]), n


def test_recorded_into_a_graph_and_on_other_streams():
    x, w, ws, bias = (t.to(DEV) for t in make(40, 512, 256, torch.bfloat16, seed=4))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        idf.project_rows(x, w, ws, bias=bias)
    torch.cuda.current_stream().wait_stream(side)
    still = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = idf.project_rows(still, w, ws, bias=bias)
    for i in range(4):
        still.copy_(x * (i + 1) + i)
        want = idf.project_rows(still, w, ws, bias=bias)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals_of_tensors():
    x, w, ws, bias = (t.to(DEV) for t in make(4, 64, 32, torch.float32))
    for call in (lambda: idf.project_rows(x, w[:, :48].contiguous(), ws), lambda: idf.project_rows(x, w, ws[:5]), lambda: idf.project_rows(x, w, ws, bias=bias.double()), lambda: idf.project_rows(x, w, ws, x_scales=ws[:4]),
                 lambda: idf.project_rows(w[:4], w, ws), lambda: idf.project_rows(w[:4], w, ws, x_scales=ws[:4]), lambda: idf.project_rows(x, w.float(), ws), lambda: idf.project_rows(x, w, ws, out=torch.empty(4, 31, device=DEV)),
                 lambda: idf.project_rows(x, w, ws, dtype=torch.bfloat16, out=torch.empty(4, 32, device=DEV)), lambda: idf.quantize_rows(x, codes=w), lambda: idf.project_rows(x.requires_grad_(), w, ws)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(idf.IdfError):
        idf.project_rows(x.detach().half(), w, ws)


@pytest.mark.parametrize("rows,cols", [(2047, 513), (2049, 2049), (2050, 4096), (2051, 4097), (2049, 100), (3, 513), (2047, 4096)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_rows_that_share_a_workgroup(rows, cols, dtype):
    """One, two and four rows to a workgroup, the last one half empty: each has a scale of its own, beside rows of zeros and rows that are not finite."""
    x, *_ = make(rows, cols, 1, dtype, seed=rows)
    x[1], x[2, cols - 1] = 0, float("inf")
    codes, scales = idf.quantize_rows(x.to(DEV))
    fine = torch.arange(rows) != 2
    want, want_scales = oracle.quantize_rows(f64(x)[fine])
    assert np.array_equal(f64(codes)[fine][:, :cols], want) and not codes[:, cols:].any()
    assert np.all(np.abs(f64(scales)[fine] - want_scales) <= W * want_scales) and torch.isnan(scales[2])
