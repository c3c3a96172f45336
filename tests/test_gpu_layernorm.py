"""Layer norm forward and backward against plain 64-bit forms, and the backward pass against differences."""
import os
import subprocess
import sys

import pytest
import torch

import training_ref as ref
from paper_2602_17254_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SHAPES = [(1, 1), (1, 2), (3, 7), (5, 31), (2, 32), (4, 33), (17, 128), (9, 255), (65, 256), (33, 257), (7, 1000), (300, 1024), (50, 2187),
          (19, 4096), (11, 5120), (6, 8191), (6, 6144), (5, 8192), (4, 10000), (3, 16384), (2, 20001), (1000, 64), (2500, 9), (700, 513), (400, 2048), (500, 300), (900, 600), (333, 1500), (37, 9001), (90, 16383), (200, 11264)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    assert torch.cuda.is_available()


def _inputs(rows, cols, dtype, seed, pdtype=torch.float32, offset=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(cols, generator=g) * 0.5) + offset * torch.randn(cols, generator=g)).to(dtype)
    dy = torch.randn(rows, cols, generator=g).to(dtype)
    gamma, beta = (1 + 0.3 * torch.randn(cols, generator=g)).to(pdtype), torch.randn(cols, generator=g).to(pdtype)
    return [t.to(DEV) for t in (x, dy, gamma, beta)]


def _check_forward(x, gamma, beta, eps, **kw):
    y, mean, rstd = binding.layernorm_forward_tensor(x, gamma, beta, eps, **kw)
    torch.cuda.synchronize()
    g = gamma.double() if gamma is not None else torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
    b = beta.double() if beta is not None else torch.zeros(x.shape[1], dtype=torch.float64, device=x.device)
    wy, wm, wr = ref.ln_forward(x, g, b, eps)
    ey, em, er = ref.ln_forward_bounds(x, g, b, eps)
    ref.within(y, wy, ref.rounded(ey, wy, x.dtype), "y")
    ref.within(mean, wm, em + ref.U * wm.abs(), "mean")
    ref.within(rstd, wr, er, "rstd")
    return y, mean, rstd


def _check_backward(dy, x, mean, rstd, gamma, **kw):
    dx, dg, db = binding.layernorm_backward_tensor(dy, x, mean, rstd, gamma, **kw)
    torch.cuda.synchronize()
    g = gamma.double() if gamma is not None else torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
    want, bound = ref.ln_backward(dy, x, mean, rstd, g), ref.ln_backward_bounds(dy, x, mean, rstd, g)
    ref.within(dx, want[0], ref.rounded(bound[0], want[0], x.dtype), "dx")
    ref.within(dg, want[1], bound[1] + 1e-45, "dgamma")
    ref.within(db, want[2], bound[2] + 1e-45, "dbeta")
    return dx, dg, db


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward_and_backward(rows, cols, dtype):
    x, dy, gamma, beta = _inputs(rows, cols, dtype, rows * 7 + cols)
    _, mean, rstd = _check_forward(x, gamma, beta, 1e-5)
    _check_backward(dy, x, mean, rstd, gamma)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(20001, 100), (15001, 512), (9001, 1000), (3001, 2187), (2003, 4096), (1500, 5000), (1201, 8192), (701, 12288)])
def test_several_rows_per_cta(rows, cols, dtype):
    """More rows than the resident CTAs take at once, so that rows are on their way while others are reduced."""
    x, dy, gamma, beta = _inputs(rows, cols, dtype, 15)
    _, mean, rstd = _check_forward(x, gamma, beta, 1e-5)
    _check_backward(dy, x, mean, rstd, gamma)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(3, 100), (40, 1024), (5, 3001), (3, 12288)])
def test_parameters_of_the_type_of_x(rows, cols, dtype):
    x, dy, gamma, beta = _inputs(rows, cols, dtype, 3, dtype)
    _, mean, rstd = _check_forward(x, gamma, beta, 1e-6)
    _check_backward(dy, x, mean, rstd, gamma)


@pytest.mark.parametrize("cols", [40, 1024, 4100, 16384])
def test_without_parameters(cols):
    x, dy, gamma, beta = _inputs(21, cols, torch.bfloat16, 4)
    _, mean, rstd = _check_forward(x, None, None, 1e-5)
    _check_backward(dy, x, mean, rstd, None)
    _check_forward(x, gamma, None, 1e-5)
    _check_forward(x, None, beta, 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,pad,shift", [(64, 1, 0), (64, 8, 8), (1000, 24, 1), (4096, 3, 2), (4096, 64, 16), (16384, 5, 3), (20000, 16, 0)])
def test_strides_and_offsets(cols, pad, shift, dtype):
    """Views into wider matrices: row strides and first elements of every alignment; nothing outside the view is written."""
    rows = 23
    x, dy, gamma, beta = _inputs(rows, cols + pad + shift, dtype, 5)
    x, dy = x[:, shift:shift + cols], dy[:, shift:shift + cols]
    frame = torch.full((rows, cols + pad + shift), 7.0, dtype=dtype, device=DEV)
    _, mean, rstd = _check_forward(x, gamma[:cols].clone(), beta[:cols].clone(), 1e-5, out=frame[:, shift:shift + cols])
    assert bool((frame[:, :shift] == 7).all()) and bool((frame[:, shift + cols:] == 7).all())
    frame.fill_(7.0)
    _check_backward(dy, x, mean, rstd, gamma[:cols].clone(), out=frame[:, shift:shift + cols])
    assert bool((frame[:, :shift] == 7).all()) and bool((frame[:, shift + cols:] == 7).all())


def _view(t, pad, shift):
    """t's values as a view into a wider matrix of sevens; and that matrix."""
    frame = torch.full((t.shape[0], t.shape[1] + pad + shift), 7.0, dtype=t.dtype, device=DEV)
    view = frame[:, shift:shift + t.shape[1]]
    view.copy_(t)
    return view, frame


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(23, 9), (23, 33), (50, 100), (23, 257), (23, 1000), (40, 2047), (23, 4096), (23, 4097), (11, 9000), (5, 16384),
                                       (5, 20000), (20001, 60), (3001, 500), (2501, 1000), (1301, 3000), (1201, 4096), (700, 5000)])
@pytest.mark.parametrize("mixed", [0, 1])
def test_every_operand_with_a_stride_and_an_offset_of_its_own(rows, cols, dtype, mixed):
    """Rows that start at different places of a 16-byte vector in x, dy and the results, several rows to a CTA among them; nothing
    outside the results is written.  mixed = 0: only x is a view, the results are contiguous."""
    x, dy, gamma, beta = _inputs(rows, cols, dtype, 17)
    x, _ = _view(x, 3, 1)
    y, yf = _view(torch.zeros_like(dy), 5, 2) if mixed else (None, None)
    dx, dxf = _view(torch.zeros_like(dy), 9, 4) if mixed else (None, None)
    if mixed:
        dy, _ = _view(dy, 2, 0)
    _, mean, rstd = _check_forward(x, gamma, beta, 1e-5, out=y)
    _check_backward(dy, x, mean, rstd, gamma, out=dx)
    for view, frame, shift in ((y, yf, 2), (dx, dxf, 4)) if mixed else ():
        assert bool((frame[:, :shift] == 7).all()) and bool((frame[:, shift + cols:] == 7).all())


def test_parameters_at_odd_addresses():
    x, dy, gamma, beta = _inputs(12, 513, torch.float32, 6)
    x, dy = x[:, :512].contiguous(), dy[:, :512].contiguous()
    _, mean, rstd = _check_forward(x, gamma[1:], beta[1:], 1e-5)
    _check_backward(dy, x, mean, rstd, gamma[1:])


@pytest.mark.parametrize("dtype", TYPES)
def test_large_mean(dtype):
    """The variance is of the differences from the mean, not of squares: a level 100 times the width costs no digits beyond the bound."""
    x, dy, gamma, beta = _inputs(30, 1500, dtype, 8)
    x = (x.float() + 300).to(dtype)
    _, mean, rstd = _check_forward(x, gamma, beta, 1e-5)
    _check_backward(dy, x, mean, rstd, gamma)


def test_constant_and_zero_rows():
    x = torch.zeros(4, 640, device=DEV)
    x[1] = 3.0
    beta = torch.arange(640, device=DEV).float()
    y, mean, rstd = binding.layernorm_forward_tensor(x, None, beta, 1e-5)
    assert torch.equal(y, beta.expand(4, 640)) and torch.equal(mean, x[:, 0])
    assert torch.allclose(rstd, torch.full((4,), 1e-5 ** -0.5, device=DEV), rtol=4 * ref.U)


def test_nan_and_infinity_stay_in_their_rows():
    x, dy, gamma, beta = _inputs(5, 900, torch.bfloat16, 9)
    clean, _, _ = binding.layernorm_forward_tensor(x, gamma, beta)
    x[1, 3], x[3, 899] = float("nan"), float("inf")
    y, mean, rstd = binding.layernorm_forward_tensor(x, gamma, beta)
    keep = [0, 2, 4]
    assert torch.equal(y[keep], clean[keep]) and bool(y[1].isnan().all()) and bool(y[3].isnan().all())
    dx, dg, db = binding.layernorm_backward_tensor(dy, x, mean, rstd, gamma)
    assert bool(dx[keep].isfinite().all()) and bool(dx[1].isnan().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [3, 16, 100, 300, 1000, 2187, 4100, 9001, 12000])
def test_level_times_rstd_beyond_binary32(cols, dtype):
    """Constant rows far from zero: mean rstd overflows, every (x - mean) rstd is 0.  Places behind a row's end must not turn that into NaN."""
    _, dy, gamma, _ = _inputs(11, cols, dtype, 16)
    x = torch.full((11, cols), 2.0 ** 110, device=DEV).to(dtype)
    mean, rstd = torch.full((11,), 2.0 ** 110, device=DEV), torch.full((11,), 2.0 ** 20, device=DEV)
    dx, _, _ = _check_backward(dy, x, mean, rstd, gamma)
    assert bool(dx.isfinite().all())
    wide = torch.full((11, cols + 5), 2.0 ** 110, device=DEV).to(dtype)[:, 2:2 + cols]          # rows off 16-byte boundaries, dx and dy on them
    dx, _, _ = _check_backward(dy, wide, mean, rstd, gamma)
    assert bool(dx.isfinite().all())
    x = torch.full((11, 64), 2.0 ** 120, device=DEV).to(dtype)                                   # and through the forward pass
    _, mean, rstd = _check_forward(x, None, None, 1e-5)
    _check_backward(dy.repeat(1, 22)[:, :64].contiguous(), x, mean, rstd, None)


def test_no_rows():
    x = torch.empty(0, 100, device=DEV)
    y, mean, rstd = binding.layernorm_forward_tensor(x)
    assert y.shape == (0, 100) and mean.numel() == 0
    dx, dg, db = binding.layernorm_backward_tensor(x, x.clone(), mean, rstd)
    assert dx.shape == (0, 100) and bool((dg == 0).all()) and bool((db == 0).all())
    y, _, _ = binding.layernorm_forward_tensor(torch.empty(5, 0, device=DEV))
    assert y.shape == (5, 0)


@pytest.mark.parametrize("cols", [96, 1024, 3000])
def test_backward_against_differences(cols):
    """d/dt of sum(w y(x + t dx)) and of the same in gamma, beta by central differences of the 64-bit form; the step's own error is
    of order t^2 times the third derivative, far below the binary32 error at these widths."""
    x, dy, gamma, beta = _inputs(6, cols, torch.float32, 10)
    eps = 1e-5
    y, mean, rstd = binding.layernorm_forward_tensor(x, gamma, beta, eps)
    dx, dg, db = binding.layernorm_backward_tensor(dy, x, mean, rstd, gamma)
    gen = torch.Generator().manual_seed(1)
    vx, vg, vb = (torch.randn(s, generator=gen, dtype=torch.float64).to(DEV) for s in (x.shape, gamma.shape, beta.shape))
    t = 1e-4

    def value(s):
        return float((ref.ln_forward(x.double() + s * vx, gamma.double() + s * vg, beta.double() + s * vb, eps)[0] * dy.double()).sum())

    slope = (value(t) - value(-t)) / (2 * t)
    parts = [(dx.double() * vx), (dg.double() * vg), (db.double() * vb)]
    got, size = sum(float(p.sum()) for p in parts), sum(float(p.abs().sum()) for p in parts)
    # 1e-5 of the summed magnitudes: binary32 rounding of mean and rstd enters dx once (about 20 U); differences: t^2 = 1e-8
    assert abs(got - slope) <= 1e-5 * size


def test_same_bits_every_time_and_on_other_streams():
    x, dy, gamma, beta = _inputs(3000, 1024, torch.bfloat16, 11)
    y0, mean, rstd = binding.layernorm_forward_tensor(x, gamma, beta)
    b0 = binding.layernorm_backward_tensor(dy, x, mean, rstd, gamma)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            got.append((binding.layernorm_forward_tensor(x, gamma, beta), binding.layernorm_backward_tensor(dy, x, mean, rstd, gamma)))
    torch.cuda.synchronize()
    for f, b in got:
        assert torch.equal(f[0], y0) and all(torch.equal(p, q) for p, q in zip(b, b0))


def test_the_bits_do_not_depend_on_the_widths_of_earlier_calls():
    """Two fresh processes, the same widths in opposite orders; many of them share a CTA size with others."""
    code = """
import hashlib, sys, torch
from paper_2602_17254_b200 import binding
for dtype in (torch.bfloat16, torch.float32):
    for cols in sorted((40, 100, 250, 300, 500, 600, 700, 1000, 1500, 2000, 2187, 3000, 4096), reverse=sys.argv[1] == "down"):
        g = torch.Generator(device="cuda").manual_seed(cols)
        x = torch.randn(4000, cols, device="cuda", generator=g).to(dtype)
        dy = torch.randn(4000, cols, device="cuda", generator=g).to(dtype)
        y, mean, rstd = binding.layernorm_forward_tensor(x)
        parts = (y, *binding.layernorm_backward_tensor(dy, x, mean, rstd))
        print(dtype, cols, hashlib.sha256(b"".join(t.float().cpu().numpy().tobytes() for t in parts)).hexdigest())
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = [subprocess.run([sys.executable, "-c", code, order], cwd=root, capture_output=True, text=True, timeout=300, check=True).stdout.splitlines()
             for order in ("up", "down")]
    assert len(lines[0]) == 26 and sorted(lines[0]) == sorted(lines[1])


def test_inside_a_graph():
    x, dy, gamma, beta = _inputs(200, 777, torch.float32, 12)
    want = binding.layernorm_forward_tensor(x, gamma, beta)
    wantb = binding.layernorm_backward_tensor(dy, x, want[1], want[2], gamma)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = binding.layernorm_forward_tensor(x, gamma, beta)
        gotb = binding.layernorm_backward_tensor(dy, x, got[1], got[2], gamma)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and all(torch.equal(p, q) for p, q in zip(gotb, wantb))


def test_more_than_2_to_the_31_elements():
    """Offsets beyond 32 bits: the last rows of a 2.2-billion-element matrix equal the same rows on their own."""
    rows, cols = 270000, 8192
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    x.fill_(0.5)
    tail, dyt, gamma, beta = _inputs(5, cols, torch.bfloat16, 13)
    x[-5:] = tail
    y, mean, rstd = binding.layernorm_forward_tensor(x, gamma, beta)
    w = binding.layernorm_forward_tensor(tail, gamma, beta)
    assert torch.equal(y[-5:], w[0]) and torch.equal(mean[-5:], w[1]) and torch.equal(rstd[-5:], w[2])
    y.zero_()
    y[-5:] = dyt
    dx, dg, db = binding.layernorm_backward_tensor(y, x, mean, rstd, gamma)
    wb = binding.layernorm_backward_tensor(dyt, tail, w[1], w[2], gamma)
    assert torch.equal(dx[-5:], wb[0]) and bool((dx[:-5] == 0).all())
    bound = ref.ln_backward_bounds(dyt, tail, w[1], w[2], gamma.double())
    ref.within(dg, wb[1].double(), 2 * bound[1], "dgamma")
    ref.within(db, wb[2].double(), 2 * bound[2], "dbeta")
