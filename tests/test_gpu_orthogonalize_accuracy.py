"""Accuracy of the orthogonalisation as the header states it: numbers that do not come from the implementation's formats, on the
spectra where low precision shows, weak directions that grow beside strong ones, and on steps that amplify every rounding."""
import math

import pytest
import torch

import training_ref as ref
from paper_2602_17254_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# five steps whose polynomials are steep where singular values pass (up to 12 times on the way), with the largest gain first
STEEP = [(8.287, -23.60, 17.30), (4.107, -2.948, 0.545), (3.949, -2.909, 0.552), (3.318, -2.488, 0.510), (2.301, -1.669, 0.419)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    assert torch.cuda.is_available()


def _strong(rows, cols, weak, seed=0):
    """One singular value 1, the others `weak`, in random directions."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    m, n = sorted((rows, cols))
    u, _ = torch.linalg.qr(torch.randn(m, m, generator=g, dtype=torch.float64, device=DEV))
    v, _ = torch.linalg.qr(torch.randn(n, m, generator=g, dtype=torch.float64, device=DEV))
    s = torch.full((m,), weak, dtype=torch.float64, device=DEV)
    s[0] = 1
    x = ((u * s) @ v.T).float()
    return x if rows <= cols else x.T.contiguous()


def _noise(rows, cols, level=0.0, width=1.0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (level + width * torch.randn(rows, cols, generator=g, dtype=torch.float64, device=DEV)).float()


def _check(g, share, coefficients=None):
    """2-norm of the error at most `share` of the result's, beside the rounding of the exact result to bfloat16 (independent of it)."""
    got = binding.orthogonalize_tensor(g, steps=5, coefficients=coefficients).double()
    want = ref.orthogonalize(g, coefficients=coefficients)
    error, size, rounding = (float(t.norm()) for t in (got - want, want, want.bfloat16().double() - want))
    assert error <= math.hypot(rounding, share * size), "error %.4f %%, rounding %.4f %%" % (100 * error / size, 100 * rounding / size)


ON_CHIP = [(16, 1024), (27, 81), (64, 1024), (128, 1000), (128, 512), (40, 60), (5, 2049), (1000, 128), (81, 27), (100, 200), (20, 4000), (65, 64)]


@pytest.mark.parametrize("weak", [1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("rows,cols", ON_CHIP)
def test_one_strong_direction_on_chip(rows, cols, weak):
    _check(_strong(rows, cols, weak), 1e-3)


@pytest.mark.parametrize("rows,cols", ON_CHIP)
def test_a_level_over_small_noise_on_chip(rows, cols):
    _check(_noise(rows, cols, 1.0, 1e-3), 1e-3)
    _check(_noise(rows, cols, 1.0, 1e-4, 1), 1e-3)
    _check(_noise(rows, cols, 1.0, 2.0 ** -6, 2).bfloat16(), 1e-3)


@pytest.mark.parametrize("seed", [0, 5])
@pytest.mark.parametrize("rows,cols", ON_CHIP)
def test_steep_steps_on_chip(rows, cols, seed):
    _check(_noise(rows, cols, seed=seed), 1e-3, STEEP)
    _check(_strong(rows, cols, 1e-3, seed), 1e-3, STEEP)


TILED = [(129, 129), (150, 200), (200, 300), (300, 1000), (1000, 300), (512, 512), (1024, 600), (700, 1100), (2300, 2100)]
THIN = [(3, 9000), (16, 8192), (40, 5000), (9001, 100)]                    # a side of at most 128, the other too long to stay on chip


@pytest.mark.parametrize("weak", [1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("rows,cols", TILED + THIN)
def test_one_strong_direction_tiled(rows, cols, weak):
    _check(_strong(rows, cols, weak), 1e-3)


@pytest.mark.parametrize("rows,cols", TILED + THIN)
def test_a_level_over_small_noise_tiled(rows, cols):
    """Roundings of A and B beside the diagonal, which the strong direction fills evenly."""
    _check(_noise(rows, cols, 1.0, 1e-3), 2.5e-3)
    _check(_noise(rows, cols, 1.0, 1e-4, 1), 2.5e-3)


@pytest.mark.parametrize("rows,cols", TILED)
def test_steep_steps_tiled(rows, cols):
    """Every rounding to binary16 counts up to 40 times."""
    _check(_noise(rows, cols), 7.5e-3, STEEP)
    _check(_strong(rows, cols, 1e-3), 7.5e-3, STEEP)


def test_a_thousandth_at_300_by_1000():
    for seed in (0, 1):
        for weak in (1e-3, 1e-4):
            _check(_strong(300, 1000, weak, seed), 1e-3)
        _check(_noise(300, 1000, 1.0, 1e-3, seed), 1e-3)
        _check(_noise(300, 1000, seed=seed), 1e-3, STEEP)


def test_one_strong_direction_in_a_batch():
    for rows, cols in ((48, 300), (160, 220)):
        g = torch.stack([_strong(rows, cols, 1e-4, s) for s in range(5)])
        got = binding.orthogonalize_tensor(g).double()
        for one, o in zip(g, got):
            want = ref.orthogonalize(one)
            error, size, rounding = (float(t.norm()) for t in (o - want, want, want.bfloat16().double() - want))
            assert error <= math.hypot(rounding, 1e-3 * size)


def test_many_thin_matrices():
    """So many that CTA pairs take them."""
    g = torch.stack([_strong(100, 4200, 1e-4, s % 3) if s % 2 else _noise(100, 4200, 1.0, 1e-3, s % 3) for s in range(40)])
    got = binding.orthogonalize_tensor(g).double()
    for s in range(40):
        want = ref.orthogonalize(g[s])
        error, size, rounding = (float(t.norm()) for t in (got[s] - want, want, want.bfloat16().double() - want))
        assert error <= math.hypot(rounding, 1e-3 * size)
