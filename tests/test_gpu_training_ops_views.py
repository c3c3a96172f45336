"""Training operators whose operands are column slices of one buffer: accepted where no element is shared, with the bits of a call on
buffers of their own; and refused where one is."""
import pytest
import torch

from paper_2602_17254_b200 import binding as B
from paper_2602_17254_b200 import build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    assert torch.cuda.is_available()


def _slices(rows, cols, n, dtype, seed, gap=0):
    """n matrices side by side, `gap` columns between them; and the buffer."""
    g = torch.Generator().manual_seed(seed)
    wide = torch.randn(rows, n * (cols + gap), generator=g).to(dtype).to(DEV)
    return wide, [wide[:, i * (cols + gap):i * (cols + gap) + cols] for i in range(n)]


def _refused(call):
    before = B.launch_count()
    with pytest.raises(B.TrivanceError) as e:
        call()
    assert e.value.status == B.ERR_INVALID_ARG and B.launch_count() == before


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,gap", [(40, 64, 0), (33, 1000, 8), (700, 97, 3), (21, 5000, 0), (5, 20000, 1)])
def test_layernorm(rows, cols, gap, dtype):
    wide, (dy, x, a, b) = _slices(rows, cols, 4, dtype, 1, gap)
    y0, mean, rstd = B.layernorm_forward_tensor(x.clone())
    dx0, dg0, db0 = B.layernorm_backward_tensor(dy.clone(), x.clone(), mean, rstd)
    old = wide.clone()
    y, _, _ = B.layernorm_forward_tensor(x, out=a)
    dx, dg, db = B.layernorm_backward_tensor(dy, x, mean, rstd, out=b)
    assert torch.allclose(y.float(), y0.float(), rtol=2 ** -7, atol=1e-5) and torch.allclose(dx.float(), dx0.float(), rtol=2 ** -6, atol=1e-4)
    assert torch.allclose(dg, dg0, rtol=1e-4, atol=1e-3) and torch.allclose(db, db0, rtol=1e-4, atol=1e-3)
    a.copy_(old[:, 2 * (cols + gap):2 * (cols + gap) + cols])
    b.copy_(old[:, 3 * (cols + gap):3 * (cols + gap) + cols])
    assert torch.equal(wide, old)                                           # nothing but the outputs was written
    for one in (x, wide[:, cols + gap + 1:2 * cols + gap + 1]):             # the same columns, and all but one of them
        _refused(lambda: B.layernorm_forward_tensor(x, out=one))
        _refused(lambda: B.layernorm_backward_tensor(dy, x, mean, rstd, out=one))
    if rows > 1:
        _refused(lambda: B.layernorm_forward_tensor(x[1:], out=x[:-1]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts,gap", [(9, 0), (64, 0), (81, 2), (256, 16)])
def test_router_backward(experts, gap, dtype):
    wide, (logits, out) = _slices(300, experts, 2, dtype, 2, gap)
    ids, gates, counts, _ = B.router_forward_tensor(logits, 3)
    want = B.router_backward_tensor(logits, ids, counts, 0.1, gates)
    old = wide.clone()
    assert torch.equal(B.router_backward_tensor(logits, ids, counts, 0.1, gates, out=out), want)
    out.copy_(old[:, experts + gap:2 * experts + gap])
    assert torch.equal(wide, old)
    _refused(lambda: B.router_backward_tensor(logits, ids, counts, 0.1, gates, out=logits))
    _refused(lambda: B.router_backward_tensor(logits, ids, counts, 0.1, gates, out=wide[:, 1:1 + experts]))


@pytest.mark.parametrize("rows,cols", [(30, 60), (200, 136), (300, 500)])
def test_orthogonalize(rows, cols):
    wide, (g, out) = _slices(2 * rows, cols, 2, torch.bfloat16, 3)
    want = B.orthogonalize_tensor(g[:rows].clone())
    old = wide.clone()
    assert torch.equal(B.orthogonalize_tensor(g[:rows], out=out[:rows]), want)
    pair = (g.unflatten(0, (2, rows)), out.unflatten(0, (2, rows)))         # a batch of two, one behind the other
    both = B.orthogonalize_tensor(pair[0].clone())
    assert torch.equal(B.orthogonalize_tensor(pair[0], out=pair[1]), both)
    out.copy_(old[:, cols:])
    assert torch.equal(wide, old)
    _refused(lambda: B.orthogonalize_tensor(g[:rows], out=g[:rows]))
    _refused(lambda: B.orthogonalize_tensor(g[:rows], out=wide[:rows, 1:1 + cols]))
