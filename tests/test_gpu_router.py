"""Expert router with balance loss: forward, loss and gradient against plain 64-bit forms, ties, masks, and differences."""
import math

import pytest
import torch

import training_ref as ref
from paper_2602_17254_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
COEF = 0.02


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    assert torch.cuda.is_available()


def _logits(tokens, experts, dtype, seed, closed=0.0, scale=1.5):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(tokens, experts, generator=g) * scale + 0.5 * torch.randn(experts, generator=g)
    if closed:
        l[torch.rand(tokens, experts, generator=g) < closed] = -math.inf
        l[torch.rand(tokens, generator=g) < 0.1] = -math.inf
    mask = torch.rand(tokens, generator=g) < 0.8
    return l.to(dtype).to(DEV), mask.to(DEV), torch.randn(tokens, 32, generator=g).to(DEV)


def _check(logits, k, mask, normalize, dgates, other=3, **kw):
    """Forward, loss and both backward forms; counts of `other` more ranks enter the backward pass."""
    ids, gates, counts, prob = binding.router_forward_tensor(logits, k, mask, normalize)
    loss = binding.balance_loss_tensor(counts, prob, k, COEF)
    torch.cuda.synchronize()
    hm = None if mask is None else mask.cpu()
    wi, wg, wc, p = ref.router_forward(logits, k, hm, normalize)
    assert torch.equal(ids.cpu(), wi) and torch.equal(counts.cpu().long(), wc)
    tol = ref.probability_bound(logits, p)
    ref.within(gates, wg, wg * (2 * tol + 8 * ref.U) + 1e-37, "gates")
    T = logits.shape[0]
    e_prob = (p * (tol + (T / 8 + 600) * ref.U)).sum(0) + 1e-37 * T
    ref.within(prob, p.sum(0), e_prob, "prob_sum")
    want = ref.router_loss(wc, p.sum(0), k, COEF)
    e_loss = ref.router_loss(wc, e_prob, k, COEF) + (logits.shape[1] / 32 + 24) * ref.U * abs(want)
    assert abs(float(loss) - want) <= e_loss
    total = (counts * (1 + other)).to(torch.int32)
    for dg in (None, dgates[:, :k].contiguous()):
        dl = binding.router_backward_tensor(logits, ids, total, COEF, dg, mask, normalize, **kw)
        torch.cuda.synchronize()
        wd = ref.router_backward(logits, wi, total.cpu(), COEF, None if dg is None else dg.cpu(), hm, normalize)
        # magnitude of what is added up for each value: p (|up| + sum p |up|), with the incoming gradients' size for every chosen one
        E, n = logits.shape[1], max(1, int(total[-1]))
        q = COEF * E / (k * float(n) ** 2) * total[:E].double().cpu()
        live = p.sum(1, keepdim=True) > 0
        size = p * (q + (p * q).sum(1, keepdim=True))
        if dg is not None:
            there = wi >= 0
            g = torch.zeros_like(p).scatter_add_(1, wi.clamp(min=0).long(), torch.where(there, dg.double().cpu().abs(), 0.0))
            w = p
            if normalize:
                sel = torch.zeros_like(p).scatter_add_(1, wi.clamp(min=0).long(), there.double())
                w = p * sel / torch.where(live, (p * sel).sum(1, keepdim=True), 1.0)
            size = size + w * (g + (w * g).sum(1, keepdim=True))
        bound = size * (4 * tol + (E / 32 + 30) * ref.U) + 1e-37
        ref.within(dl, wd, ref.rounded(bound, wd, logits.dtype), "dlogits")
    return ids, gates, counts, prob


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,k", [(1, 1, 1), (1, 2, 1), (3, 2, 2), (27, 9, 2), (64, 8, 8), (50, 16, 4), (33, 31, 3), (40, 32, 32), (61, 33, 5),
                                              (100, 64, 6), (37, 81, 3), (29, 100, 7), (40, 128, 8), (31, 160, 6), (25, 256, 8), (17, 257, 1),
                                              (19, 384, 8), (13, 512, 16), (9, 513, 4), (7, 1000, 10), (5, 1024, 32)])
@pytest.mark.parametrize("normalize", [False, True])
def test_against_plain(tokens, experts, k, dtype, normalize):
    logits, mask, dg = _logits(tokens, experts, dtype, tokens + experts)
    _check(logits, k, None, normalize, dg)
    _check(logits, k, mask, normalize, dg)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,k", [(60, 9, 4), (50, 40, 8), (40, 256, 8), (30, 700, 3)])
@pytest.mark.parametrize("normalize", [False, True])
def test_closed_experts_and_empty_rows(tokens, experts, k, dtype, normalize):
    logits, mask, dg = _logits(tokens, experts, dtype, 5, closed=0.7)
    ids, _, _, _ = _check(logits, k, mask, normalize, dg)
    logits[:] = -math.inf
    ids, gates, counts, prob = _check(logits, k, None, normalize, dg)
    assert bool((ids == -1).all()) and bool((gates == 0).all()) and bool((counts == 0).all()) and bool((prob == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts,k", [(8, 3), (100, 8), (256, 8), (600, 9)])
def test_ties_go_to_the_lowest_index(experts, k, dtype):
    g = torch.Generator().manual_seed(2)
    logits = torch.randint(-1, 2, (50, experts), generator=g).to(dtype).to(DEV)      # three values only, among them zeros
    logits[3] = 0
    logits[4, ::2], logits[4, 1::2] = 0.0, -0.0                                      # equal zeros
    _, mask, dg = _logits(50, experts, dtype, 6)
    ids, _, _, _ = _check(logits, k, mask, True, dg)
    if bool(mask[3]):
        assert ids[3].tolist() == list(range(k))
    ids, _, _, _ = _check(logits, k, None, False, dg)
    assert ids[3].tolist() == list(range(k)) and ids[4].tolist() == list(range(k))


@pytest.mark.parametrize("dtype", TYPES)
def test_masks_of_the_lowest_value(dtype):
    """Closed by the type's lowest number instead of -inf: still open for choice, probability 0."""
    logits, mask, dg = _logits(40, 64, dtype, 7)
    low = torch.finfo(dtype).min
    logits[:, 10:] = low
    logits[0] = low                                                                  # all equal: an even row
    ids, gates, _, _ = _check(logits, 8, None, True, dg)
    assert ids[0].tolist() == list(range(8)) and torch.allclose(gates[0], torch.full((8,), 0.125, device=DEV))
    logits[:, 3:] = low
    ids, gates, _, _ = _check(logits, 8, None, False, dg)
    assert ids[1, 3:].tolist() == [3, 4, 5, 6, 7] and bool((gates[1, 3:] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_subnormals_keep_their_order(dtype):
    tiny = torch.finfo(dtype).smallest_normal
    step = torch.finfo(dtype).tiny * torch.finfo(dtype).eps                          # the smallest subnormal
    logits = torch.zeros(1, 40, dtype=torch.float64)
    logits[0, 5], logits[0, 30], logits[0, 11], logits[0, 2] = step, 2 * step, tiny, -step
    ids, _, _, _ = binding.router_forward_tensor(logits.to(dtype).to(DEV)[:, :32], 32)
    rest = [e for e in range(32) if e not in (11, 30, 5, 2)]
    assert ids[0].tolist() == [11, 30, 5] + rest + [2]


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinity(dtype):
    logits, mask, dg = _logits(6, 40, dtype, 8)
    logits[1, 7] = float("nan")
    logits[2] = float("nan")
    logits[1, 7] = -logits[1, 7]                                                      # a NaN with its sign bit set ranks the same
    logits[3, 5] = float("inf")
    ids, gates, counts, prob = binding.router_forward_tensor(logits, 3)
    assert int(ids[1, 0]) == 7 and ids[2].tolist() == [0, 1, 2] and int(ids[3, 0]) == 5 and int(counts[40]) == 6
    assert bool(gates[[1, 2, 3]].isnan().all()) and bool(gates[[0, 4, 5]].isfinite().all()) and bool(prob.isnan().all())
    hide = torch.tensor([1, 0, 0, 0, 1, 1], device=DEV, dtype=torch.uint8)
    ids, gates, counts, prob = binding.router_forward_tensor(logits, 3, hide)         # NaN in masked tokens goes nowhere
    assert int(counts[40]) == 3 and bool(prob.isfinite().all()) and bool((gates[1:4] == 0).all()) and bool((ids[1:4] == -1).all())
    dl = binding.router_backward_tensor(logits, ids, counts, COEF, dg[:, :3].contiguous(), hide)
    assert bool(dl.isfinite().all()) and bool((dl[1:4] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts,pad,shift", [(9, 3, 1), (64, 8, 0), (64, 8, 3), (256, 1, 1), (256, 64, 8), (500, 12, 4)])
def test_strides_and_offsets(experts, pad, shift, dtype):
    wide, mask, dg = _logits(45, experts + pad + shift, dtype, 9)
    view = wide[:, shift:shift + experts]
    frame = torch.full_like(wide, 7.0)
    _check(view, 2, mask, True, dg, out=frame[:, shift:shift + experts])
    assert bool((frame[:, :shift] == 7).all()) and bool((frame[:, shift + experts:] == 7).all())


def test_ids_outside_the_experts_are_skipped():
    logits, _, dg = _logits(20, 30, torch.float32, 10)
    ids, _, counts, _ = binding.router_forward_tensor(logits, 4)
    odd = ids.clone()
    odd[:, 1], odd[:, 2] = -5, 30
    for normalize in (False, True):
        got = binding.router_backward_tensor(logits, odd, counts, COEF, dg[:, :4].contiguous(), None, normalize)
        want = ref.router_backward(logits, odd.cpu(), counts.cpu(), COEF, dg[:, :4].cpu(), None, normalize)
        assert float((got.double().cpu() - want).abs().max()) <= 1e-5 * float(dg.abs().max())      # about 100 U times the largest summand


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts,k", [(6, 5), (40, 12), (81, 3), (256, 8), (600, 8)])
def test_gates_gradients_without_an_expert_count_for_nothing(experts, k, dtype):
    """NaN and infinities where a token has fewer open experts than choices, or is left out."""
    logits, mask, dg = _logits(60, experts, dtype, 15, closed=1 - 1.5 * k / (experts + k))
    dg = dg[:, :k].contiguous()
    for normalize in (False, True):
        ids, _, counts, _ = binding.router_forward_tensor(logits, k, mask, normalize)
        none = ids < 0
        assert bool((none & (ids[:, :1] >= 0)).any())                                # tokens with some choices but not all
        for bad in (float("nan"), float("inf"), -float("inf")):
            got = binding.router_backward_tensor(logits, ids, counts, COEF, torch.where(none, bad, dg), mask, normalize)
            assert torch.equal(got, binding.router_backward_tensor(logits, ids, counts, COEF, torch.where(none, 0.0, dg), mask, normalize))


@pytest.mark.parametrize("normalize", [False, True])
def test_gradient_against_differences(normalize):
    """Central differences of the 64-bit loss + sum(w gates) with the counts and the choice held fixed."""
    tokens, experts, k = 12, 20, 3
    logits, mask, dg = _logits(tokens, experts, torch.float32, 11)
    dg = dg[:, :k].contiguous()
    ids, _, counts, _ = binding.router_forward_tensor(logits, k, mask, normalize)
    got = binding.router_backward_tensor(logits, ids, counts, COEF, dg, mask, normalize)
    l, m, at = logits.double().cpu(), mask.cpu(), ids.cpu().clamp(min=0).long()

    def value(l):
        p = torch.softmax(l, 1) * m[:, None]
        gates = torch.gather(p, 1, at)
        if normalize:
            gates = gates / gates.sum(1, keepdim=True).clamp(min=1e-300)
        return ref.router_loss(counts.cpu(), p.sum(0), k, COEF) + float((gates * dg.double().cpu() * m[:, None]).sum())

    gen = torch.Generator().manual_seed(1)
    t = 1e-4
    for _ in range(4):
        v = torch.randn(tokens, experts, generator=gen, dtype=torch.float64)
        slope = (value(l + t * v) - value(l - t * v)) / (2 * t)
        part = got.double().cpu() * v
        assert abs(float(part.sum()) - slope) <= 1e-5 * float(part.abs().sum()) + 1e-7     # binary32 and t^2


@pytest.mark.parametrize("experts,k", [(16, 2), (64, 6), (256, 8)])
def test_many_tokens(experts, k):
    """More tokens than the kernels have warps: counts and probability sums against sums over the ids and a 64-bit softmax."""
    tokens = 100003
    g = torch.Generator(device=DEV).manual_seed(3)
    logits = (torch.randn(tokens, experts, device=DEV, generator=g)).to(torch.bfloat16)
    ids, gates, counts, prob = binding.router_forward_tensor(logits, k)
    assert torch.equal(counts[:experts].long(), torch.bincount(ids.flatten().long(), minlength=experts)) and int(counts[experts]) == tokens
    p = torch.softmax(logits.double(), 1)
    value, index = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), index[:, :k])
    bound = (p * ((2 * 30 + experts / 32 + 30 + tokens / 64) * ref.U)).sum(0)
    ref.within(prob, p.sum(0), bound, "prob_sum")
    dl = binding.router_backward_tensor(logits, ids, counts, COEF)
    n = float(tokens)
    q = COEF * experts / (k * n * n) * counts[:experts].double()
    want = p * (q - (p * q).sum(1, keepdim=True))
    bound = p * (q + (p * q).sum(1, keepdim=True)) * (4 * (2 * 30 + experts / 32 + 30)) * ref.U
    ref.within(dl, want, ref.rounded(bound, want, torch.bfloat16), "dlogits")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,k", [(9973, 256, 8), (15013, 256, 3), (30011, 100, 6), (60013, 40, 20), (9973, 500, 1), (150001, 9, 2)])
def test_several_turns_per_warp(tokens, experts, k, dtype):
    """Choices of several turns are written together: more turns than that, and a last write of fewer, give every token the bits it
    has in a call of few tokens (which the tests above hold against the plain form)."""
    logits, mask, dg = _logits(tokens, experts, dtype, 14)
    dg = dg[:, :k].contiguous()
    for m, normalize in ((mask, True), (None, False)):
        ids, gates, counts, _ = binding.router_forward_tensor(logits, k, m, normalize)
        dl = binding.router_backward_tensor(logits, ids, counts, COEF, dg, m, normalize)
        assert torch.equal(counts[:experts].long(), torch.bincount(ids[ids >= 0].long(), minlength=experts))
        assert int(counts[experts]) == (tokens if m is None else int(m.sum()))
        for first in [*range(0, tokens, tokens // 7), tokens - 100]:
            at = slice(first, first + 100)
            part = None if m is None else m[at].contiguous()
            few = binding.router_forward_tensor(logits[at], k, part, normalize)
            assert torch.equal(ids[at], few[0]) and torch.equal(gates[at], few[1])
            assert torch.equal(dl[at], binding.router_backward_tensor(logits[at], few[0], counts, COEF, dg[at].contiguous(), part, normalize))


def test_same_bits_every_time_and_on_other_streams():
    logits, mask, dg = _logits(5000, 128, torch.bfloat16, 12)
    first = binding.router_forward_tensor(logits, 8, mask)
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(4)]:
        with torch.cuda.stream(s):
            got.append(binding.router_forward_tensor(logits, 8, mask))
    torch.cuda.synchronize()
    for r in got:
        assert all(torch.equal(p, q) for p, q in zip(r, first))


def test_no_tokens():
    logits = torch.empty(0, 24, device=DEV)
    ids, gates, counts, prob = binding.router_forward_tensor(logits, 2)
    assert ids.shape == (0, 2) and bool((counts == 0).all()) and bool((prob == 0).all())
    assert float(binding.balance_loss_tensor(counts, prob, 2, COEF)) == 0
    assert binding.router_backward_tensor(logits, ids, counts, COEF).shape == (0, 24)


def test_counts_of_all_ranks_through_the_allreduce():
    """Ranks with tokens of their own: the summed counts and probability sums give the loss and gradients of the whole batch."""
    n, tokens, experts, k = 9, 40, 27, 3
    plan = binding.Plan((n,), binding.LATENCY_OPTIMAL)
    logits, _, dg = _logits(n * tokens, experts, torch.float32, 13)
    counts = torch.zeros(n, 32, dtype=torch.int32, device=DEV)
    probs = torch.zeros(n, 32, dtype=torch.float32, device=DEV)
    ids = []
    for r in range(n):
        i, _, c, p = binding.router_forward_tensor(logits[r * tokens:(r + 1) * tokens], k)
        ids.append(i)
        counts[r, :experts + 1], probs[r, :experts] = c, p
    binding.allreduce_tensor(plan, counts)
    binding.allreduce_tensor(plan, probs)
    wi, _, wc, wp = binding.router_forward_tensor(logits, k)
    assert torch.equal(torch.cat(ids), wi) and all(torch.equal(counts[r, :experts + 1], wc) for r in range(n))
    assert torch.allclose(probs[:, :experts], wp.expand(n, -1), rtol=400 * ref.U, atol=0)       # two orders of 360 additions
    whole = binding.router_backward_tensor(logits, wi, wc, COEF)
    for r in range(n):
        part = binding.router_backward_tensor(logits[r * tokens:(r + 1) * tokens], ids[r], counts[r, :experts + 1].contiguous(), COEF)
        assert torch.equal(part, whole[r * tokens:(r + 1) * tokens])
