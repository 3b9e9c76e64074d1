"""Distillation from a teacher's top logits on the GPU against a plain implementation in 64 bits, row by row.

Tolerances, derived from the operations: with u = 2^-23, an exponent x carries three roundings, 3 |x| u; a power 2 u; the sum of
powers one rounding per addition (vocabulary / 256 in sequence at most, then a tree). So a student's probability is off by
r = (8 + 6 X + vocabulary / 256) u relatively, X the largest |x| whose power does not underflow, and a logarithm of a
probability by as much absolutely with the |x| of the listed entries, which no underflow bounds; a teacher's probability by
r too, with the size of t / tau and lse as X. A term q (log q - log p) is then off by r q (1 + |log q - log p|), the class of
entries left out by r (1 + |log q_rest - log p_rest|) as q_rest is 1 - sum q, and a gradient entry by
r (p (Q + (q_rest + sum q) / p_rest) + q) w / tau (sum q, as q_rest is 1 - sum q and a binary32 sum near 1 is no finer), plus
one rounding to the logits' type.
"""
import math

import numpy as np
import pytest
import torch

from paper_2309_01507_b200 import lpmm

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -126, BF16: 2.0 ** -126, F16: 2.0 ** -24}
U = 2.0 ** -23


def _lse(v):
    m = v.max(initial=-np.inf)
    return m + math.log(np.exp(v - m).sum()) if np.isfinite(m) else -np.inf


def _plain_row(z, ids, t, tau, lse, w):
    """(loss, gradient, size of the gradient's terms, tolerance r) of one row, in 64 bits, from the definition."""
    V, tau = len(z), float(np.float32(tau))       # the temperature is a binary32 argument
    if w == 0:
        return 0.0, np.zeros(V), np.zeros(V), (0.0, 0.0)
    ok = (ids >= 0) & (ids < V) & (t > -np.inf)
    any_id = (ids >= 0) & (ids < V)
    x = z / tau
    top = x.max() if np.isfinite(x.max()) else 0.0
    logZ = _lse(x - top)                   # relative to the largest, which may be the type's lowest value
    logp = x - top - logZ if logZ > -np.inf else np.full(V, -np.inf)
    p = np.exp(logp)
    q = np.zeros(V)
    listed = np.zeros(V, bool)
    listed[ids[any_id]] = True
    tt = t[ok] / tau
    logq = tt - (lse if lse is not None else _lse(tt))
    qk = np.exp(logq)
    loss = 0.0
    for i, lq, qv in zip(ids[ok], logq, qk):
        q[i] += qv
        if qv > 0:
            loss += qv * (lq - logp[i])
    rest = max(0.0, 1 - qk.sum()) if lse is not None and not listed.all() else 0.0
    p_rest = p[~listed].sum()
    if rest > 0:
        loss += rest * (math.log(rest) - (math.log(p_rest) if p_rest > 0 else -np.inf))
    Q = qk.sum() + rest if lse is not None else (1.0 if len(qk) else 0.0)
    ratio = rest / p_rest if p_rest > 0 else 0.0
    grad = np.where(listed, p * Q - q, p * (Q - ratio)) * w / tau
    size = np.where(listed, p * Q + q, p * (Q + ratio + (qk.sum() / p_rest if rest > 0 and p_rest > 0 else 0))) * abs(w) / tau
    X = min(np.abs(x[np.isfinite(x)] - top).max(initial=0.0) * 1.4427, 150.0)
    live = qk > 0
    xl = [0.0, abs(logZ) if np.isfinite(logZ) else 0.0, abs(lse) if lse is not None else 0.0]
    xl += list(np.abs(tt[live])) if lse is not None else list(np.abs(logq[live]))
    xl += [abs(v - top) for v in x[ids[ok][live]] if np.isfinite(v)]
    r = (8 + 6 * max(X, 1.4427 * max(xl)) + V / 256) * U
    D = np.abs(logq[live] - logp[ids[ok][live]])
    terms = (qk[live] * (1 + np.where(np.isfinite(D), D, 0))).sum()
    if rest > 0 and p_rest > 0:
        terms += 1 + abs(math.log(rest / p_rest))
    return w * loss, grad, size, (r, abs(w) * (r * terms + U * abs(loss)) if np.isfinite(loss) else 0.0)


def _check(logits, ids, t, tau=1.0, lse=None, weights=None, rows=None, **kw):
    loss, grad = lpmm.distill_grad(logits, ids, t, temperature=tau, teacher_lse=lse, weights=weights, **kw)
    alone = lpmm.distill_loss(logits, ids, t, temperature=tau, teacher_lse=lse, weights=weights)
    assert torch.equal(alone, loss) or torch.equal(alone.isnan(), loss.isnan())
    assert loss.dtype == F32 and grad.dtype == logits.dtype
    z, i, tt = logits.double().cpu().numpy(), ids.cpu().numpy(), t.double().cpu().numpy()
    lo, g = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    L = lse.double().cpu().numpy() if lse is not None else None
    W = weights.double().cpu().numpy() if weights is not None else None
    for r in (range(len(z)) if rows is None else rows):
        w = 1.0 if W is None else W[r]
        want, wg, size, (rel, tol) = _plain_row(z[r], i[r], tt[r], tau, None if L is None else L[r], w)
        if np.isfinite(want):
            assert abs(lo[r] - want) <= tol + 1e-37, (r, lo[r], want, tol)
        else:
            assert lo[r] == want, (r, lo[r], want)
        rel *= 2      # the sums that a probability is divided by, and the probability itself
        bound = rel * size + (ROUND[grad.dtype] * (1 + rel)) * np.abs(wg) + TINY[grad.dtype] * max(1.0, abs(w) / tau)
        bad = np.abs(g[r] - wg) > bound
        assert not bad.any(), (r, np.flatnonzero(bad)[:5], g[r][bad][:5], wg[bad][:5], bound[bad][:5])
    return loss, grad


def _case(tokens, vocab, top, dtype=F32, seed=0, tau=1.0, tail=False, spread=2.5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn(tokens, vocab, generator=g, device="cuda") * spread
    t = z + torch.randn(tokens, vocab, generator=g, device="cuda")
    v, ids = torch.topk(t, top, dim=1)
    lse = torch.logsumexp(t / tau, dim=1) if tail else None
    return z.to(dtype), ids, v, lse


@pytest.mark.parametrize("tail", [False, True], ids=["renormalized", "tail"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,vocab,top", [(1, 1, 1), (1, 2, 1), (3, 7, 7), (2, 8, 3), (5, 33, 4), (4, 255, 16), (2, 1000, 1), (3, 4097, 64), (2, 5003, 1024), (1, 40001, 33)])
def test_shapes(tokens, vocab, top, dtype, tail):
    for tau in (1.0, 3.5):
        z, ids, t, lse = _case(tokens, vocab, top, dtype, vocab, tau, tail)
        _check(z, ids, t, tau, lse)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,vocab", [(1, 32000), (300, 3001), (1, 131073), (2, 262144), (40, 50265), (700, 32000), (1200, 1001)])
def test_sizes_from_one_row_to_many(tokens, vocab, dtype):
    z, ids, t, lse = _case(tokens, vocab, 50, dtype, tokens, 2.0, True)
    w = torch.rand(tokens, device="cuda")
    _check(z, ids, t, 2.0, lse, w, rows=sorted({0, tokens // 2, tokens - 1, min(5, tokens - 1)}))


@pytest.mark.parametrize("vocab,top", [(50000, 1024), (52900, 1024), (53500, 700), (17300, 1024), (262144, 1024)])
def test_the_longest_rows_that_fit_with_the_longest_lists(vocab, top):
    for dtype in (F32, BF16):
        for tokens in (2, 160):
            z, ids, t, lse = _case(tokens, vocab, top, dtype, vocab, 1.0, True)
            _check(z, ids, t, 1.0, lse, rows=[0, tokens - 1])


def test_rows_without_a_weight_anywhere():
    z, ids, t, lse = _case(1500, 700, 5, BF16, 77, 1.0, True)
    for share in (0.0, 0.02, 0.5, 0.97, 1.0):
        w = (torch.rand(1500, generator=torch.Generator("cuda").manual_seed(3), device="cuda") >= share).float() * 0.25
        w[0], w[-1] = float(share == 0.5), float(share == 0.97)
        z2 = torch.where(w[:, None] == 0, float("nan"), z.float()).to(BF16)      # rows that are not to be read
        loss, grad = _check(z2, ids, t, 1.0, lse, w, rows=w.nonzero()[:, 0][:: max(1, int(w.count_nonzero()) // 40)].tolist())
        assert (loss[w == 0] == 0).all() and (grad[w == 0] == 0).all() and torch.isfinite(loss).all()
        base, gbase = lpmm.distill_grad(z, ids, t, teacher_lse=lse)
        assert torch.equal(loss, torch.where(w == 0, 0.0, base * w))            # weights only scale


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_types_of_ids_and_teacher_strides_and_in_place(dtype):
    z, ids, t, lse = _case(6, 999, 20, dtype, 3, 1.0, True)
    want = _check(z, ids, t, 1.0, lse)
    got = lpmm.distill_grad(z, ids.int(), t, teacher_lse=lse)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for td in (BF16, F16):
        _check(z, ids, t.to(td), 1.0, lse)
    for pitch, off in ((1000, 0), (1008, 3), (1024, 8), (1001, 2)):      # rows at every alignment, NaN between them
        buf = torch.full((6, pitch + off), float("nan"), device="cuda", dtype=dtype)
        view = buf[:, off:off + 999]
        view.copy_(z)
        out = torch.full((6, pitch + 11), 3.0, device="cuda", dtype=dtype)
        loss, grad = _check(view, ids, t, 1.0, lse, out=out[:, 5:5 + 999])
        assert (out[:, :5] == 3).all() and (out[:, 5 + 999:] == 3).all()
        loss2, grad2 = lpmm.distill_grad(view, ids, t, teacher_lse=lse, out=view)      # the gradient replaces the logits
        assert torch.equal(loss2, loss) and torch.equal(grad2, grad) and grad2.data_ptr() == view.data_ptr()
        assert buf[:, :off].isnan().all() and buf[:, off + 999:].isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [70, 3000, 140001])
def test_masked_rows_and_entries(dtype, vocab):
    inf, low = float("inf"), torch.finfo(dtype).min
    z, ids, t, lse = _case(12, vocab, 6, dtype, 8, 1.5, True)
    z[0, vocab // 2:] = low                      # masked with the type's lowest value
    z[1, vocab // 2:] = -inf
    z[2] = low                                   # everything masked: uniform
    z[3] = -inf                                  # nothing left: p = 0
    z[4] = float("nan")                          # a row that does not count holds anything
    ids[5, 2:] = -1                              # fewer entries than columns
    ids[6] = -1                                  # none at all
    ids[7, 3] = vocab                            # outside the vocabulary: no entry
    ids[8, 0] = torch.iinfo(torch.int64).max
    t[9, 1] = -inf                               # an entry without probability
    t[10] = -inf
    z[11, ids[11, 0]] = -inf                     # the teacher's best entry is impossible for the student
    w = torch.linspace(0.5, 2.0, 12, device="cuda")
    w[4] = 0
    keep = [r for r in range(12) if r != 4]
    for l in (None, lse):
        loss, grad = _check(z, ids, t, 1.5, l, w, rows=keep)
        assert loss[4] == 0 and (grad[4] == 0).all()
        assert torch.isfinite(grad.float()).all()
    loss, grad = lpmm.distill_grad(z, ids, t, temperature=1.5, weights=w)
    assert loss[6] == 0 and (grad[6] == 0).all() and loss[10] == 0 and (grad[10] == 0).all()
    assert loss[11] == inf and loss[3] == inf
    z[0, 1], z[1, 1] = float("nan"), inf
    loss, grad = lpmm.distill_grad(z, ids, t, temperature=1.5, weights=w)
    assert loss[:2].isnan().all() and grad[:2].isnan().any(1).all() and not loss[2:3].isnan().any() and not grad[2:].isnan().any()
    w[:] = 0
    loss, grad = lpmm.distill_grad(z, ids, t, temperature=1.5, weights=w)
    assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("tail", [False, True], ids=["renormalized", "tail"])
def test_entries_listed_twice_and_whole_vocabulary(tail):
    z, ids, t, lse = _case(4, 3000, 40, F32, 21, 1.0, tail)
    ids[0, 1::2] = ids[0, 0::2]                  # pairs
    ids[1] = ids[1, 0]                           # one entry, forty times
    ids[2, 39] = ids[2, 0]
    if tail:
        lse = torch.full_like(lse, float(t.max()) + 5)
    first = _check(z, ids, t, 1.0, lse)
    for _ in range(5):
        again = lpmm.distill_grad(z, ids, t, teacher_lse=lse)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    z, ids, t, lse = _case(3, 500, 500, F32, 22, 1.0, tail)     # the teacher lists everything: nothing is left out
    loss, grad = _check(z, ids, t, 1.0, lse)
    assert torch.isfinite(loss).all()


def test_extreme_temperatures_and_logits():
    for tau, spread in ((1e-3, 1.0), (1e3, 1.0), (1.0, 100.0), (1.0, 1e-4), (0.5, 1e4)):
        z, ids, t, lse = _case(3, 2000, 8, F32, 31, tau, True, spread)
        _check(z, ids, t, tau, lse)
        _check(z, ids, t, tau)
    z, ids, t, lse = _case(3, 2000, 8, F32, 32)
    shifted, _ = lpmm.distill_grad(z + 4096, ids, t)             # a constant added to a row changes only its rounding
    want, _ = lpmm.distill_grad(((z + 4096).double() - 4096).float(), ids, t)
    assert torch.equal(shifted, want)


@pytest.mark.parametrize("tail", [False, True], ids=["renormalized", "tail"])
def test_gradient_against_differences(tail):
    # Central differences of the loss, h = 0.05: off by h^2 / 6 times the third derivative (a log-sum-exp's is below 0.1 / tau^3,
    # two of them with the class of entries left out) and by the loss's own error over h.
    tau, h = 1.3, 0.05
    z, ids, t, lse = _case(2, 600, 9, F32, 41, tau, tail, 1.0)
    w = torch.tensor([0.7, 1.9], device="cuda")
    _, grad = lpmm.distill_grad(z, ids, t, temperature=tau, teacher_lse=lse, weights=w)
    for j in sorted({0, 17, 599, *ids[0, :3].tolist(), *ids[1, :3].tolist()}):
        up, down = z.clone(), z.clone()
        up[:, j] += h
        down[:, j] -= h
        kw = dict(temperature=tau, teacher_lse=lse, weights=w)
        d = (lpmm.distill_loss(up, ids, t, **kw).double() - lpmm.distill_loss(down, ids, t, **kw).double()) / (up[:, j].double() - down[:, j].double())
        r = (8 + 6 * 15 + 3) * U * 2 * w.double()
        tol = r / h + h * h / 6 * 0.3 / tau ** 3 * w.double()
        assert ((d - grad[:, j].double()).abs() <= tol).all()


def test_rows_beyond_2_31_elements_and_another_stream():
    tokens, vocab = 34_000, 65_536               # 2.2 G logits
    z = torch.randn(tokens, vocab, device="cuda", dtype=BF16)
    ids = torch.randint(0, vocab // 8, (tokens, 8), device="cuda") + torch.arange(8, device="cuda") * (vocab // 8)
    t = torch.randn(tokens, 8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, grad = lpmm.distill_grad(z, ids, t, stream=side)
    side.synchronize()
    for part in (slice(0, 3), slice(tokens - 3, tokens)):
        l2, g2 = _check(z[part].clone(), ids[part].clone(), t[part].clone(), rows=[0, 2])
        assert torch.allclose(l2, loss[part], rtol=1e-5, atol=1e-5) and torch.allclose(g2.float(), grad[part].float(), rtol=2.0 ** -7, atol=1e-7)


def test_in_a_graph_between_other_work():
    """Captured between kernels that produce its inputs and consume its outputs, and replayed with new values in the same buffers."""
    z, ids, t, lse = _case(64, 5001, 12, BF16, 51, 1.0, True)
    src, logits, grad = z.clone(), torch.empty_like(z), torch.empty_like(z)
    after = torch.empty(64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        lpmm.distill_grad(z, ids, t, teacher_lse=lse)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        logits.copy_(src)
        loss, _ = lpmm.distill_grad(logits, ids, t, teacher_lse=lse, out=grad)
        after.copy_(loss * 2)
    for k in range(5):
        src.copy_(z * (1 + k))
        graph.replay()
        want, gwant = lpmm.distill_grad(z * (1 + k), ids, t, teacher_lse=lse)
        assert torch.equal(after, want * 2) and torch.equal(grad, gwant)
