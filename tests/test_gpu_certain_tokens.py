"""Rows with one all but certain choice: its log-probability, the entropy and its gradient are small, and
as exact relative to themselves as large ones are.

With x = sum of the other choices' weights relative to the largest, log p = -log(1 + x), 1 - p = x / (1 + x)
and H = log(1 + x) + sum e d / (1 + x), d the distance of a logit from the largest and e = exp(-d).  U is half
a step of a 32-bit number.  A weight is off by (1 + d) 2 U of itself (its distance, the constant and the
product, and the power of two by 2 U), so x by (1 + d) 2 U and by U for each addition that one lane makes
in a row: A / 64 + 64 at most with all joins, and A of up to 16.  log1p, expm1 and the constants around
them add 2 U each: 12 U."""
import numpy as np
import pytest
import torch

import learn_ref as ref
import paper_2407_04221_amd as av

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def rows_with_a_certain_choice(N, A, lo, hi, dtype, seed):
    """Distances between lo and hi from the largest, which is anywhere and of any size."""
    r = np.random.default_rng(seed)
    at = r.integers(0, A, size=N)
    base = np.round(r.uniform(-2, 2, size=(N, 1)))
    l = torch.from_numpy(base - r.uniform(lo, hi, size=(N, A)))
    l[torch.arange(N), torch.from_numpy(at)] = torch.from_numpy(base[:, 0])
    return l.to(TYPES[dtype]).cuda(), at


def relative(A, reach):
    return ref.U * (2.0 * (1.0 + reach) + min(A, A / 64.0 + 64.0) + 12.0)


def exact(logits, at):
    """(log p, x, H) of the largest choice, which no other equals."""
    l = host(logits)
    d = np.take_along_axis(l, at[:, None], 1) - l
    e = np.exp(-d)
    e[np.arange(len(l)), at] = 0.0
    x, xd = e.sum(1), (e * np.where(np.isfinite(d), d, 0.0)).sum(1)
    return -np.log1p(x), x, np.log1p(x) + xd / (1.0 + x)


SHAPES = [(300, 2), (300, 5), (70, 16), (70, 17), (70, 40), (70, 131), (40, 300), (40, 1000), (20, 2040),
          (20, 4096), (600, 5003), (5, 5003), (5, 20001), (3, 70001), (2, 131072)]


@pytest.mark.parametrize("N,A", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("above", [0.0, 12.0])
def test_certain_choices(N, A, dtype, above):
    """x of about 1e-1, and of about 1e-6."""
    lo = 3.0 + above + np.log(A)
    logits, at = rows_with_a_certain_choice(N, A, lo, lo + 3.0, dtype, A)
    f = dict(dtype=torch.float32, device="cuda")
    ids = torch.from_numpy(at).cuda()
    logp, ent, st = torch.empty(N, **f), torch.empty(N, **f), torch.empty((N, 2), **f)
    tl, ti = torch.empty((N, 1), **f), torch.empty((N, 1), dtype=torch.int32, device="cuda")
    av.av_log_probs(logits, ids, logp, ent, st, tl, ti)
    want, x, H = exact(logits, at)
    tol = relative(A, lo + 4.0)
    assert np.array_equal(ti[:, 0].cpu().numpy(), at)
    for got in (logp, tl[:, 0]):
        ref.check(host(got), (want, tol * np.abs(want)), "logp")
    # H: its sum of weights and distances by U more for each distance, its division and product
    ref.check(host(ent), (H, (tol + 6.0 * ref.U) * H), "entropy")
    # the gradient of log p: 1 - p for itself, -p_i for the others; p_i by tol of itself and by lse's error
    d = torch.empty_like(logits)
    one = torch.ones(N, **f)
    av.av_log_probs_backward(logits, ids, st, None, one, None, d)
    p = np.exp(host(logits) - host(logits)[np.arange(N), at][:, None] - np.log1p(x)[:, None])
    g = -p
    g[np.arange(N), at] = x / (1.0 + x)
    ref.check(host(d), (g, ref.stored(g, 2.0 * tol * np.abs(g), dtype)), "gradient of log p", dtype)
    # that of the entropy: -p (log p + H); what is left of log p + H at the certain choice,
    # (sum e d) / (1 + x), is larger than either of the two here (d >= 3), so no more is lost
    av.av_log_probs_backward(logits, None, st, ent, None, one, d)
    lp = host(logits) - host(logits)[np.arange(N), at][:, None] - np.log1p(x)[:, None]
    g = -p * (lp + H[:, None])
    ref.check(host(d), (g, ref.stored(g, 8.0 * tol * np.abs(g), dtype)), "gradient of the entropy", dtype)


def test_as_the_draw_says():
    """An agent's two records of one action: drawn, and looked up afterwards."""
    logits, at = rows_with_a_certain_choice(500, 5, 8.0, 20.0, "f32", 3)
    drawn, actions = torch.empty(500, device="cuda"), torch.empty(500, dtype=torch.uint8, device="cuda")
    av.av_draw_actions(logits, torch.full((500,), 0.5, device="cuda"), actions, drawn)
    logp = torch.empty(500, device="cuda")
    av.av_log_probs(logits, actions, logp)
    want = exact(logits, at)[0]
    for got in (drawn, logp):
        ref.check(host(got), (want, relative(5, 20.0) * np.abs(want)), "logp")


@pytest.mark.parametrize("A", [5, 100, 3000, 9000])
def test_beyond_any_weight(A):
    """Others too far away for a weight, or masked: log p is 0, and so are entropy and gradient."""
    for other in (-1.0e4, -np.inf):
        logits = torch.full((4, A), other, device="cuda")
        logits[:, A // 2] = 2.5
        ids = torch.full((4,), A // 2, device="cuda")
        logp, ent = torch.ones(4, device="cuda"), torch.ones(4, device="cuda")
        st, d = torch.empty((4, 2), device="cuda"), torch.ones((4, A), device="cuda")
        av.av_log_probs(logits, ids, logp, ent, st)
        av.av_log_probs_backward(logits, ids, st, ent, torch.ones(4, device="cuda"),
                                 torch.ones(4, device="cuda"), d)
        assert (logp == 0).all() and (ent == 0).all() and (d == 0).all()
