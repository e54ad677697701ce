"""The gradient of a gate per value, summed over all steps and rows, in whole numbers (or multiples of a power
of two) small enough that 32 bits hold every partial sum in any order: the sum is exact and compared bit
for bit, and a row or a run of rows that is left out or counted twice shows.

How the sum is shared (a workgroup's steps, its waves, the chunks of time, runs of rows, the threads of a
run) goes by the sizes; the shapes below have one stage and two, a last run shorter than the others,
chunks of time, rows one behind the other and apart."""
import numpy as np
import pytest
import torch

import paper_2407_04221_amd as av

# steps, rows, width, form
SHAPES = [(3, 1100, 1, "gated"), (3, 5000, 2, "gated"), (4, 1025, 3, "linear"), (9, 5000, 2, "linear"),
          (12, 140000, 1, "linear"), (9, 40000, 5, "linear"), (40, 700, 16, "linear"),
          (300, 16384, 1, "linear"), (500, 600, 3, "linear"), (2000, 300, 1, "linear"),
          (5003, 1, 6, "linear"), (1000, 70, 20, "linear")]


def make(T, B, D, form, flags=True):
    """Inputs as numpy arrays, and every step's and row's own part of the gradient [T][B][D] in 64 bits."""
    r = np.random.default_rng(T + B + D)
    draw = lambda *shape: r.integers(-2, 3, size=shape)
    x, dy, h0, dlast = draw(T, B, D), draw(T, B, D), draw(B, D), draw(B, D)
    # linear: gates of 1, -1 and 0.  gated: sigmoid(0), a half
    gate = np.resize([1, -1, 1, 0], D) if form == "linear" else np.zeros(D, dtype=np.int64)
    cut = (r.random((T, B)) < 0.4).astype(np.uint8) if flags else None
    a = gate.astype(float) if form == "linear" else np.full(D, 0.5)
    rest = 1.0 if form == "linear" else 0.5
    keep = np.ones((T, B)) if cut is None else 1.0 - cut
    came, s = np.empty((T, B, D)), h0.astype(float)
    for t in range(T):
        came[t] = keep[t][:, None] * s
        s = a * came[t] + rest * x[t]
    part, back = np.empty((T, B, D)), dlast.astype(float)
    for t in reversed(range(T)):
        lam = dy[t] + back
        part[t] = lam * came[t] if form == "linear" else lam * (came[t] - x[t]) * 0.25
        back = keep[t][:, None] * a * lam
    return x, gate, h0, cut, dy, dlast, part


def grain(T, form):
    """What every partial sum is a multiple of: a half for each step of s and of lam, and the quarter."""
    return 1.0 if form == "linear" else 2.0 ** -(2 * T + 2)


@pytest.mark.parametrize("T,B,D,form", SHAPES)
def test_sums_are_exact_and_every_run_of_rows_shows(T, B, D, form):
    """On the CPU: of the parts that the test below sums, any order fits 24 bits, and leaving out, or taking
    twice, any of the runs that the rows could be shared in changes the sum, in every value but those whose
    gate is 0 (in which nothing but cut steps would differ)."""
    *_, part = make(T, B, D, form)
    assert np.abs(part).sum((0, 1)).max() < 2 ** 24 * grain(T, form)
    assert np.array_equal(part / grain(T, form), np.round(part / grain(T, form)))
    rows = part.sum(0)
    for runs in (1, 2, 4, 19, 64):
        each = -(-B // runs)
        for r0 in range(0, B, each):
            assert (rows[r0:r0 + each] != 0).any(), (runs, r0)
    for chunks in (2, 8, 64):
        each = -(-T // chunks)
        for t0 in range(0, T, each):
            assert (part[t0:t0 + each] != 0).any(), (chunks, t0)


@pytest.mark.gpu
@pytest.mark.parametrize("T,B,D,form", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("layout", ["time", "batch"])
def test_sum_of_a_gate_per_value(T, B, D, form, dtype, reverse, layout):
    x, gate, h0, cut, dy, dlast, part = make(T, B, D, form)

    def steps(v):                     # in processing order, then in memory's
        v = torch.from_numpy(np.ascontiguousarray(v[::-1] if reverse else v))
        v = (v if v.dtype == torch.uint8 else v.to(dtype)).cuda()
        return v if layout == "time" else v.transpose(0, 1).contiguous().transpose(0, 1)
    state = lambda v: torch.from_numpy(v).float().cuda()
    x, dy, cut, gate = steps(x), steps(dy), steps(cut), torch.from_numpy(gate).to(dtype).cuda()
    y, dx, dgate = torch.empty_like(x), torch.empty_like(x), torch.full_like(gate, 9.0)
    how = dict(cut=cut, form=form, reverse=reverse)
    av.av_scan(x, gate, y, h0=state(h0), **how)
    av.av_scan_backward(x, gate, y, dy, dx, dgate, h0=state(h0), dlast=state(dlast), **how)
    want = torch.from_numpy(part.sum((0, 1))).to(dtype)
    assert torch.equal(dgate.cpu(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("T,B,D", [(4, 1300, 3), (20, 3000, 1), (3000, 2, 4)])
def test_sum_without_flags(T, B, D):
    """Rows one behind the other, as one."""
    x, gate, h0, _, dy, dlast, part = make(T, B, D, "linear", flags=False)
    gate[:] = 0
    part = np.where(np.arange(T)[:, None, None] == 0, h0, np.roll(x, 1, 0)) * \
        (dy + np.where(np.arange(T) == T - 1, 1, 0)[:, None, None] * dlast)
    on = lambda v: torch.from_numpy(v).float().cuda()
    x, dy, gate = on(x), on(dy), on(gate)
    y, dx, dgate = torch.empty_like(x), torch.empty_like(x), torch.full_like(gate, 9.0)
    av.av_scan(x, gate, y, h0=on(h0))
    av.av_scan_backward(x, gate, y, dy, dx, dgate, h0=on(h0), dlast=on(dlast))
    assert torch.equal(dgate.cpu().double(), torch.from_numpy(part.sum((0, 1))).double())


@pytest.mark.gpu
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("T,at", [(6, 3), (300, 200), (9000, 7001)])
def test_no_gradient_passes_a_cut(T, at, columns):
    """NaN and infinity in the gradients after a cut, and in the states before it, stay where they are."""
    x, dy = torch.ones((T, 1, 2), device="cuda"), torch.ones((T, 1, 2), device="cuda")
    gate = torch.full((2,) if columns else (T, 1, 2), 0.5, device="cuda")
    cut = torch.zeros((T, 1), dtype=torch.uint8, device="cuda")
    cut[at] = 1
    y, dx, dgate = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gate)
    dh0 = torch.empty((1, 2), device="cuda")
    av.av_scan(x, gate, y, cut=cut)
    dy[at + 1, 0, 0], dy[at + 1, 0, 1] = float("nan"), float("inf")
    av.av_scan_backward(x, gate, y, dy, dx, dgate, dh0=dh0, cut=cut)
    fine = torch.isfinite(dx)
    assert fine[:at].all() and not fine[at:at + 2].any() and fine[at + 2:].all()
    assert torch.isfinite(dh0).all()
    assert columns or torch.isfinite(dgate[:at]).all()
    x[at - 1] = float("nan")
    av.av_scan(x, gate, y, cut=cut)
    av.av_scan_backward(x, gate, y, torch.ones_like(dy), dx, dgate, dh0=dh0, cut=cut)
    assert torch.isfinite(dx).all() and torch.isfinite(dgate if columns else dgate[at]).all()
