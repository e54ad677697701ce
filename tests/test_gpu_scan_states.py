"""The gradient of 16-bit recurrences against 64 bits, with states that are held in 32 bits: what is rounded
to 16 bits is the stored result alone.  A sum over steps and rows whose terms cancel, or a state close to
x, shows every rounding on the way.

The bounds are those of a 32-bit recurrence (tests/learn_ref.py) on the same 16-bit inputs, and one rounding
of the output to its type.  That of a gate per value counts one rounding for each step of a column's sum,
and the joins of at most 16 waves, 64 runs and rows in powers of two, of the sum of absolute terms."""
import numpy as np
import pytest
import torch

import learn_ref as ref
import paper_2407_04221_amd as av

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def tensor(v, dtype, layout="time", pad=0, shift=0):
    T, B, D = v.shape
    dims = (T, B) if layout == "time" else (B, T)
    flat = torch.full((shift + dims[0] * dims[1] * (D + pad),), 7.0, dtype=TYPES[dtype], device="cuda")
    t = flat[shift:].view(dims[0], dims[1], D + pad)[:, :, :D]
    if layout != "time":
        t = t.transpose(0, 1)
    t.copy_(torch.from_numpy(v))
    return t


def run(T, B, D, dtype, form="linear", reverse=False, columns=False, cut=0.1, state=True, layout="time",
        pad=0, shift=0, seed=0, steady=False):
    r = np.random.default_rng(seed + T + B + D)
    kw = dict(dtype=dtype, layout=layout, pad=pad, shift=shift)
    x = tensor(np.full((T, B, D), 1.0) if steady else r.normal(size=(T, B, D)), **kw)
    shape = D if columns else (T, B, D)
    g = r.normal(size=shape) + 1.0 if form == "gated" else r.uniform(-1, 1, size=shape)
    gate = torch.from_numpy(g).to(TYPES[dtype]).cuda() if columns else tensor(g, **kw)
    dy = tensor(np.ones((T, B, D)) if steady else r.normal(size=(T, B, D)), **kw)
    flags = (r.random((T, B)) < cut).astype(np.uint8) if cut is not None else None
    c = torch.from_numpy(flags).cuda() if cut is not None else None
    f32 = lambda: torch.from_numpy(r.normal(size=(B, D))).float().cuda() if state else None
    h0, dlast = f32(), f32()
    y, dx = torch.empty_like(x), tensor(np.zeros((T, B, D)), **kw)
    dgate = torch.empty_like(gate) if columns else tensor(np.zeros((T, B, D)), **kw)
    dh0 = torch.empty((B, D), device="cuda") if state else None
    how = dict(cut=c, form=form, reverse=reverse)
    av.av_scan(x, gate, y, h0=h0, **how)
    av.av_scan_backward(x, gate, y, dy, dx, dgate, h0=h0, dlast=dlast, dh0=dh0, **how)
    opt = lambda t: None if t is None else host(t)
    args = (host(x), host(gate), opt(h0), flags, form, reverse, host(dy), opt(dlast))
    want = ref.scan(*args, "f32")                       # with the bounds of 32 bits throughout
    for name, got in (("dx", dx), ("dgate", dgate), ("dh0", dh0)):
        if got is None:
            continue
        v, bound = want[name]
        if name == "dgate" and columns:
            each = ref.scan(host(x), np.broadcast_to(host(gate), x.shape).copy(), *args[2:], "f32")["dgate"]
            depth = T + 16.0 + 64.0 + np.log2(max(2.0, T * B)) + B / 64.0
            bound = each[1].sum((0, 1)) + depth * ref.U * np.abs(each[0]).sum((0, 1))
        if name != "dh0":
            bound = ref.stored(v, bound, dtype)
        ref.check(host(got), (v, bound), f"{name} (T {T}, B {B}, D {D})", dtype if name != "dh0" else "f32")


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 8, 9, 31, 32, 33, 63, 64, 65, 130, 517])
@pytest.mark.parametrize("form", ["linear", "gated"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_lengths(T, form, dtype):
    run(T, 3, 5, dtype, form)
    run(T, 2, 64, dtype, form, reverse=True, columns=True)


@pytest.mark.parametrize("form", ["linear", "gated"])
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("reverse", [False, True])
def test_kinds(form, columns, dtype, reverse):
    """Chunks of time with single columns and words of two and four, uncut words, several tiles, widths
    that share columns, rows one behind the other with a flag for each and without."""
    kw = dict(dtype=dtype, form=form, columns=columns, reverse=reverse)
    run(5003, 1, 6, cut=0.003, **kw)
    run(2048, 2, 65, cut=None, **kw)
    run(1000, 2, 12, **kw)
    run(700, 1, 9, **kw)
    run(2500, 1, 1, **kw)
    run(70, 258, 130, state=False, **kw)
    run(37, 300, 128, **kw)
    run(900, 130, 1, cut=0.02, **kw)
    run(600, 20, 3, cut=None, **kw)
    run(300, 2100, 8, cut=0.02, **kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("form", ["linear", "gated"])
def test_many_columns_and_short(dtype, form):
    for columns in (False, True):
        run(130, 1024, 64, dtype, form, columns=columns)
        for T in (2, 5, 7):
            run(T, 500, 33, dtype, form, columns=columns, reverse=T == 5)


@pytest.mark.parametrize("layout", ["time", "batch"])
@pytest.mark.parametrize("pad,shift", [(2, 0), (1, 1), (3, 5)])
def test_layouts(layout, pad, shift):
    for T, B, D in ((19, 4, 12), (300, 3, 1), (1000, 3, 7)):
        run(T, B, D, "bf16", "gated", layout=layout, pad=pad, shift=shift)
        run(T, B, D, "f16", layout=layout, pad=pad, shift=shift, columns=True, reverse=True)


@pytest.mark.parametrize("T,B,D", [(6, 40, 8), (50, 3, 10), (2000, 2, 6)])
def test_states_that_settle_at_x(T, B, D):
    """A state next to x, whose difference is far below a step of the 16-bit type."""
    for columns in (False, True):
        run(T, B, D, "bf16", "gated", steady=True, cut=None, columns=columns)


@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("T,B,D", [(5, 300, 325), (60, 420, 325), (1000, 3, 325), (700, 1, 9)])
def test_over_its_inputs(T, B, D, columns):
    """dx over dy and dgate over the gate, equal bits; and the same call twice."""
    r = np.random.default_rng(3)
    new = lambda *s: torch.from_numpy(r.normal(size=s)).bfloat16().cuda()
    x, dy, gate = new(T, B, D), new(T, B, D), new(D) if columns else new(T, B, D)
    h = torch.from_numpy(r.normal(size=(B, D))).float().cuda()
    cut = torch.from_numpy((r.random((T, B)) < 0.1).astype(np.uint8)).cuda()
    y = torch.empty_like(x)
    how = dict(cut=cut, form="gated")
    av.av_scan(x, gate, y, h0=h, **how)
    outs = []
    for over in (False, False, True):
        d, g = dy.clone(), gate.clone()
        dx = d if over else torch.empty_like(x)
        dg = g if over and not columns else torch.empty_like(gate)
        dh = torch.empty_like(h)
        av.av_scan_backward(x, g, y, d, dx, dg, h0=h, dlast=h, dh0=dh, **how)
        outs.append((dx, dg, dh))
    for o in outs[1:]:
        for a, b in zip(o, outs[0]):
            assert torch.equal(a, b)


def test_linear_over_x():
    """Where the recurrence was written over x, or x is not given, y stands for the states."""
    r = np.random.default_rng(4)
    T, B, D = 50, 3, 10
    x = torch.from_numpy(r.normal(size=(T, B, D))).half().cuda()
    gate, dy = (torch.from_numpy(r.uniform(-1, 1, size=(T, B, D))).half().cuda() for _ in range(2))
    y = x.clone()
    av.av_scan(y, gate, y)
    dx, dgate = torch.empty_like(x), torch.empty_like(x)
    av.av_scan_backward(y, gate, y, dy, dx, dgate)
    want = ref.scan(host(x), host(gate), dy=host(dy), dtype="f16")
    ref.check(host(dx), want["dx"], "dx", "f16")
    ref.check(host(dgate), want["dgate"], "dgate", "f16")


@pytest.mark.parametrize("form", ["linear", "gated"])
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("T,B,D", [(6, 50, 8), (70, 300, 130), (1500, 2, 12)])
def test_without_the_gates_gradient(T, B, D, form, columns):
    """dx and dh0, asked for dgate or not."""
    r = np.random.default_rng(6)
    new = lambda *s: torch.from_numpy(r.uniform(-1, 1, size=s)).half().cuda()
    x, dy, gate = new(T, B, D), new(T, B, D), new(D) if columns else new(T, B, D)
    cut = torch.from_numpy((r.random((T, B)) < 0.05).astype(np.uint8)).cuda()
    y = torch.empty_like(x)
    av.av_scan(x, gate, y, cut=cut, form=form)
    outs = []
    for dgate in (torch.empty_like(gate), None):
        dx, dh0 = torch.empty_like(x), torch.empty((B, D), device="cuda")
        av.av_scan_backward(x, gate, y, dy, dx, dgate, dh0=dh0, cut=cut, form=form)
        outs.append((dx, dh0))
    if form == "gated":                    # the linear one reads y then, in words of other widths
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    want = ref.scan(host(x), host(gate), None, cut.cpu().numpy(), form, dy=host(dy), dtype="f16")
    for dx, dh0 in outs:
        ref.check(host(dx), want["dx"], "dx", "f16")
        ref.check(host(dh0), want["dh0"], "dh0")


def test_a_graph_beside_eager_calls():
    T, B, D = 400, 3, 20
    r = np.random.default_rng(5)
    new = lambda: torch.from_numpy(r.normal(size=(T, B, D))).bfloat16().cuda()
    x, gate, dy = new(), new(), new()
    y = torch.empty_like(x)
    av.av_scan(x, gate, y, form="gated")
    want = torch.empty_like(x), torch.empty_like(x)
    av.av_scan_backward(x, gate, y, dy, *want, form="gated")
    got = torch.zeros_like(x), torch.zeros_like(x)
    ws = torch.empty(av.av_scan_workspace(T, B, D, False, True, av.AV_BF16), dtype=torch.uint8,
                     device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        av.av_scan_backward(x, gate, y, dy, *got, form="gated", workspace=ws)
    for _ in range(3):
        g.replay()
        again = torch.empty_like(x), torch.empty_like(x)
        av.av_scan_backward(x, gate, y, dy, *again, form="gated")
        torch.cuda.synchronize()
        for a, b, c in zip(want, got, again):
            assert torch.equal(a, b) and torch.equal(a, c)
            b.zero_()


@pytest.mark.parametrize("T", [7, 8, 30, 33, 70, 96])
@pytest.mark.parametrize("columns", [False, True])
def test_rows_far_apart(T, columns):
    """Rows of x past a wave's 32-bit distances: the same in whole numbers as rows that lie together."""
    D, apart = 4, (1 << 31) // 3 + 24
    r = np.random.default_rng(T)
    whole = lambda *s: torch.from_numpy(r.integers(-2, 3, size=s)).bfloat16().cuda()
    near, dy, h = whole(T, 3, D), whole(T, 3, D), whole(3, D).float()
    gate = torch.ones(D, dtype=torch.bfloat16, device="cuda") if columns else \
        torch.ones((T, 3, D), dtype=torch.bfloat16, device="cuda")
    cut = torch.from_numpy((r.random((T, 3)) < 0.2).astype(np.uint8)).cuda()
    far = torch.empty(2 * apart + T * D, dtype=torch.bfloat16, device="cuda").as_strided(
        (T, 3, D), (D, apart, 1))
    far.copy_(near)
    outs = []
    for x in (near, far):
        y, dx = torch.empty_like(near), torch.empty_like(near)
        dgate, dh0 = torch.empty_like(gate), torch.empty_like(h)
        av.av_scan(x, gate, y, h0=h, cut=cut)
        av.av_scan_backward(x, gate, y, dy, dx, dgate, h0=h, dlast=h, dh0=dh0, cut=cut)
        outs.append((y, dx, dgate, dh0))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
