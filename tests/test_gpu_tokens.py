"""av_log_probs, av_log_probs_backward and av_draw_actions on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

import learn_ref as ref
import paper_2407_04221_amd as av

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
IDS = {"u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}


def host(t):
    return t.detach().double().cpu().numpy()


def rows_of(N, A, dtype, pad=0, shift=0):
    flat = torch.full((shift + N * (A + pad),), 9.0, dtype=TYPES[dtype], device="cuda")
    return flat[shift:].view(N, A + pad)[:, :A]


def compare(logits, ids, dtype, top=0, back_pad=0, back_shift=0, seed=0):
    """Forward and gradient of these logits (device [N][A]) and ids (numpy) against 64 bits."""
    N, A = logits.shape
    r = np.random.default_rng(seed)
    wide = torch.from_numpy(ids).to("cuda")
    f = dict(dtype=torch.float32, device="cuda")
    logp, ent, stats = torch.empty(N, **f), torch.empty(N, **f), torch.empty((N, 2), **f)
    tl = ti = None
    if top:
        tl, ti = torch.empty((N, top), **f), torch.empty((N, top), dtype=torch.int32, device="cuda")
    av.av_log_probs(logits, wide, logp, ent, stats, tl, ti)
    g = torch.from_numpy(r.normal(size=N)).float().cuda()
    gh = torch.from_numpy(r.normal(size=N)).float().cuda()
    d = rows_of(N, A, dtype, back_pad, back_shift)
    av.av_log_probs_backward(logits, wide, stats, ent, g, gh, d)
    want = ref.tokens(host(logits), ids.astype(np.int64), host(g), host(gh), top, dtype)
    where = f"(N {N}, A {A}, {dtype})"
    ref.check(host(logp), want["logp"], "logp " + where)
    ref.check(host(ent), want["entropy"], "entropy " + where)
    if top:
        assert np.array_equal(ti.cpu().numpy(), want["top_ids"]), "top_ids " + where
        ref.check(host(tl), want["top_logp"], "top_logp " + where)
    ref.check(host(d), want["dlogits"], "dlogits " + where, dtype)
    return logp, ent, stats, d


def some(N, A, dtype, seed=0, scale=2.0, pad=0, shift=0, masked=0.0):
    r = np.random.default_rng(seed)
    v = torch.from_numpy(r.normal(size=(N, A)) * scale)
    if masked:
        v[torch.from_numpy(r.random((N, A)) < masked)] = -np.inf
    logits = rows_of(N, A, dtype, pad, shift)
    logits.copy_(v)
    return logits, r


SIZES = [1, 2, 3, 4, 5, 8, 9, 16, 17, 63, 64, 65, 255, 511, 513, 1023, 1025, 2041, 2047, 2048, 2049,
         5000, 16385]


@pytest.mark.parametrize("A", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_sizes(A, dtype):
    logits, r = some(7, A, dtype)
    compare(logits, r.integers(-1, A + 1, size=7), dtype, top=min(A, 6))


@pytest.mark.parametrize("A", [140, 300, 1000, 2001])
@pytest.mark.parametrize("top", [1, 3, 4, 5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_alternatives(A, top, dtype):
    """Equal logits in several lanes and words, fewer choices than alternatives, none at all."""
    logits, r = some(9, A, dtype, seed=A, masked=0.1)
    logits[1] = 0.25
    logits[2] = torch.where(torch.arange(A, device="cuda") % 37 == 5, 1.5, -2.0).to(logits.dtype)
    logits[3, :] = -np.inf
    logits[3, A - 1] = -7.0
    logits[4, :] = -np.inf
    logits[5] = torch.where(torch.arange(A, device="cuda") % 2 == 0, 0.0, -0.0).to(logits.dtype)
    compare(logits, r.integers(0, A, size=9), dtype, top=top)


@pytest.mark.parametrize("A", [2100, 3001, 3100, 4095, 4096, 4097])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_longest_rows_of_a_wave(A, dtype):
    logits, r = some(6, A, dtype, seed=A, masked=0.1)
    ids = r.integers(0, A, size=6)
    compare(logits, ids, dtype, top=9)
    logits[2] = 0.5                             # all equal: too many for a list of candidates
    logits[3, 5:] = -np.inf                     # fewer than the alternatives
    compare(logits, ids, dtype, top=9)


@pytest.mark.parametrize("N,A", [(1, 5), (255, 5), (256, 5), (257, 5), (1000, 3), (5, 100), (1, 70000),
                                 (600, 2500), (511, 4100), (3000, 40)])
def test_rows(N, A):
    for dtype in ("f32", "bf16"):
        logits, r = some(N, A, dtype)
        compare(logits, r.integers(0, A, size=N), dtype, top=3)


@pytest.mark.parametrize("A", [19, 30, 45, 51, 64, 66, 91, 96, 113, 128, 148, 200, 256, 300, 381, 509, 700])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_of_medium_length(A, dtype):
    """61 rows against 64 bits, and again and again in one call: every time the same bits."""
    few, r = some(61, A, dtype, seed=A, masked=0.1)
    few[2] = -np.inf
    few[3] = 2.0
    few[4, 1:] = -np.inf
    few[5, A // 3] = float("nan")
    few[6] = torch.where(torch.arange(A, device="cuda") % 9 == 4, 1.0, 0.5).to(few.dtype)
    ids = r.integers(-1, A, size=61)
    g, gh = r.normal(size=61).astype(np.float32), r.normal(size=61).astype(np.float32)
    times = -(-(1 << 20) * (4 if dtype == "f32" else 8) // (A * 61)) + 1
    logits, N = few.repeat(times, 1), 61 * times
    many = lambda v: torch.from_numpy(v).cuda().repeat(times)
    f = dict(dtype=torch.float32, device="cuda")
    logp, ent, stats = torch.empty(N, **f), torch.empty(N, **f), torch.empty((N, 2), **f)
    for top in (4, 9):
        tl, ti = torch.empty((N, top), **f), torch.empty((N, top), dtype=torch.int32, device="cuda")
        av.av_log_probs(logits, many(ids), logp, ent, stats, tl, ti)
        want = ref.tokens(host(few), ids, g, gh, top, dtype)
        ref.check(host(logp[:61]), want["logp"], "logp")
        ref.check(host(ent[:61]), want["entropy"], "entropy")
        assert np.array_equal(ti[:61].cpu().numpy(), want["top_ids"])
        ref.check(host(tl[:61]), want["top_logp"], "top_logp")
        for t in (logp, ent, tl, ti):
            same = t.view(torch.int32).view(times, 61, -1)
            assert torch.equal(same, same[:1].expand_as(same))
    av.av_log_probs(logits, many(ids), logp, ent, stats)
    ref.check(host(logp[:61]), want["logp"], "logp")
    ref.check(host(ent[:61]), want["entropy"], "entropy")
    d = torch.empty_like(logits)
    av.av_log_probs_backward(logits, many(ids), stats, ent, many(g), many(gh), d)
    ref.check(host(d[:61]), want["dlogits"], "dlogits", dtype)
    bits = d.view(torch.int32 if dtype == "f32" else torch.int16).view(times, 61, A)
    assert torch.equal(bits, bits[:1].expand_as(bits))
    av.av_log_probs_backward(logits, many(ids), stats, ent, many(g), many(gh), logits)
    assert torch.equal(logits.view(bits.dtype), d.view(bits.dtype))


@pytest.mark.parametrize("A,dtype", [(16387, "f32"), (40003, "f16"), (32768, "bf16")])
def test_many_long_rows(A, dtype):
    """2100 rows, the first seven compared, the others the same again."""
    few, r = some(7, A, dtype, seed=3, masked=0.1)
    few[2, : A // 2] = -np.inf
    few[3] = 2.0
    ids = r.integers(0, A, size=7)
    logits = few.repeat(300, 1)
    N = len(logits)
    f = dict(dtype=torch.float32, device="cuda")
    logp, ent, stats = torch.empty(N, **f), torch.empty(N, **f), torch.empty((N, 2), **f)
    tl, ti = torch.empty((N, 4), **f), torch.empty((N, 4), dtype=torch.int32, device="cuda")
    wide = torch.from_numpy(ids).cuda().repeat(300)
    av.av_log_probs(logits, wide, logp, ent, stats, tl, ti)
    assert torch.equal(ti.view(300, 7, 4), ti[:7].expand(300, 7, 4))
    assert torch.equal(logp.view(300, 7), logp[:7].expand(300, 7))
    assert torch.equal(ent.view(300, 7), ent[:7].expand(300, 7))
    want = ref.tokens(host(few), ids, np.zeros(7), np.zeros(7), 4, dtype)
    ref.check(host(logp[:7]), want["logp"], "logp")
    ref.check(host(ent[:7]), want["entropy"], "entropy")
    ref.check(host(tl[-7:]), want["top_logp"], "top_logp")
    assert np.array_equal(ti[:7].cpu().numpy(), want["top_ids"])


@pytest.mark.parametrize("ids", ["u8", "i32", "i64"])
def test_id_types_and_padding(ids):
    for A in (5, 300, 3001):
        logits, r = some(50, A, "f32")
        v = r.integers(0, min(A, 256), size=50)
        v[::7] = 255 if ids == "u8" else -1
        if ids == "i64":
            v[1::7] = 1 << 32                              # not id 0
        logp, *_ = compare(logits, v.astype({"u8": np.uint8, "i32": np.int32, "i64": np.int64}[ids]),
                           "f32")
        if A == 5:
            assert (logp[::7] == 0).all()


@pytest.mark.parametrize("pad,shift,bpad,bshift", [(0, 0, 0, 0), (1, 0, 1, 0), (3, 1, 3, 1),
                                                   (8, 0, 0, 0), (0, 1, 0, 2), (7, 5, 1, 3)])
@pytest.mark.parametrize("A", [5, 130, 2600])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_strides(pad, shift, bpad, bshift, A, dtype):
    """Rows and their gradients at any distance from a word's border; what lies between is left."""
    logits, r = some(9, A, dtype, pad=pad, shift=shift)
    *_, d = compare(logits, r.integers(0, A, size=9), dtype, top=4, back_pad=bpad,
                    back_shift=bshift)
    if bpad:
        between = d.as_strided((9, bpad), (A + bpad, 1), d.storage_offset() + A)[:-1]
        assert (between == 9.0).all()


@pytest.mark.parametrize("A", [5, 100, 2000, 9000, 33000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masks(A, dtype):
    """Masked choices, given tokens among them, and rows that a mask leaves one or no choice."""
    logits, r = some(12, A, dtype, masked=0.5)
    logits[0] = -np.inf                                    # nothing left
    logits[1] = -np.inf
    logits[1, A - 1] = 3.0                                 # one left, the last
    logits[2] = -np.inf
    logits[2, 0] = -7.0
    lowest = torch.finfo(TYPES[dtype]).min
    logits[3] = lowest                                     # all of the lowest value: uniform
    logits[4] = lowest
    logits[4, A // 2] = 0.0
    logits[5] = torch.finfo(TYPES[dtype]).max
    logits[6, ::2] = lowest
    ids = r.integers(0, A, size=12)
    ids[2], ids[4] = A - 1, 0                              # masked, and all but masked
    logp, ent, _, d = compare(logits, ids, dtype, top=min(A, 8))
    assert logp[0] == -np.inf and ent[0] == 0 and (d[0] == 0).all()
    assert logp[2] == -np.inf and ent[1] == 0


@pytest.mark.parametrize("A", [3, 60, 1500, 7000, 20001])
def test_infinities_and_nan(A):
    """A row with a NaN or +inf is NaN throughout and leaves its neighbours alone."""
    logits, r = some(8, A, "f32")
    logits[1, A - 1] = float("nan")
    logits[3, A // 2] = float("inf")
    logits[5] = float("nan")
    logits[6] = -np.inf
    logits[6, A - 1] = float("nan")
    ids = r.integers(0, A, size=8)
    ids[5] = -1
    logp, ent, _, d = compare(logits, ids, "f32", top=2)
    assert logp[5] == 0 and torch.isnan(ent[5])


@pytest.mark.parametrize("A", [16, 500, 2048, 3000, 40000])
@pytest.mark.parametrize("order", ["equal", "rising", "falling", "steps", "one_thread"])
def test_alternatives_of_hard_orders(A, order):
    """Ties, and rows whose largest values sit together: the lowest index of equal ones first."""
    i = torch.arange(A, dtype=torch.float64)
    v = {"equal": i * 0, "rising": i / A * 4, "falling": -i / A * 4, "steps": -(i // 37 % 5),
         "one_thread": torch.where(i % 1024 < 8, i / A, i * 0 - 1)}[order]
    for dtype in ("f32", "bf16"):
        for top in (1, 32 if A > 32 else A):
            for N in (2, 600 if A == 3000 else 3):
                logits = rows_of(N, A, dtype)
                logits.copy_(v.expand(N, A))
                compare(logits, np.zeros(N, np.int64), dtype, top=top)


@pytest.mark.parametrize("case", ["few_threads", "one_lane_in_three", "equal"])
def test_alternatives_that_do_not_fit_the_list(case):
    """The largest values in the hands of fewer than `top` threads, thousands of them; almost all
    masked; all equal.  One row for all (a stride of 0), so many rows cost no memory."""
    A, top = 60000, 32
    i = torch.arange(A)
    word = i // 4
    r = np.random.default_rng(7)
    v = torch.from_numpy(r.normal(size=A)).float()
    if case == "few_threads":
        v += torch.where(word % 512 < 31, 100.0, 0.0)
    elif case == "one_lane_in_three":
        v = torch.where(word % 64 % 3 == 0, v, -np.inf)
    else:
        v = torch.zeros(A)
    row = torch.empty(A, device="cuda")
    row.copy_(v)
    want = ref.tokens(host(row)[None], np.zeros(1, np.int64), top=top)
    for N in (2, 520, 2100):
        tl = torch.empty((N, top), device="cuda")
        ti = torch.empty((N, top), dtype=torch.int32, device="cuda")
        av.av_log_probs(row.expand(N, A), top_logp=tl, top_ids=ti)
        for n in (0, N // 2, N - 1):
            assert np.array_equal(ti[n:n + 1].cpu().numpy(), want["top_ids"])
            ref.check(host(tl[n:n + 1]), want["top_logp"], f"top_logp, {N} rows")


def test_many_rows_and_offsets_past_32_bits():
    """Rows of more than one launch, and more than 2^32 bytes of logits: the last rows come out as
    they do alone."""
    for N, A, dtype in (((1 << 22) + 5, 17, "f16"), (70001, 32768, "f16"), ((1 << 22) + 3, 4, "f32"),
                        ((1 << 22) + 7, 65, "bf16")):
        l = torch.empty((N, A), dtype=TYPES[dtype], device="cuda").normal_()
        ids = torch.randint(0, A, (N,), device="cuda", dtype=torch.int32)
        f = dict(device="cuda")

        def call(l, ids):
            n = len(ids)
            o = [torch.zeros(n, **f), torch.zeros(n, **f), torch.zeros((n, 2), **f),
                 torch.zeros((n, 2), **f), torch.zeros((n, 2), dtype=torch.int32, **f)]
            av.av_log_probs(l, ids, *o)
            o.append(torch.zeros_like(l))
            av.av_log_probs_backward(l, ids, o[2], o[1], o[0], o[0], o[5])
            if A <= 256:
                o.append(torch.zeros(n, dtype=torch.uint8, **f))
                av.av_draw_actions(l, torch.sigmoid(o[0]), o[6])
            return o
        whole, tail = call(l, ids), call(l[-600:], ids[-600:])
        # (another number of rows may take other kernels for rows above four words: sums in another
        # order, compared with 64 bits where there is a bound of the gradient's rounding to bf16)
        if A == 65:
            o, few = [t[-600:] for t in whole], host(l[-600:])
            want = ref.tokens(few, ids[-600:].cpu().numpy().astype(np.int64), host(o[0]), host(o[0]),
                              2, dtype)
            ref.check(host(o[0]), want["logp"], "logp")
            ref.check(host(o[1]), want["entropy"], "entropy")
            ref.check(host(o[3]), want["top_logp"], "top_logp")
            assert np.array_equal(o[4].cpu().numpy(), want["top_ids"])
            ref.check(host(o[5]), want["dlogits"], "dlogits", dtype)
            assert np.array_equal(o[6].cpu().numpy(), ref.draw(few, host(torch.sigmoid(o[0])))[0])
            continue
        exact = A <= 2048
        for a, b in zip(whole, tail):
            a = a[-600:]
            assert torch.equal(a, b) if exact else torch.allclose(a.float(), b.float(), atol=1e-4)
        del whole, tail, l


def test_more_alternatives_than_choices():
    logits, _ = some(4, 3, "f32")
    compare(logits, np.zeros(4, np.int64), "f32", top=5)
    zero = torch.tensor([[0.0, -0.0, 0.0]], device="cuda")
    compare(zero, np.zeros(1, np.int64), "f32", top=3)


def test_confident_and_wide_rows():
    for scale in (0.0, 1e-3, 30.0, 1e4):
        for A in (5, 1000, 6000):
            logits, r = some(6, A, "f32", scale=scale)
            compare(logits, r.integers(0, A, size=6), "f32", top=2)


def test_parts_on_request():
    """Any output alone, either gradient alone, and the gradient in place."""
    for A in (5, 300, 4000, 30000):
        logits, r = some(10, A, "f32")
        ids = torch.from_numpy(r.integers(0, A, size=10)).cuda()
        f = dict(device="cuda")
        logp, ent, stats = torch.empty(10, **f), torch.empty(10, **f), torch.empty((10, 2), **f)
        av.av_log_probs(logits, ids, logp, ent, stats)
        a, b, c = torch.empty(10, **f), torch.empty(10, **f), torch.empty((10, 2), **f)
        av.av_log_probs(logits, ids, a)
        av.av_log_probs(logits, entropy=b)
        av.av_log_probs(logits, stats=c)
        assert torch.equal(a, logp) and torch.equal(b, ent) and torch.equal(c, stats)
        g, gh, zero = torch.randn(10, **f), torch.randn(10, **f), torch.zeros(10, **f)
        d = [torch.empty_like(logits) for _ in range(5)]
        av.av_log_probs_backward(logits, ids, stats, None, g, None, d[0])
        av.av_log_probs_backward(logits, ids, stats, ent, g, zero, d[1])
        av.av_log_probs_backward(logits, None, stats, ent, None, gh, d[2])
        av.av_log_probs_backward(logits, ids, stats, ent, zero, gh, d[3])
        assert torch.equal(d[0], d[1]) and torch.equal(d[2], d[3])
        av.av_log_probs_backward(logits, ids, stats, ent, g, gh, d[4])
        same = logits.clone()
        av.av_log_probs_backward(same, ids, stats, ent, g, gh, same)
        assert torch.equal(same, d[4])


@pytest.mark.parametrize("N,A", [(700, 5), (700, 7), (300, 131), (20, 2043), (40, 9001), (1, 70003)])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_gradient_over_the_logits(N, A, dtype):
    """dlogits in the logits' own place, rows' last words sharing elements with the word before."""
    logits, r = some(N, A, dtype, seed=8, pad=1, masked=0.05)
    ids = torch.from_numpy(r.integers(0, A, size=N)).cuda()
    f = dict(dtype=torch.float32, device="cuda")
    logp, ent, stats = torch.empty(N, **f), torch.empty(N, **f), torch.empty((N, 2), **f)
    av.av_log_probs(logits, ids, logp, ent, stats)
    g, gh = torch.randn(N, **f), torch.randn(N, **f)
    d = rows_of(N, A, dtype, 1, 0)
    av.av_log_probs_backward(logits, ids, stats, ent, g, gh, d)
    av.av_log_probs_backward(logits, ids, stats, ent, g, gh, logits)
    assert torch.equal(d, logits)


def test_one_row_for_all():
    """A row stride of 0."""
    row = torch.randn((1, 50), device="cuda")
    logits, ids = row.expand(20, 50), torch.arange(20, device="cuda")
    a, b = torch.empty(20, device="cuda"), torch.empty(20, device="cuda")
    av.av_log_probs(logits, ids, a)
    av.av_log_probs(logits.contiguous(), ids, b)
    want = ref.tokens(host(logits), np.arange(20))
    ref.check(host(a), want["logp"], "logp, one row for all")
    ref.check(host(b), want["logp"], "logp, copied rows")
    with pytest.raises(av.AvError):
        av.av_log_probs_backward(logits, ids, torch.empty((20, 2), device="cuda"), None, a, None,
                                 torch.empty((1, 50), device="cuda").expand(20, 50))


@pytest.mark.parametrize("A", [1, 2, 5, 8, 9, 17, 64, 65, 128, 129, 255, 256])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_draw(A, dtype):
    for N in (1, 131, 1000):
        logits, r = some(N, A, dtype, masked=0.3, pad=A % 3)
        if N > 1:
            logits[0] = -np.inf
            logits[1, A - 1] = float("nan")
            logits[2, A // 2] = float("inf")
            logits[3] = 0.0
        u = r.random(N).astype(np.float32)
        u[-3:] = (0.0, 1.0 - 2.0 ** -24, 1.0)[-min(3, N):]
        actions = torch.empty(N, dtype=torch.uint8, device="cuda")
        logp = torch.empty(N, device="cuda")
        av.av_draw_actions(logits, torch.from_numpy(u).cuda(), actions, logp)
        want, want_logp = ref.draw(host(logits), u)
        assert np.array_equal(actions.cpu().numpy(), want)
        # the sum of weights in 32 bits: each is off by (1 + |t| ln 2) 2 U of itself with the mean of
        # |t| at most log2 A, fourteen additions and the logarithm by U each: 2 (1 + 0.7 log2 A) + 16
        # of U, and the two subtractions by U of what they give and of the logits' distance
        size = np.abs(np.nan_to_num(want_logp, neginf=0.0))
        bound = ref.U * (18.0 + 1.4 * np.log2(max(A, 2)) + 3.0 * size + 2.0 * np.log(A))
        ref.check(host(logp), (want_logp, bound), "logp")
        again = torch.empty_like(actions)
        av.av_draw_actions(logits, torch.from_numpy(u).cuda(), again)
        assert torch.equal(again, actions)


def test_long_rows_in_graphs_with_workspaces():
    """A few long rows, whose parts meet in a workspace: two captured launches with one each."""
    f = dict(device="cuda")
    l = [torch.randn((3, 50000), **f) for _ in range(2)]
    ids = torch.arange(3, **f)

    def buffers():
        return [torch.zeros(3, **f), torch.zeros(3, **f), torch.zeros((3, 2), **f),
                torch.zeros((3, 9), **f), torch.zeros((3, 9), dtype=torch.int32, **f)]
    want, outs, graphs = [buffers(), buffers()], [buffers(), buffers()], []
    for v, w in zip(l, want):
        av.av_log_probs(v, ids, *w)
    torch.cuda.synchronize()
    for v, o in zip(l, outs):
        ws = torch.empty(av.av_log_probs_workspace(3, 50000, 9), dtype=torch.uint8, **f)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            av.av_log_probs(v, ids, *o, workspace=ws)
        graphs.append((g, ws))
    for _ in range(3):
        for g, _ in graphs:
            g.replay()
        again = buffers()
        av.av_log_probs(l[0], ids, *again)
        torch.cuda.synchronize()
        for o, w in zip(outs + [again], want + [want[0]]):
            for x, y in zip(o, w):
                assert torch.equal(x, y)
        for o in outs:
            for x in o:
                x.zero_()
    with pytest.raises(av.AvError):
        av.av_log_probs(l[0], ids, *again, workspace=torch.empty(64, dtype=torch.uint8, **f))


def test_draw_follows_the_distribution():
    """Numbers spread evenly over [0, 1) draw each choice as often as its probability says, to one
    draw either side of each border."""
    N = 4096
    p = np.array([0.1, 0.0, 0.4, 0.25, 0.25])
    with np.errstate(divide="ignore"):
        logits = torch.from_numpy(np.log(p)).float().cuda().expand(N, 5)
    u = (torch.arange(N, device="cuda") + 0.5) / N
    actions = torch.empty(N, dtype=torch.uint8, device="cuda")
    av.av_draw_actions(logits, u, actions)
    count = np.bincount(actions.cpu().numpy(), minlength=5)
    assert (np.abs(count - p * N) <= 2).all() and count[1] == 0


@pytest.mark.parametrize("A", [2, 5, 40, 200])
def test_draw_of_a_certain_action(A):
    """The log-probability of an action that is all but certain is small, and as exact as a large one.
    Relative to it: the other weights by (1 + d) 2 U of themselves, d <= 12 the distance of their logits,
    sixteen additions and the logarithm by 20 U."""
    r = np.random.default_rng(A)
    v = -r.uniform(9, 12, size=(300, A))
    v[:, 0] = 0.0
    v[7, 1] = 0.0                                # two of the largest
    logits, u = torch.from_numpy(v).float().cuda(), np.zeros(300, dtype=np.float32)
    actions = torch.empty(300, dtype=torch.uint8, device="cuda")
    logp = torch.empty(300, device="cuda")
    av.av_draw_actions(logits, torch.from_numpy(u).cuda(), actions, logp)
    l = host(logits)
    want = -np.log1p(np.exp(l[:, 1:]).sum(1))
    assert not actions.any()
    ref.check(host(logp), (want, ref.U * 46.0 * np.abs(want)), "logp")


def test_draw_close_to_a_border():
    """Numbers at and next to the borders between choices, where 32 bits do not tell the side."""
    for A in (5, 64, 200):
        N = 4 * A
        logits = torch.zeros((N, A), device="cuda")
        i = np.repeat(np.arange(A), 4)
        u = (i / A).astype(np.float32)
        u[1::4] = np.nextafter(u[1::4], 2.0, dtype=np.float32)
        u[2::4] = np.nextafter(u[2::4], -1.0, dtype=np.float32)
        u[3::4] += np.float32(2.0 ** -21)
        u = np.clip(u, 0.0, np.float32(1.0 - 2.0 ** -24))
        actions = torch.empty(N, dtype=torch.uint8, device="cuda")
        av.av_draw_actions(logits, torch.from_numpy(u).cuda(), actions)
        # equal weights: the first i with (i + 1) > u A, u and A exact in 64 bits
        want = np.minimum(np.floor(u.astype(np.float64) * A), A - 1)
        assert np.array_equal(actions.cpu().numpy(), want)


def test_binding_refuses():
    l = torch.zeros((4, 6), device="cuda")
    ids, f = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    st = torch.zeros((4, 2), device="cuda")
    top_i = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    bad = [
        lambda: av.av_log_probs(l.double(), ids, f),
        lambda: av.av_log_probs(l.t(), torch.zeros(6, dtype=torch.int64, device="cuda"),
                                torch.zeros(6, device="cuda")),
        lambda: av.av_log_probs(l, ids.to(torch.int16), f),
        lambda: av.av_log_probs(l, ids[:3], f),
        lambda: av.av_log_probs(l, ids, f[:3]),
        lambda: av.av_log_probs(l, ids),
        lambda: av.av_log_probs(l, ids, f, top_logp=st),
        lambda: av.av_log_probs(l, ids, f, top_logp=st, top_ids=top_i.long()),
        lambda: av.av_log_probs(l, ids, f, top_logp=torch.zeros((4, 33), device="cuda"),
                                top_ids=torch.zeros((4, 33), dtype=torch.int32, device="cuda")),
        lambda: av.av_log_probs_backward(l, ids, st, None, f, f, torch.empty_like(l)),
        lambda: av.av_log_probs_backward(l, None, st, f, f, f, torch.empty_like(l)),
        lambda: av.av_log_probs_backward(l, ids, st, f, f, f, torch.empty_like(l).half()),
        lambda: av.av_draw_actions(torch.zeros((4, 257), device="cuda"), f,
                                   torch.zeros(4, dtype=torch.uint8, device="cuda")),
        lambda: av.av_draw_actions(l, f, ids),
        lambda: av.av_draw_actions(l, f.double(), torch.zeros(4, dtype=torch.uint8, device="cuda")),
    ]
    for g in bad:
        with pytest.raises((TypeError, ValueError, av.AvError)):
            g()


def test_streams_and_graphs():
    l = torch.randn((300, 5000), device="cuda")
    ids = torch.arange(300, device="cuda")
    f = dict(device="cuda")
    outs = []
    for _ in range(2):
        outs.append([torch.zeros(300, **f), torch.zeros(300, **f), torch.zeros((300, 2), **f),
                     torch.zeros((300, 4), **f), torch.zeros((300, 4), dtype=torch.int32, **f),
                     torch.zeros_like(l), torch.zeros(300, dtype=torch.uint8, **f)])
    g, u = torch.randn(300, **f), torch.rand(300, **f)

    def call(o):
        av.av_log_probs(l, ids, *o[:5])
        av.av_log_probs_backward(l, ids, o[2], o[1], g, g, o[5])
        av.av_draw_actions(l[:, :200], u, o[6])
    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1])
    for _ in range(3):
        graph.replay()
        call(outs[0])
        torch.cuda.synchronize()
        for a, b in zip(*outs):
            assert torch.equal(a, b)
            b.zero_()


def test_an_agent_learns_from_a_rollout():
    """The operators together, as a policy gradient uses them: actions drawn for every step of a
    batch, returns of its rewards and done flags, the agent's memory over the rollout, the
    log-probabilities of the drawn actions, and the gradient back through all of it, against the same
    chain in 64 bits."""
    from paper_2407_04221_amd import inputs
    wl = inputs.WORKLOADS["c1"].with_(B=70, L=9)
    maps, rules, _ = inputs.make_all(wl.with_(T=2), 0, "planted")
    b = av.Batch.for_workload(wl)
    b.load_rules(*rules)
    b.reset(maps)
    T, B, D, w = 20, wl.B, 24, 5
    r = np.random.default_rng(5)
    obs_n = wl.C * w * w
    W1 = torch.from_numpy(r.normal(size=(obs_n, 2 * D)) * 0.1).float().cuda()
    W2 = torch.from_numpy(r.normal(size=(D, 5)) * 0.5).float().cuda()
    uniform = torch.from_numpy(r.random((T, B))).float().cuda()
    obs = b.observe(w).reshape(B, obs_n).float()
    state = torch.zeros((B, D), device="cuda")
    seen, acted, rewards, done, drawn_logp = [], [], [], [], []
    was_done = torch.zeros(B, dtype=torch.uint8, device="cuda")
    flags = []
    y1 = torch.empty((1, B, D), device="cuda")
    for t in range(T):                          # acting: one token of every environment at a time
        h = obs @ W1
        flags.append(was_done.clone())
        av.av_scan(h[None, :, :D], h[None, :, D:], y1, h0=state, last=state, cut=was_done[None],
                   form="gated")
        actions, logp = b.act(state @ W2, uniform[t])
        seen.append(obs)
        acted.append(actions)
        drawn_logp.append(logp)
        rew, dn, window = b.step_observe(actions[None], w)
        rewards.append(rew[0])
        done.append(dn[0])
        was_done = dn[0].clone()
        obs = window.reshape(B, obs_n).float()
    rewards, done, flags = torch.stack(rewards), torch.stack(done), torch.stack(flags)
    acted, drawn_logp = torch.stack(acted), torch.stack(drawn_logp)
    assert bool(done.any())
    # learning: the same states from one scan over the rollout
    ret = b.returns(rewards, done, 0.9)
    X = torch.stack(seen)
    h = X @ W1
    x, gate = h[:, :, :D], h[:, :, D:]
    y = torch.empty((T, B, D), device="cuda")
    av.av_scan(x, gate, y, cut=flags, form="gated")
    logits = (y.reshape(T * B, D) @ W2).contiguous()
    n = T * B
    logp, ent, st = (torch.empty(n, device="cuda"), torch.empty(n, device="cuda"),
                     torch.empty((n, 2), device="cuda"))
    av.av_log_probs(logits, acted.reshape(n), logp, ent, st)
    dlogits = torch.empty_like(logits)
    dlogp = (-ret / n).reshape(n)
    dent = torch.full((n,), -0.01 / n, device="cuda")
    av.av_log_probs_backward(logits, acted.reshape(n), st, ent, dlogp, dent, dlogits)
    dy = (dlogits @ W2.t()).view(T, B, D)
    dh = torch.empty_like(h)
    av.av_scan_backward(x, gate, y, dy, dh[:, :, :D], dh[:, :, D:], cut=flags, form="gated")
    dW1 = X.reshape(n, obs_n).t() @ dh.reshape(n, 2 * D)
    # in 64 bits, on the host, by torch's own differentiation
    V1, V2 = W1.double().cpu().requires_grad_(), W2.double().cpu().requires_grad_()
    s = torch.zeros((B, D), dtype=torch.float64)
    F, Xh, total, logps, acts = flags.cpu(), X.double().cpu(), 0.0, [], acted.cpu().long()
    rh = torch.zeros(B, dtype=torch.float64)
    rets = []
    for t in reversed(range(T)):
        rh = rewards[t].double().cpu() + 0.9 * rh * (done[t].cpu() == 0)
        rets.append(rh)
    rets = torch.stack(rets[::-1])
    for t in range(T):
        z = Xh[t] @ V1
        s = torch.where(F[t][:, None] != 0, 0.0, s)
        a = torch.sigmoid(z[:, D:])
        s = a * s + (1 - a) * z[:, :D]
        lp = torch.log_softmax(s @ V2, 1)
        own = lp.gather(1, acts[t][:, None])[:, 0]
        logps.append(own)
        H = -(lp.exp() * lp).sum(1)
        total = total - (rets[t] * own).sum() / n - 0.01 / n * H.sum()
    total.backward()
    logps = torch.stack(logps).detach()
    # 32-bit products over obs_n, 2 D and n terms between the operators, each term of order one at
    # most: n U with n the longest sum, and twenty steps of memory
    tol = (obs_n + D + 20 * 20) * ref.U * 4
    assert float((logp.view(T, B).double().cpu() - logps).abs().max()) < tol
    assert float((drawn_logp.double().cpu() - logps).abs().max()) < tol
    scale = float(V1.grad.abs().max())
    assert float((dW1.double().cpu() - V1.grad).abs().max()) < scale * (n + obs_n) * ref.U * 4
    b.close()
