"""Arguments of the learner's operators that are refused, all on the host before any device
work (no GPU here; the pointers are never followed)."""
import ctypes

import pytest

import paper_2407_04221_amd as av

P = ctypes.c_void_p(4096)        # a well aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    return av.load_library()


def scan_config(**kw):
    c = av.av_scan_config()
    base = dict(steps=4, rows=2, width=8, x_step=16, x_row=8, gate_step=16, gate_row=8, y_step=16,
                y_row=8, dy_step=16, dy_row=8, dx_step=16, dx_row=8, dgate_step=16, dgate_row=8,
                cut_step=2, cut_row=1)
    base.update(kw)
    for k, v in base.items():
        setattr(c, k, v)
    return ctypes.byref(c)


BAD_SCANS = [dict(steps=-1), dict(steps=(1 << 30) + 1), dict(rows=1 << 14, width=(1 << 14) + 1), dict(rows=-1), dict(width=0),
             dict(rows=1 << 16, width=1 << 15), dict(rows=1 << 40, width=1 << 40), dict(dtype=3),
             dict(dtype=-1), dict(form=2), dict(reverse=2), dict(gate_per_value=-1),
             dict(x_step=1 << 60), dict(x_row=-8), dict(gate_step=-16)]


@pytest.mark.parametrize("bad", BAD_SCANS + [dict(y_step=0), dict(y_row=7), dict(y_step=4)])
def test_scan_refuses(lib, bad):
    assert lib.av_scan(scan_config(**bad), P, P, P, P, P, P, P, 1 << 20) == av.AV_EINVAL
    assert av.av_last_error()


@pytest.mark.parametrize("bad", BAD_SCANS + [dict(dx_step=0), dict(dx_row=7), dict(dgate_step=4),
                                             dict(dgate_row=0)])
def test_scan_backward_refuses(lib, bad):
    assert lib.av_scan_backward(scan_config(**bad), P, P, P, P, P, P, P, P, P, P, P,
                                1 << 20) == av.AV_EINVAL
    assert av.av_last_error()


def test_scan_refuses_missing_and_misaligned(lib):
    odd = ctypes.c_void_p(4097)
    for i in (0, 1, 4):                                       # x, gate, y
        args = [P, P, None, None, P, None, None]
        for p in (None, odd):
            args[i] = p
            assert lib.av_scan(scan_config(), *args, 0) == av.AV_EINVAL
    assert lib.av_scan(None, P, P, None, None, P, None, None, 0) == av.AV_EINVAL
    for i in (1, 4, 5, 7):                                    # gate, y, dy, dx
        args = [P, P, None, None, P, P, None, P, P, None, None]
        for p in (None, odd):
            args[i] = p
            assert lib.av_scan_backward(scan_config(), *args, 0) == av.AV_EINVAL
    args = [None, P, None, None, P, P, None, P, P, None, None]
    assert lib.av_scan_backward(scan_config(form=1), *args, 0) == av.AV_EINVAL   # gated reads x
    assert lib.av_scan(scan_config(), P, P, None, odd, P, None, None, 0) == av.AV_EINVAL


def test_scan_workspace(lib):
    n = ctypes.c_size_t(1)
    assert lib.av_scan_workspace(scan_config(), 0, ctypes.byref(n)) == av.AV_OK
    assert n.value == 0                                       # a short one needs none
    assert lib.av_scan_workspace(scan_config(), 0, None) == av.AV_EINVAL
    assert lib.av_scan_workspace(None, 0, ctypes.byref(n)) == av.AV_EINVAL
    assert lib.av_scan_workspace(scan_config(steps=-1), 0, ctypes.byref(n)) == av.AV_EINVAL
    long = dict(steps=1 << 16, cut_step=2)
    assert lib.av_scan_workspace(scan_config(**long), 0, ctypes.byref(n)) == av.AV_OK
    assert n.value > 0
    for ws, size in ((None, n.value), (P, n.value - 1), (ctypes.c_void_p(4104), n.value)):
        assert lib.av_scan(scan_config(**long), P, P, None, None, P, None, ws,
                           size) == av.AV_EINVAL
        assert "workspace" in av.av_last_error()
    # the sums of a gate per value need one however short
    assert lib.av_scan_workspace(scan_config(gate_per_value=1), 1, ctypes.byref(n)) == av.AV_OK
    assert n.value > 0
    assert av.av_scan_workspace(1 << 16, 2, 8) > 0 == av.av_scan_workspace(4, 2, 8)


def test_many_steps_of_far_rows(lib):
    """Rows past a wave's 32-bit distances take their steps one by one: not too many of them."""
    apart = dict(steps=(1 << 16) + 1, rows=3, width=4, x_row=1 << 29, x_step=4, y_step=12, y_row=4,
                 gate_per_value=1)
    n = ctypes.c_size_t(0)
    assert lib.av_scan_workspace(scan_config(**apart), 0, ctypes.byref(n)) == av.AV_OK
    assert lib.av_scan(scan_config(**apart), P, P, None, None, P, None, P, n.value) == av.AV_EINVAL
    assert "apart" in av.av_last_error()
    far = dict(apart, x_row=4, x_step=12, dx_step=12, dx_row=4, dy_step=4, dy_row=1 << 29)
    assert lib.av_scan_workspace(scan_config(**far), 1, ctypes.byref(n)) == av.AV_OK
    assert lib.av_scan_backward(scan_config(**far), P, P, None, None, P, P, None, P, P, None, P,
                                n.value) == av.AV_EINVAL
    assert "apart" in av.av_last_error()


def tokens_config(**kw):
    c = av.av_tokens_config()
    base = dict(rows=3, choices=5, row_stride=5, drow_stride=5)
    base.update(kw)
    for k, v in base.items():
        setattr(c, k, v)
    return ctypes.byref(c)


BAD_TOKENS = [dict(rows=-1), dict(rows=1 << 31), dict(choices=0), dict(choices=(1 << 31) - 1024),
              dict(dtype=3), dict(ids_type=3), dict(ids_type=-1), dict(row_stride=1 << 60), dict(row_stride=-5)]


@pytest.mark.parametrize("bad", BAD_TOKENS)
def test_tokens_refuse(lib, bad):
    assert lib.av_log_probs(tokens_config(**bad), P, P, P, P, P, None, None, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs_backward(tokens_config(**bad), P, P, P, P, P, P, P) == av.AV_EINVAL
    assert lib.av_draw_actions(tokens_config(**bad), P, P, P, P) == av.AV_EINVAL
    assert av.av_last_error()


def test_tokens_refuse_missing_and_misaligned(lib):
    odd, four = ctypes.c_void_p(4097), ctypes.c_void_p(4100)
    cfg = tokens_config()
    assert lib.av_log_probs(None, P, P, P, P, P, None, None, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(cfg, None, P, P, P, P, None, None, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(cfg, odd, P, P, P, P, None, None, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(cfg, P, None, P, P, P, None, None, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(cfg, P, P, None, P, P, None, None, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(cfg, P, P, P, P, four, None, None, None, 0) == av.AV_EINVAL
    for top in (-1, 33):
        assert lib.av_log_probs(tokens_config(top=top), P, P, P, P, P, P, P, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(tokens_config(top=1), P, P, P, P, P, None, P, None, 0) == av.AV_EINVAL
    assert lib.av_log_probs(tokens_config(ids_type=2), P, four, P, P, P, None,
                            None, None, 0) == av.AV_EINVAL
    good = [P, P, P, P, P, P, P]
    for i in (0, 1, 2, 3, 6):             # logits, ids, stats, entropy, dlogits
        args = list(good)
        args[i] = None
        assert lib.av_log_probs_backward(cfg, *args) == av.AV_EINVAL
        args[i] = odd
        if i != 1:
            assert lib.av_log_probs_backward(cfg, *args) == av.AV_EINVAL
    for bad in (dict(drow_stride=4), dict(drow_stride=0), dict(drow_stride=1 << 60)):
        assert lib.av_log_probs_backward(tokens_config(**bad), *good) == av.AV_EINVAL
    for i in (0, 1, 2):
        args = [P, P, P, None]
        args[i] = None
        assert lib.av_draw_actions(cfg, *args) == av.AV_EINVAL
    assert lib.av_draw_actions(tokens_config(choices=257), P, P, P, P) == av.AV_EINVAL


def test_tokens_workspace(lib):
    n = ctypes.c_size_t(1)
    assert lib.av_log_probs_workspace(tokens_config(), ctypes.byref(n)) == av.AV_OK
    assert n.value == 0
    assert lib.av_log_probs_workspace(tokens_config(), None) == av.AV_EINVAL
    assert lib.av_log_probs_workspace(None, ctypes.byref(n)) == av.AV_EINVAL
    assert lib.av_log_probs_workspace(tokens_config(top=33), ctypes.byref(n)) == av.AV_EINVAL
    few = dict(choices=100000, row_stride=100000, top=3)
    assert lib.av_log_probs_workspace(tokens_config(**few), ctypes.byref(n)) == av.AV_OK
    assert n.value > 0
    assert n.value == av.av_log_probs_workspace(3, 100000, 3)
    for ws, size in ((None, n.value), (P, n.value - 1), (ctypes.c_void_p(4104), n.value)):
        assert lib.av_log_probs(tokens_config(**few), P, P, P, P, P, P, P, ws,
                                size) == av.AV_EINVAL
        assert "workspace" in av.av_last_error()


def test_no_rows_need_nothing(lib):
    empty = tokens_config(rows=0)
    assert lib.av_log_probs(empty, None, None, None, None, None, None, None, None, 0) == av.AV_OK
    assert lib.av_log_probs_backward(empty, None, None, None, None, None, None, None) == av.AV_OK
    assert lib.av_draw_actions(empty, None, None, None, None) == av.AV_OK


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((2, 1, 3))
    with pytest.raises(TypeError):
        av.av_scan(x, x, x)
    with pytest.raises(TypeError):
        av.av_log_probs(torch.zeros((2, 3)))
    with pytest.raises(TypeError):
        av.av_draw_actions(torch.zeros((2, 3)), torch.zeros(2), torch.zeros(2, dtype=torch.uint8))


def test_packed_configs_have_the_structs_layout():
    """The binding packs its configs in one step: field for field what the structs hold."""
    for pack, struct in ((av._SCAN, av.av_scan_config), (av._TOKENS, av.av_tokens_config)):
        assert pack.size == ctypes.sizeof(struct)
        values = list(range(1, len(struct._fields_) + 1))
        c = struct.from_buffer_copy(pack.pack(*values))
        assert [getattr(c, f) for f, _ in struct._fields_] == values
