"""Strides that av_scan's header calls unused take no part in what is refused (no GPU here: the calls are
refused for the workspace that they lack, which is looked at after the strides)."""
import ctypes

import paper_2407_04221_amd as av

P = ctypes.c_void_p(4096)        # a well aligned address that nothing reads


def config(**kw):
    c = av.av_scan_config()
    base = dict(steps=4, rows=3, width=4, gate_per_value=1, x_step=12, x_row=4, y_step=12, y_row=4,
                dy_step=12, dy_row=4, dx_step=12, dx_row=4, cut_step=3, cut_row=1)
    base.update(kw)
    for k, v in base.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def forward(**kw):
    rc = av.load_library().av_scan(config(**kw), P, P, P, None, P, None, None, 0)
    return rc, av.av_last_error()


def backward(**kw):
    rc = av.load_library().av_scan_backward(config(**kw), P, P, P, None, P, P, None, P, P, None, None, 0)
    return rc, av.av_last_error()


MANY = (1 << 16) + 1             # more steps than rows far apart may have


def test_strides_of_a_gate_per_value():
    for kw in (dict(gate_step=-1), dict(gate_row=-8), dict(gate_step=1 << 60), dict(dgate_step=-1),
               dict(dgate_row=1 << 60)):
        rc, why = backward(**kw)
        assert rc == av.AV_EINVAL and "workspace" in why, (kw, why)
        rc, why = forward(steps=MANY, **kw)
        assert rc == av.AV_EINVAL and "workspace" in why, (kw, why)
    for kw in (dict(gate_row=1 << 31), dict(dgate_row=1 << 31)):
        for call in (forward, backward):
            rc, why = call(steps=MANY, **kw)
            assert rc == av.AV_EINVAL and "workspace" in why, (kw, why)


def test_rows_of_an_input_that_is_not_read():
    """x in the gradient of the linear form."""
    rc, why = backward(steps=MANY, x_row=1 << 31)
    assert rc == av.AV_EINVAL and "workspace" in why
    rc, why = backward(steps=MANY, x_row=1 << 31, form=av.AV_SCAN_GATED)
    assert rc == av.AV_EINVAL and "apart" in why


def test_rows_of_flags_are_bytes():
    """Three rows of flags 2^29 bytes apart lie within 2^32 bytes; 2^31 apart they do not."""
    for call in (forward, backward):
        rc, why = call(steps=MANY, cut_row=1 << 29)
        assert rc == av.AV_EINVAL and "workspace" in why, why
        rc, why = call(steps=MANY, cut_row=1 << 31)
        assert rc == av.AV_EINVAL and "apart" in why, why
