"""Masked choices take no gradient, whatever comes in from outside: a loss over rows without any choice has
infinities and NaN of its own (a log-probability of -inf, a ratio of two of them)."""
import numpy as np
import pytest
import torch

import learn_ref as ref
import paper_2407_04221_amd as av

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("N,A", [(40, 5), (40, 16), (40, 30), (40, 200), (20, 1500), (20, 2500), (7, 20000)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf"), 3.0e38])
def test_masked_choices_take_none(N, A, dtype, what):
    r = np.random.default_rng(A)
    v = torch.from_numpy(r.normal(size=(N, A)))
    off = torch.from_numpy(r.random((N, A)) < 0.4)
    off[:, 0] = False
    off[1] = off[4] = True                       # no choice at all
    v[off] = -np.inf
    v[2, A - 1] = np.nan                         # NaN throughout, masked choices too
    logits = v.to(TYPES[dtype]).cuda()
    ids = torch.from_numpy(r.integers(0, A, size=N)).cuda()
    f = dict(dtype=torch.float32, device="cuda")
    logp, ent, st = torch.empty(N, **f), torch.empty(N, **f), torch.empty((N, 2), **f)
    av.av_log_probs(logits, ids, logp, ent, st)
    # rows 3 to 5 and the empty row 1 get something that is no gradient, by either way in
    strange, g = torch.zeros(N, **f), torch.from_numpy(r.normal(size=N)).float().cuda()
    strange[1] = strange[3] = strange[4] = what
    mask = off.cuda()
    mask[2] = False
    for dlogp, dent in ((g + strange, g), (g, g + strange), (g + strange, None), (None, g + strange)):
        d = torch.full_like(logits, 7.0)
        av.av_log_probs_backward(logits, ids, st, ent, dlogp, dent, d)
        assert (d[mask] == 0).all()
        assert torch.isnan(d[2]).all()
        # the other rows are as ever
        keep = [n for n in range(N) if n not in (1, 2, 3, 4)]
        h = lambda t: None if t is None else t[keep].double().cpu().numpy()
        want = ref.tokens(h(logits), ids[keep].cpu().numpy(), h(dlogp), h(dent), 0, dtype)
        ref.check(h(d), want["dlogits"], "dlogits", dtype)
