"""The two weights of the gated form, a = 1 / (1 + exp(-g)) and 1 - a, in float32: a few roundings of
themselves, and |g| of them.

With U = 2^-24 a rounding: e = exp(-|g|) is 2^t with t = |g| log2 e, which the constant, off by 1.34e-8 =
0.23 U of itself, and the product's rounding put off by (0.23 + 1) U t, and so e by 1.23 U t ln 2 = 1.23 |g| U
of itself.  The power of two is off by 1 unit (2 U), 1 + e by U, the reciprocal by 2 U, the product by U and
the state's own product by U: 7 U, 8 U with what the terms leave out.  Below 2^-126 they count as 0."""
import numpy as np
import pytest
import torch

import learn_ref as ref
import paper_2407_04221_amd as av

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,B", [(1, 20011), (9, 2011)])
def test_weights(T, B):
    r = np.random.default_rng(1)
    g = r.uniform(-86.0, 86.0, size=(T, B, 1)).astype(np.float32)
    g[0, :8, 0] = [0.0, -0.0, 1e-30, -1e-30, 16.6, -16.6, 86.0, -86.0]
    gate = torch.from_numpy(g).cuda()
    one, zero = torch.ones_like(gate), torch.zeros_like(gate)
    cut = torch.ones((T, B), dtype=torch.uint8, device="cuda")
    rest, a = torch.empty_like(gate), torch.empty_like(gate)
    av.av_scan(one, gate, rest, cut=cut, form="gated")          # every step anew: (1 - a) x
    # the gradient of what came in: a times that of the state
    av.av_scan_backward(zero, gate, zero, one, a, None, cut=cut, form="gated")
    assert torch.equal(a, rest)                                 # dx = (1 - a) dy
    want = 1.0 / (1.0 + np.exp(g.astype(np.float64)))
    some = (8.0 + 1.25 * np.abs(g)) * ref.U
    ref.check(rest.double().cpu().numpy(), (want, some * want), "1 - a")
    for t in range(T):                                          # a, as one step's share of its state
        last = torch.empty((B, 1), device="cuda")
        y = torch.empty_like(gate[t:t + 1])
        av.av_scan(zero[t:t + 1], gate[t:t + 1], y, h0=one[t], last=last, form="gated")
        want = 1.0 / (1.0 + np.exp(-g[t].astype(np.float64)))
        ref.check(last.double().cpu().numpy(), (want, some[t] * want), "a")


def test_ends():
    """Gates so far out that a weight is 0, and infinite ones."""
    g = torch.tensor([200.0, -200.0, float("inf"), -float("inf")], device="cuda").view(1, 4, 1)
    y, last = torch.empty_like(g), torch.empty((4, 1), device="cuda")
    av.av_scan(torch.full_like(g, 3.0), g, y, h0=torch.full((4, 1), 5.0, device="cuda"), last=last,
               form="gated")
    assert last.ravel().tolist() == [5.0, 3.0, 5.0, 3.0]
