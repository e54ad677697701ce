"""av_scan and av_scan_backward at the edges of their layouts and sizes: whole numbers, so that every sum is
exact in 32 bits and compared bit for bit."""
import pytest
import torch

import paper_2407_04221_amd as av

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,D", [(600, 4), (40, 300)])
def test_rows_of_flags_far_apart(T, D):
    """Flags of neighbouring rows 2^29 bytes apart, as packed ones give."""
    apart = (1 << 29) + 5
    near = (torch.rand((T, 3), device="cuda") < 0.1).to(torch.uint8)
    cut = torch.empty(2 * apart + T, dtype=torch.uint8, device="cuda").as_strided((T, 3), (1, apart))
    cut.copy_(near)
    x = torch.randint(-3, 4, (T, 3, D), device="cuda").float()
    gate = torch.ones((T, 3, D), device="cuda")
    out = [[torch.empty_like(x) for _ in range(3)] for _ in range(2)]
    for flags, (y, dx, dgate) in zip((near, cut), out):
        av.av_scan(x, gate, y, cut=flags)
        av.av_scan_backward(x, gate, y, x, dx, dgate, cut=flags)
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1, 2])
def test_widest_gate_per_value(T):
    """2^26 gates and more, each summed over the steps: with 1024 threads for sixteen of them, one launch
    for all would pass 2^32 threads."""
    D = (1 << 26) + 3
    kw = dict(dtype=torch.float16, device="cuda")
    x, dy = torch.empty((T, 1, D), **kw), torch.empty((T, 1, D), **kw)
    i = torch.arange(D, device="cuda")
    for t in range(T):
        x[t, 0], dy[t, 0] = i % 5 - 2, i % 7 - 3 + t
    gate, h0 = (i % 3 - 1).half(), (i % 11 - 5).float()[None]
    y, dx, dgate = torch.empty_like(x), torch.empty_like(x), torch.full_like(gate, 9.0)
    av.av_scan(x, gate, y, h0=h0)
    av.av_scan_backward(x, gate, y, dy, dx, dgate, h0=h0)
    # lam_t = dy_t + gate lam_{t+1}, dgate = sum lam_t s_{t-1}: below 2^11 in size
    lam, want = dy[T - 1, 0].float(), 0.0
    for t in reversed(range(T)):
        want = want + lam * (y[t - 1, 0].float() if t else h0[0])
        if t:
            lam = dy[t - 1, 0].float() + gate.float() * lam
    assert torch.equal(dgate.float(), want)
