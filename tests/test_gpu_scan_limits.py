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
