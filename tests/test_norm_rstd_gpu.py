"""The norm's s = (mean h^2 + eps)^(-1/2) where every step has an exact float32: a rounded root and a rounded reciprocal, to the last bit."""
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [64, 4096, 8192, 16384, 32768])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_of_one_value(H, dtype):
    """A row of k <= 255: k^2 has 16 bits, and a sum of n of them is exact while the odd part of n has no more than 8, as those of all
    partial sums here; their mean is k^2, its root k."""
    k = torch.arange(1, 256, device="cuda")
    x = k.to(dtype)[:, None].repeat(1, H)
    s = b.dvp_rms_norm(x, torch.ones(H, device="cuda"), eps=0.0).rstd
    assert torch.equal(s.double(), (1.0 / k.double()).float().double())


@pytest.mark.parametrize("H", [64, 4096])
def test_roots_that_are_rounded(H):
    """Means that float32 holds exactly: a root and then a reciprocal, each rounded once."""
    k = torch.arange(1, 4096, device="cuda")
    # rows of ones with one entry e: mean = (H - 1 + e^2) / H
    x = torch.ones(4095, H, device="cuda")
    x[:, 3] = k.float()
    mean = (x.double().square().sum(1) / H).float()
    exact = x.double().square().sum(1) < 2.0 ** 24
    s = b.dvp_rms_norm(x, torch.ones(H, device="cuda"), eps=0.0).rstd
    want = (1.0 / mean.double().sqrt().float().double()).float()
    assert torch.equal(s[exact], want[exact])
