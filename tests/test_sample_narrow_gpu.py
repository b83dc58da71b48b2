"""Nuclei whose border is hard to bracket: tens of thousands of logits in a range so narrow that a histogram of the row's whole range says
little of them, aims next to the row's whole sum, and clusters at both ends of the range with the aim next to the first one's sum."""
import pytest
import torch

from test_sample_gpu import DTYPES, F32, _check, _uniform

pytestmark = pytest.mark.gpu


def _narrow(V, centre, scale, seed, masked=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = centre + scale * torch.randn(2, V, generator=g, device="cuda")
    return z.masked_fill(torch.rand(2, V, generator=g, device="cuda") < masked, float("-inf"))


@pytest.mark.parametrize("top_p", [0.3, 0.9999, 0.999999, 0.9999999, 1 - 1e-9])
@pytest.mark.parametrize("V,centre,scale,temperature", [(127755, 10.0, 1.25e-3, 1.0), (151840, 10.0, 2e-3, 2.5), (10114, 10.0, 2e-3, 1.0),
                                                        (102801, 1000.0, 0.055, 300.0), (300001, -3.0, 1e-4, 0.7)])
def test_logits_in_a_narrow_range(V, centre, scale, temperature, top_p):
    z = _narrow(V, centre, scale, V, 0.3)
    _check(z, _uniform(2), hints=(1, 2, 8), top_p=top_p, temperature=temperature)


@pytest.mark.parametrize("top_p", [0.9999, 0.999999, 0.9999999, 1 - 1e-8, 1 - 1e-9])
@pytest.mark.parametrize("dtype,centre", [("f16", 20000.0), ("bf16", 3000.0)])
def test_a_few_values(dtype, centre, top_p):
    _check(_narrow(10114, centre, 8.4, 5, 0.6).to(DTYPES[dtype]), _uniform(2), hints=(1, 2), top_p=top_p, temperature=2.5)


@pytest.mark.parametrize("beside", [-3e-3, -1e-4, -1e-6, 0.0, 1e-6, 1e-4, 3e-3])
@pytest.mark.parametrize("high,low,temperature", [(10.0, -10.0, 30.0), (10.0, 9.0, 1.0), (-1.0, -9.0, 4.0), (1000.0, -1000.0, 2.0 ** 20)])
def test_clusters_at_both_ends(high, low, temperature, beside):
    """30,000 logits near each end; the aim is the first cluster's sum, or that and a little."""
    g = torch.Generator(device="cuda").manual_seed(7)
    n = 30000
    z = torch.cat([high + 1e-3 * torch.randn(n, generator=g, device="cuda"), low + 1e-3 * torch.randn(n, generator=g, device="cuda")])
    z = z[torch.randperm(2 * n, generator=g, device="cuda")][None].to(F32)
    w = torch.exp((z.double() - z.double().max()) / temperature)
    # between two logits' sums, so that the order of the definition's additions does not matter
    share = float((w[z > (high + low) / 2].sum() - 0.5 * float(w[z > (high + low) / 2].min())) / w.sum())
    _check(z, _uniform(1), hints=(1, 4), top_p=share * (1 + beside), temperature=temperature)


def test_one_logit_far_below_many():
    """What lies far below the others is kept or not by the aim alone."""
    z = _narrow(64065, 10.0, 1e-3, 9)
    z[:, 777] = -6.0
    z[:, 888] = -7.0
    for top_p in (0.99, 0.9999999, 1 - 1e-11, 1 - 5e-12):
        _check(z, _uniform(2), hints=(1, 2), top_p=top_p)


def test_cuts_behind_other_cuts():
    z = _narrow(100003, 10.0, 2e-3, 3)
    for settings in (dict(top_k=60000, top_p=0.9999999), dict(rho=0.9985, top_p=0.9999999), dict(top_k=50000, rho=0.999, top_p=0.999999)):
        _check(z, _uniform(2), hints=(1, 2), **settings)
