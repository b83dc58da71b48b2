"""Rows long enough that their nucleus' border is guessed from a part of them: what the guess, the sums behind it and the list around it
can get wrong."""
import pytest
import torch

from test_sample_gpu import DTYPES, _check, _uniform

pytestmark = pytest.mark.gpu
V = 140_001


def _rows(dtype, seed):
    """Eight rows from flat to decided, half of them with tokens that are not to be drawn, in an order that is none."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(8, V, generator=g, device="cuda")
    z *= torch.tensor([0.0, 0.01, 0.5, 1.0, 2.0, 3.0, 5.0, 2.0], device="cuda")[:, None]
    z += torch.tensor([0.0, 3.0, -40.0, 100.0, 0.0, -7.0, 0.0, 0.0], device="cuda")[:, None]
    z[7].copy_(z[7].sort().values)      # what the part of a row says of it is wrong as to the order, not the values
    z[4:7, ::3] = float("-inf")
    z[3, 5000:] = float("-inf")
    return z.to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("top_p", [0.03, 0.5, 0.9, 0.95, 0.999, 0.9999999])
def test_nucleus(dtype, top_p):
    _check(_rows(dtype, 3), _uniform(8), hints=(1, 2), top_p=top_p)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("temperature", [2.0 ** -100, 1e-3, 0.25, 30.0, 1e4, 2.0 ** 100])
def test_nucleus_at_a_temperature(dtype, temperature):
    _check(_rows(dtype, 4), _uniform(8, 5), hints=(1, 2), top_p=0.9, temperature=temperature)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("settings", [dict(top_k=300), dict(top_k=3000), dict(top_k=100_000, top_p=0.9), dict(rho=1e-3, top_p=0.9), dict()],
                         ids=str)
def test_other_cuts(dtype, settings):
    _check(_rows(dtype, 6), _uniform(8, 7), hints=(1, 2, 8), **settings)


def test_draws_at_every_place():
    """One row, many random numbers: those whose border is near go the long way and agree with the others."""
    z = _rows("bf16", 8)[5:6].expand(64, V).contiguous()
    u = torch.linspace(0, 1, 64, device="cuda")
    _check(z, u, hints=(1,), top_p=0.95)
    _check(z, u, hints=(1, 4))


def test_results_do_not_change_from_run_to_run():
    from paper_2512_23087_b200 import binding as b
    z = _rows("bf16", 9).repeat(40, 1)
    u = _uniform(z.shape[0], 11)
    for settings in (dict(), dict(top_p=0.95), dict(top_k=700)):
        first = b.dvp_sample(z, u, **settings)
        for _ in range(3):
            again = b.dvp_sample(z, u, **settings)
            for name in ("ids", "count", "logp", "logp_mp"):
                assert torch.equal(getattr(first, name), getattr(again, name)), (settings, name)
