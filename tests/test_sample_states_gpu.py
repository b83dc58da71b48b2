"""Draws in the bounds-checking build, which also notes a draw that takes sums for the first sweep's after another pass has replaced
them: rows whose nucleus' border lies among more logits than the list holds, at the first bracket and at the next."""
import pytest
import torch

from paper_2512_23087_b200 import binding

from test_sample_gpu import DTYPES, _check, _uniform

pytestmark = pytest.mark.gpu


@pytest.fixture()
def checked():
    with binding.bounds_checking_library():
        assert binding.dvp_debug_bounds_status() == 0
        yield
        assert binding.dvp_debug_bounds_status() == 0


def _dense(V, dtype, centre, scale):
    g = torch.Generator(device="cuda").manual_seed(11)
    return (centre + scale * torch.randn(3, V, generator=g, device="cuda")).to(DTYPES[dtype])


@pytest.mark.parametrize("V", [9001, 100_003, 600_011])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("centre,scale", [(0.0, 1e-6), (1000.0, 1e-3), (-7.0, 0.05), (0.0, 0.5), (0.0, 3.0), (0.0, 30.0)])
def test_dense_borders(checked, V, dtype, centre, scale):
    z = _dense(V, dtype, centre, scale)
    for top_p in (0.5, 0.95):
        _check(z, _uniform(3), hints=(1, 2), top_p=top_p)


@pytest.mark.parametrize("settings", [dict(), dict(top_k=700), dict(top_k=30000, top_p=0.9), dict(rho=1e-2, top_p=0.9), dict(rho=0.2)], ids=str)
def test_other_cuts(checked, settings):
    _check(_dense(100_003, "f32", -7.0, 0.05), _uniform(3), hints=(1, 4), **settings)
    _check(_dense(100_003, "bf16", 0.0, 3.0), _uniform(3), hints=(1, 4), **settings)
