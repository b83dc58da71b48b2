"""Rows of which a nucleus keeps a small part: ln pi of the kept is as good as the kept logits' sum, whatever the whole row's is."""
import pytest
import torch

from test_sample_gpu import DTYPES, _check, _uniform

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,V", [("bf16", 436), ("f32", 5000), ("bf16", 100_003), ("f32", 262_144), ("f16", 600_011)])
@pytest.mark.parametrize("scale", [0.02, 0.5, 2.0])
@pytest.mark.parametrize("top_p", [1e-5, 1e-4, 1e-3, 0.01, 0.1, 0.4])
def test_few_kept(dtype, V, scale, top_p):
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (scale * torch.randn(6, V, generator=g, device="cuda")).to(DTYPES[dtype])
    _check(z, _uniform(6, 2), hints=(1, 2), top_p=top_p)
