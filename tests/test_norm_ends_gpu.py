"""Inputs that end where mapped memory ends: a vector read past its end, by as little as one element, would be no error of the result, but a
fault.  A block of the allocator's that lies at the end of its segment holds the input in its last bytes."""
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16, FP8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _at_the_end(v):
    """A copy of `v` whose last element is the last of a segment: an allocation of 20 MB has one of its own."""
    n = v.numel() * v.element_size()
    torch.cuda.empty_cache()
    out = torch.empty(20 << 20, dtype=torch.uint8, device="cuda")[(20 << 20) - n:].view(v.dtype).view(v.shape)
    return out.copy_(v)


def _normal(*shape, seed=1):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def test_guarded_loads_are_ordinary_ones():
    """On the CPU: loads that stand behind a comparison with a row's end are not of the kind that may be executed ahead of it."""
    for name in ("dvp_norm.cu", "dvp_sample.cu", "dvp_gemm_fp8.cu"):
        text = open(os.path.join(ROOT, "paper_2512_23087_b200", "csrc", name)).read()
        text = re.sub(r"/\*.*?\*/|//[^\n]*", "", text, flags=re.S)
        # the 8-bit product's scales: a row that does not exist has the first one's address, so that any order of the two is right
        left = [line.strip() for line in text.splitlines() if "__ldg(" in line]
        assert all(re.search(r"__ldg\(s[ab]( \+ (next|ks))?\)", line) for line in left), left
        assert not left or name == "dvp_gemm_fp8.cu"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,weight", [(F16, F32), (BF16, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("H", [1, 2, 100, 304, 1000, 4096, 8200])
def test_norm_and_backward(dtype, weight, H):
    from paper_2512_23087_b200 import binding as b
    T = 24
    x, dy = (2 * _normal(T, H)).to(dtype), _normal(T, H, seed=2)
    w = (1 + 0.2 * _normal(H, seed=3)).to(weight)
    want, want8 = b.dvp_rms_norm(x, w, residual=x), b.dvp_rms_norm(x, w, out_dtype=FP8)
    back = b.dvp_rms_norm_backward(dy, x, w, want.rstd, d_residual=x)
    for which in range(4):
        X, W, D, R = x, w, dy, want.rstd
        if which == 0:
            W = _at_the_end(w)
        elif which == 1:
            X = _at_the_end(x)
        elif which == 2:
            D = _at_the_end(dy)
        else:
            R = _at_the_end(R)
        got, got8 = b.dvp_rms_norm(X, W, residual=X), b.dvp_rms_norm(X, W, out_dtype=FP8)
        again = b.dvp_rms_norm_backward(D, X, W, R, d_residual=X)
        torch.cuda.synchronize()
        # an input that no vector fits any more has the sums of another kernel, off by float32's roundings of some hundred terms
        close = dict(rtol=2.0 ** -6 if dtype != F32 else 1e-4, atol=1e-3)
        torch.testing.assert_close(got.y.float(), want.y.float(), **close)
        torch.testing.assert_close(got8.scale, want8.scale, rtol=1e-5, atol=0)
        torch.testing.assert_close(again.d_x.float(), back.d_x.float(), **close)
        torch.testing.assert_close(again.d_weight, back.d_weight, rtol=1e-3, atol=1e-3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 4), (1, 128), (17, 132), (130, 1000), (129, 4100)])
def test_quantiser(dtype, block_rows, rows, cols):
    from paper_2512_23087_b200 import binding as b
    x = _normal(rows, cols).to(dtype)
    want, got = b.dvp_quantize_fp8(x, block_rows=block_rows), b.dvp_quantize_fp8(_at_the_end(x), block_rows=block_rows)
    assert torch.equal(got.scale, want.scale) and torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8))
