"""8-bit values and scales are float32's quotients rounded to nearest, ties to even, to the last bit: c = amax / 448, q = e4m3(y / c)."""
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu
F32, BF16, FP8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _want(y, block_rows=1):
    """Scales and values by IEEE divisions, of tensors on the host (a tensor divided by a number there may become a product elsewhere)."""
    rows, cols = y.shape
    n, m = -(-cols // 128), -(-rows // block_rows)
    y = torch.nn.functional.pad(y, (0, n * 128 - cols, 0, m * block_rows - rows)).cpu()
    amax = y.view(m, block_rows, n, 128).abs().amax((1, 3)).clamp(min=2.0 ** -96)
    # float32's quotient is the rounding of double's: 53 bits are more than twice 24 and 2
    c = (amax.double() / 448.0).float()
    per = c.repeat_interleave(block_rows, 0).repeat_interleave(128, 1)
    return (y.double() / per.double()).float().to(FP8)[:rows, :cols], c


def _borders(cols, seed, scales=0):
    """Values c t, exact in float32, with t half way between two values of e4m3, and their neighbours; the largest of 128 is 448 c."""
    g = torch.Generator().manual_seed(seed)
    n = -(-cols // 128)
    c = torch.randint(1, 2 ** 14, (n, 1), generator=torch.Generator().manual_seed(scales)) * 2 + 1   # odd, up to 15 bits
    t = (torch.randint(8, 16, (n, 128), generator=g) * 2 + 1).double() * torch.exp2(torch.randint(-9, 4, (n, 128), generator=g).double())
    v = (c * t).float()
    assert torch.equal(v.double(), c * t)
    way = torch.randint(-1, 2, (n, 128), generator=g)
    v = torch.where(way == 0, v, torch.nextafter(v, torch.where(way < 0, 0.0, 1e30)))
    v *= torch.randint(0, 2, (n, 128), generator=g) * 2 - 1
    v[:, 0] = 448.0 * c[:, 0]
    return v.flatten()[:cols]


@pytest.mark.parametrize("H", [128, 2048, 4096, 8192, 16384, 32768])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("odd", [False, True])
def test_norm_at_the_borders(H, dtype, odd):
    """Rows of ones and minus ones: the mean square is 1, its root is 1, and y is the weight."""
    weight = _borders(H, H, H)
    x = torch.ones(3, H + odd, dtype=dtype, device="cuda")[:, :H]   # a stride that no vector fits
    x[1] = -1
    res = b.dvp_rms_norm(x, weight.cuda(), eps=0.0, out_dtype=FP8)
    assert (res.rstd == 1).all()
    q, c = _want(x.cpu().float() * weight)
    assert torch.equal(res.scale.cpu(), c)
    assert torch.equal(res.y.cpu().view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("cols", [128, 300, 4096])
def test_quantiser_at_the_borders(block_rows, cols):
    x = torch.stack([_borders(cols, r, r if block_rows == 1 else 0) for r in range(128)])
    res = b.dvp_quantize_fp8(x.cuda(), block_rows=block_rows)
    q, c = _want(x, block_rows)
    assert torch.equal(res.scale.cpu(), c)
    assert torch.equal(res.q.cpu().view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("H", [256, 1000, 4096, 5003])
def test_norm_in_8_bits_is_the_quantiser_of_the_norm(H):
    g = torch.Generator(device="cuda").manual_seed(H)
    x = torch.randn(2000, H, generator=g, device="cuda").to(BF16)
    w = 1 + 0.2 * torch.randn(H, generator=g, device="cuda")
    got = b.dvp_rms_norm(x, w, out_dtype=FP8)
    want = b.dvp_quantize_fp8(b.dvp_rms_norm(x, w, out_dtype=F32).y, block_rows=1)
    assert torch.equal(got.scale, want.scale)
    assert torch.equal(got.y.view(torch.uint8), want.q.view(torch.uint8))
