"""The 8-bit product with a scale for each block of 128, and the quantiser, against their definitions in float64."""
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu
F32, BF16, F16, FP8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}


def _bytes(rows, cols, seed, ld=None, whole=False, offset=0):
    """e4m3 values in rows of `ld` bytes; what lies behind a row is 448."""
    ld = -(-cols // 16) * 16 if ld is None else ld
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + rows * ld,), 448.0, device="cuda").to(FP8)
    v = torch.randint(-4, 5, (rows, cols), generator=g, device="cuda").float() if whole else \
        torch.randn(rows, cols, generator=g, device="cuda") * 30
    x = buf[offset:].view(rows, ld)[:, :cols]
    x.copy_(v.to(FP8))
    return x


def _scales(rows, cols, seed, pad=0, power=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(rows, cols + pad, generator=g, device="cuda")
    return (torch.exp2(v.round()) if power else torch.exp(v) * 0.01)[:, :cols]


def _definition(a, sa, w, sb):
    K, N = a.shape[1], w.shape[0]
    ad = a.double() * sa.double().repeat_interleave(128, 1)[:, :K]
    wd = w.double() * sb.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    return ad @ wd.t(), ad.abs() @ wd.abs().t()


def _check(a, sa, w, sb, dtype, out, status):
    want, size = _definition(a, sa, w, sb)
    assert int(status) == 0
    # products of e4m3 are exact; sums of 128 in the tensor core cut off at 2^-23 of their size at each addition, the K / 128
    # additions outside round to half of that; one rounding to the result's type, whose least step is 2^-24 for float16
    bound = size * (128 + a.shape[1] / 128) * 2.0 ** -23 + want.abs() * UNIT[dtype] * 1.01 + (2.0 ** -25 if dtype == F16 else 0)
    err = (out.double() - want).abs()
    assert torch.isfinite(out.float()).all()
    assert (err <= bound).all(), float((err / bound.clamp(min=1e-300)).max())


@pytest.mark.parametrize("M", [1, 15, 16, 17, 32, 33, 64, 65, 128, 129, 256, 300])
@pytest.mark.parametrize("N,K", [(1, 1), (7, 100), (128, 128), (129, 416), (1000, 129), (3000, 1024)])
def test_sizes(M, N, K):
    a, w = _bytes(M, K, 1), _bytes(N, K, 2)
    sa, sb = _scales(M, -(-K // 128), 3), _scales(-(-N // 128), -(-K // 128), 4)
    for dtype in (F32, BF16):
        out, status = b.dvp_gemm_fp8(a, sa, w, sb, out_dtype=dtype)
        _check(a, sa, w, sb, dtype, out, status)


@pytest.mark.parametrize("hint", [1, 2])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,N,K", [(1, 20000, 256), (33, 19000, 700), (64, 513, 2048)])
def test_both_kernels_and_every_type(hint, dtype, M, N, K):
    a, w = _bytes(M, K, 5), _bytes(N, K, 6)
    sa, sb = _scales(M, -(-K // 128), 7), _scales(-(-N // 128), -(-K // 128), 8)
    out, status = b.dvp_gemm_fp8(a, sa, w, sb, out_dtype=dtype, launch_hint=hint)
    _check(a, sa, w, sb, dtype, out, status)


@pytest.mark.parametrize("M,hint", [(9, 0), (50, 0), (50, 1), (100, 0), (700, 0)])
def test_whole_numbers_are_exact(M, hint):
    """Products, sums and scales that float32 holds exactly: every place of every tile, to the last bit."""
    N, K = 40000, 640
    a, w = _bytes(M, K, 1, whole=True), _bytes(N, K, 2, whole=True)
    sa, sb = _scales(M, 5, 3, power=True).clamp(0.5, 2), _scales(-(-N // 128), 5, 4, power=True).clamp(0.5, 2)
    out, status = b.dvp_gemm_fp8(a, sa, w, sb, out_dtype=F32, launch_hint=hint)
    assert int(status) == 0
    assert torch.equal(out.double(), _definition(a, sa, w, sb)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [5, 130])
def test_strides_and_what_lies_behind_the_result(dtype, M):
    N, K = 300, 200
    a, w = _bytes(M, K, 1, ld=240, offset=16), _bytes(N, K, 2, ld=256, offset=32)
    sa, sb = _scales(M, 2, 3, pad=3), _scales(3, 2, 4, pad=1)
    for ld, first in ((301, 1), (304, 0), (320, 0)):
        buf = torch.full((first + (M + 2) * ld,), 9.0, dtype=dtype, device="cuda")
        out = buf[first:].view(M + 2, ld)
        got, status = b.dvp_gemm_fp8(a, sa, w, sb, out=out[:M, :N])
        _check(a, sa, w, sb, dtype, got, status)
        assert (out[M:] == 9).all() and (out[:, N:] == 9).all() and (buf[:first] == 9).all()


def test_rows_that_are_not_finite_stay_alone():
    a, w = _bytes(40, 256, 1), _bytes(600, 256, 2)
    sa, sb = _scales(40, 2, 3), _scales(5, 2, 4)
    clean, _ = b.dvp_gemm_fp8(a, sa, w, sb)
    a.view(torch.uint8)[3, 5] = 0x7f   # NaN
    sa[7, 1] = float("inf")
    out, status = b.dvp_gemm_fp8(a, sa, w, sb)
    assert int(status) == 0 and torch.isnan(out[3]).all() and not torch.isfinite(out[7]).any()
    keep = [i for i in range(40) if i not in (3, 7)]
    assert torch.equal(out[keep], clean[keep])


@pytest.mark.parametrize("M", [16, 200])
def test_captured_and_repeated_calls(M):
    a, w = _bytes(M, 384, 1), _bytes(5000, 384, 2)
    sa, sb = _scales(M, 3, 3), _scales(40, 3, 4)
    first, _ = b.dvp_gemm_fp8(a, sa, w, sb)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out, status = b.dvp_gemm_fp8(a, sa, w, sb)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0 and torch.equal(out, first)


def test_empty_products():
    a, w = _bytes(4, 128, 1), _bytes(6, 128, 2)
    sa, sb = _scales(4, 1, 3), _scales(1, 1, 4)
    out, status = b.dvp_gemm_fp8(a[:0], sa[:0], w, sb)
    assert out.shape == (0, 6) and int(status) == 0


def test_refused_layouts():
    a, w = _bytes(4, 128, 1), _bytes(6, 128, 2)
    sa, sb = _scales(4, 1, 3), _scales(1, 1, 4)
    odd = torch.zeros(6 * 130, device="cuda").to(FP8).view(6, 130)[:, :128]
    with pytest.raises(b.DvpError) as e:
        b.dvp_gemm_fp8(a, sa, odd, sb)
    assert e.value.status == b.DVP_ERR_UNSUPPORTED
    for bad in (lambda: b.dvp_gemm_fp8(a, sa[:3], w, sb), lambda: b.dvp_gemm_fp8(a, sa, w, sb.repeat(2, 1)),
                lambda: b.dvp_gemm_fp8(a, sa, w[:, :64], sb), lambda: b.dvp_gemm_fp8(a, sa, w, sb.cpu()),
                lambda: b.dvp_gemm_fp8(a, sa, w, sb, out=torch.empty(4, 7, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: b.dvp_gemm_fp8(a.float(), sa, w, sb), lambda: b.dvp_gemm_fp8(a, sa.half(), w, sb),
                lambda: b.dvp_gemm_fp8(a, sa, w, sb, out_dtype=torch.float64)):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (128, 128, 0), (129, 300, 0), (300, 1001, 0), (200, 256, 4), (200, 256, 3)])
def test_quantiser(dtype, block_rows, rows, cols, pad):
    g = torch.Generator(device="cuda").manual_seed(7)
    x = (torch.randn(rows, cols + pad, generator=g, device="cuda") * 3).to(dtype)[:, :cols]
    if rows > 2:
        x[2] = 0
    res = b.dvp_quantize_fp8(x, block_rows=block_rows)
    n, m = -(-cols // 128), -(-rows // block_rows)
    xd = torch.nn.functional.pad(x.double(), (0, n * 128 - cols, 0, m * block_rows - rows))
    amax = xd.view(m, block_rows, n, 128).abs().amax((1, 3)).clamp(min=2.0 ** -96)
    assert res.scale.shape == (m, n) and res.q.stride(0) % 16 == 0
    assert ((res.scale.double() - amax / 448).abs() <= amax / 448 * 2.0 ** -24 * 1.01).all()
    c = res.scale.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    want = x.double() / c
    # half a step of e4m3, 2^-10 below its least normal value, and the float32 roundings of scale and quotient
    assert ((res.q.double() - want).abs() <= want.abs() * (2.0 ** -4 + 2.0 ** -21) + 2.0 ** -10 * 1.001).all()


def test_head_of_a_quantised_weight_stands_for_the_weight():
    """hidden x W^T with both in 8 bits: off by the two roundings, at most 2^-4 each of every product."""
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(50, 512, generator=g, device="cuda").to(BF16)
    w = (torch.randn(1000, 512, generator=g, device="cuda") * 0.02).to(BF16)
    qh, qw = b.dvp_quantize_fp8(h, block_rows=1), b.dvp_quantize_fp8(w)
    out, status = b.dvp_gemm_fp8(qh.q, qh.scale, qw.q, qw.scale, out_dtype=F32)
    assert int(status) == 0
    want, size = h.double() @ w.double().t(), h.double().abs() @ w.double().abs().t()
    # small values round to half of 2^-9 in units of the scale: under 2^-18 of the block's largest
    bound = size * (2 * 2.0 ** -4 + 2.0 ** -8) + 512 * 2.0 ** -17 * float(h.abs().max()) * float(w.abs().max())
    assert ((out.double() - want).abs() <= bound).all()
