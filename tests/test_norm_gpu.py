"""Root-mean-square norm and its backward pass against the definition in float64."""
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu
F32, BF16, F16, FP8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
EPS = 1e-6
# A sum of squares is at most 20 additions a thread (16,384 columns: 32 a thread; the layout-free kernel 4 H / 1024) and some
# 40 more between threads, each off by half a step of 2^-24 relative to a sum of positive terms: (80 + 40) / 2 * 2^-24 < 4e-6 of
# the sum, half of that of its root; the products, the division and the root another 4 half steps.
SUM = 4e-6


def _rows(T, H, dtype, seed, pad=0, scale=1.0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((T * (H + pad) + offset,), 7.0, dtype=dtype, device="cuda")
    x = buf[offset:].view(T, H + pad)[:, :H]
    x.copy_((torch.randn(T, H, generator=g, device="cuda") * scale).to(dtype))
    return x


def _weight(H, dtype, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(H, generator=g, device="cuda")).to(dtype)


def _definition(x, r, w):
    h = x.double() + (r.double() if r is not None else 0)
    s = (h.square().mean(1) + EPS).rsqrt()
    return h, s, h * s[:, None] * w.double()


def _close(got, want, rel, floor=0.0):
    err = (got.double() - want).abs()
    bound = want.abs() * rel + floor
    assert torch.isfinite(got.double()).all()
    assert (err <= bound).all(), float((err / bound.clamp(min=1e-300)).max())


def _check(x, r, w, out, res):
    T, H = x.shape
    h, s, y = _definition(x, r, w)
    _close(res.rstd, s, SUM)
    if r is not None:
        # one rounding; of a type with subnormals the step there
        _close(res.residual, h, UNIT[x.dtype] * 1.001, 2.0 ** -25 if x.dtype == F16 else 0)
    if out != FP8:
        _close(res.y, y, SUM + UNIT[out] * 1.001, 2.0 ** -25 if out == F16 else 0)
        return
    n = -(-H // 128)
    amax = torch.stack([c.abs().amax(1) for c in y.split(128, 1)], 1).clamp(min=2.0 ** -96)
    assert res.scale.shape == (T, n)
    _close(res.scale, amax / 448, 2 * SUM)
    # half a step: 2^-4 of the value, 2^-10 below the least normal one
    q, c = res.y.double(), res.scale.double().repeat_interleave(128, 1)[:, :H]
    assert torch.isfinite(q).all()
    want = y / c
    assert ((q - want).abs() <= want.abs() * (2.0 ** -4 + 4 * SUM) + 2.0 ** -10 * 1.001).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,H,pad,offset", [
    (1, 1, 0, 0), (1, 8, 0, 0), (3, 64, 0, 0), (5, 128, 0, 0), (2, 136, 0, 0), (9, 256, 8, 0), (8, 4096, 0, 0), (33, 1000, 0, 0),
    (4, 1001, 0, 0), (7, 130, 3, 1), (300, 520, 0, 8), (3, 16384, 0, 0), (2, 16392, 0, 0), (2, 20011, 0, 0), (700, 384, 0, 0)])
def test_forward(dtype, fp8, T, H, pad, offset):
    x, r, w = _rows(T, H, dtype, 1, pad, offset=offset), _rows(T, H, dtype, 2, pad, 3.0, offset), _weight(H, dtype)
    out = FP8 if fp8 else dtype
    _check(x, r, w, out, b.dvp_rms_norm(x, w, residual=r, eps=EPS, out_dtype=out))
    _check(x, None, w, out, b.dvp_rms_norm(x, w, eps=EPS, out_dtype=out))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("H", [256, 77])
def test_output_and_weight_types(dtype, out, H):
    x, w = _rows(6, H, dtype, 5), _weight(H, F32)
    _check(x, None, w, out, b.dvp_rms_norm(x, w, eps=EPS, out_dtype=out))


@pytest.mark.parametrize("H", [512, 515])
@pytest.mark.parametrize("over", ["x", "residual"])
def test_residual_takes_an_inputs_place(H, over):
    x, r, w = _rows(40, H, BF16, 1), _rows(40, H, BF16, 2), _weight(H, BF16)
    x0, r0 = x.clone(), r.clone()
    res = b.dvp_rms_norm(x, w, residual=r, eps=EPS, out_dtype=FP8, residual_out=x if over == "x" else r)
    assert res.residual.data_ptr() == (x if over == "x" else r).data_ptr()
    _check(x0, r0, w, FP8, res)


@pytest.mark.parametrize("H", [512, 515])
def test_rows_without_content_and_rows_that_are_not_finite(H):
    x, w = _rows(6, H, BF16, 1), _weight(H, BF16)
    x[1] = 0
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    for out in (BF16, FP8):
        res = b.dvp_rms_norm(x, w, eps=EPS, out_dtype=out)
        good = [0, 1, 2, 5]
        pick = b.SimpleNamespace(y=res.y[good], rstd=res.rstd[good], residual=None,
                                 scale=res.scale[good] if out == FP8 else None)
        _check(x[good], None, w, out, pick)
        assert (res.y[1].float() == 0).all()
        assert torch.isnan(res.y[3].float()).all() and torch.isnan(res.y[4, 7].float())


def test_rows_and_columns_behind_the_last_stay():
    big = torch.full((12, 520), 5.0, dtype=BF16, device="cuda")
    x, r, w = _rows(10, 512, BF16, 1), _rows(10, 512, BF16, 2), _weight(512, BF16)
    res = b.dvp_rms_norm(x, w, residual=r, eps=EPS, residual_out=big[:10, :512])
    _check(x, r, w, BF16, res)
    assert (big[10:] == 5).all() and (big[:, 512:] == 5).all()


@pytest.mark.parametrize("dtype,dy_dtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("T,H,pad,offset", [
    (1, 1, 0, 0), (1, 64, 0, 0), (5, 128, 0, 0), (700, 96, 0, 0), (1, 4096, 0, 0), (1300, 520, 8, 0), (5, 1001, 0, 0),
    (641, 33, 0, 1), (3, 8192, 0, 0), (3, 16384, 0, 0), (2, 16392, 0, 0), (2, 20011, 0, 0)])
def test_backward(dtype, dy_dtype, T, H, pad, offset):
    h, dy = _rows(T, H, dtype, 1, pad, 3.0, offset), _rows(T, H, dy_dtype, 2, pad, 1.0, offset)
    dr, w = _rows(T, H, dtype, 4, pad, 1.0, offset), _weight(H, dtype)
    _, s, _ = _definition(h, None, w)
    rstd = s.float()
    for d_residual in (dr, None):
        res = b.dvp_rms_norm_backward(dy, h, w, rstd, d_residual=d_residual)
        _check_backward(h, dy, w, rstd, d_residual, res)


def _check_backward(h, dy, w, rstd, dr, res, before=0.0):
    T, H = h.shape
    hd, dyd, s = h.double(), dy.double(), rstd.double()[:, None]
    g = dyd * w.double()
    gh = g * hd
    want = s * (g - hd * s * s * gh.mean(1, keepdim=True)) + (dr.double() if dr is not None else 0)
    # the sum g h has terms of both signs: its error is of the size of the sum of their magnitudes
    size = s * (g.abs() + hd.abs() * s * s * gh.abs().mean(1, keepdim=True)) + (dr.double().abs() if dr is not None else 0)
    err = (res.d_x.double() - want).abs()
    unit = UNIT[h.dtype]
    assert (err <= size * 2 * SUM + want.abs() * unit * 1.01 + (2.0 ** -25 if h.dtype == F16 else 0)).all()
    # dw: at most T / 592 + 1 rows one after the other, then 74 and 8 partial sums
    terms = dyd * hd * s
    bound = ((T / 592 + 100) * 2.0 ** -24) * (terms.abs().sum(0) + abs(before)) + 1e-30
    assert ((res.d_weight.double() - before - terms.sum(0)).abs() <= bound).all()


def test_backward_adds_to_the_weights_gradient():
    h, dy, w = _rows(200, 256, BF16, 1), _rows(200, 256, F32, 2), _weight(256, BF16)
    rstd = _definition(h, None, w)[1].float()
    d_w = torch.full((256,), 2.5, device="cuda")
    res = b.dvp_rms_norm_backward(dy, h, w, rstd, d_weight=d_w, accumulate_dw=True)
    assert res.d_weight.data_ptr() == d_w.data_ptr()
    _check_backward(h, dy, w, rstd, None, res, before=2.5)


def test_backward_against_differences():
    """The gradient of sum(dy * y) by central differences of the definition in float64."""
    T, H = 3, 40
    x, dy, w = _rows(T, H, F32, 1), _rows(T, H, F32, 2), _weight(H, F32)
    fwd = b.dvp_rms_norm(x, w, eps=EPS)
    res = b.dvp_rms_norm_backward(dy, x, w, fwd.rstd)

    def loss(xd, wd):
        return float((dy.double() * _definition(xd, None, wd)[2]).sum())
    step = 1e-5   # error of a central difference: step^2 times a third derivative of order ten, and 1e-16 / step
    for t, c in [(0, 0), (1, 17), (2, 39)]:
        d = torch.zeros(T, H, dtype=torch.float64, device="cuda")
        d[t, c] = step
        num = (loss(x.double() + d, w.double()) - loss(x.double() - d, w.double())) / (2 * step)
        assert abs(num - float(res.d_x[t, c])) < 1e-5 * max(1.0, abs(num)) + 1e-6
    for c in (0, 21):
        d = torch.zeros(H, dtype=torch.float64, device="cuda")
        d[c] = step
        num = (loss(x.double(), w.double() + d) - loss(x.double(), w.double() - d)) / (2 * step)
        assert abs(num - float(res.d_weight[c])) < 1e-5 * max(1.0, abs(num)) + 1e-6


@pytest.mark.parametrize("H", [384, 387])
def test_reruns_are_bit_identical_and_captured_calls_repeat(H):
    T = 2000
    h, dy, w = _rows(T, H, BF16, 1), _rows(T, H, F32, 2), _weight(H, BF16)
    fwd = b.dvp_rms_norm(h, w, eps=EPS, out_dtype=FP8)
    one = b.dvp_rms_norm_backward(dy, h, w, fwd.rstd)
    two = b.dvp_rms_norm_backward(dy, h, w, fwd.rstd)
    assert torch.equal(one.d_weight, two.d_weight) and torch.equal(one.d_x, two.d_x)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            f = b.dvp_rms_norm(h, w, eps=EPS, out_dtype=FP8)
            g = b.dvp_rms_norm_backward(dy, h, w, f.rstd)
    h.mul_(-1.0)
    torch.cuda.synchronize()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    want = b.dvp_rms_norm(h, w, eps=EPS, out_dtype=FP8)
    assert torch.equal(f.y.view(torch.uint8), want.y.view(torch.uint8)) and torch.equal(f.scale, want.scale)
    again = b.dvp_rms_norm_backward(dy, h, w, want.rstd)
    assert torch.equal(g.d_x, again.d_x) and torch.equal(g.d_weight, again.d_weight)


def test_empty_batches():
    w = _weight(16, BF16)
    x = torch.empty(0, 16, dtype=BF16, device="cuda")
    res = b.dvp_rms_norm(x, w, out_dtype=FP8)
    assert res.y.shape == (0, 16) and res.scale.shape == (0, 1)
    back = b.dvp_rms_norm_backward(x, x, w, res.rstd)
    assert (back.d_weight == 0).all() and back.d_x.shape == (0, 16)


def test_a_call_on_a_stream_of_its_own_follows_that_stream():
    x, w = _rows(64, 1024, BF16, 1), _weight(1024, BF16)
    want = b.dvp_rms_norm(x, w, eps=EPS).y.clone()
    late = torch.zeros_like(x)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
    got = b.dvp_rms_norm(late, w, eps=EPS, stream=stream)
    stream.synchronize()
    assert torch.equal(got.y, want)
