"""Calls on a stream of the caller's own: what a call allocates for itself must not be handed out again while that stream works."""
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu


def _held():
    """Bytes that nobody holds any more and that the allocator keeps back for a stream."""
    s = torch.cuda.memory_stats()
    return s["active_bytes.all.current"] - s["allocated_bytes.all.current"]


def test_backward_workspace_outlives_the_call():
    T, H = 2048, 1024  # large enough for storages of their own
    h = torch.randn(T, H, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    w = torch.ones(H, device="cuda")
    rstd = h.square().mean(1).rsqrt()
    want = b.dvp_rms_norm_backward(h, h, w, rstd)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = _held()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = b.dvp_rms_norm_backward(h, h, w, rstd, stream=side)
    held = _held() - before
    torch.cuda.synchronize()
    assert held >= 592 * H * 4
    assert torch.equal(got.d_x, want.d_x) and torch.equal(got.d_weight, want.d_weight)


@pytest.mark.parametrize("T", [2, 600])
def test_rollout_head_keeps_its_hidden_states(T):
    H, V = 2048, 1000
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(T, H, device="cuda", generator=g).bfloat16()
    w = torch.randn(V, H, device="cuda", generator=g).bfloat16()
    u, gamma = torch.rand(T, device="cuda", generator=g), torch.ones(H, device="cuda")
    q = b.dvp_quantize_fp8(w)
    want = b.dvp_rollout_head(x, gamma, q.q, q.scale, u)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = _held()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, stream=side)
    # a small call's rstd lies in the same storage as the hidden states and holds it
    got.rstd = None
    held = _held() - before
    torch.cuda.synchronize()
    assert held >= T * H
    assert torch.equal(got.ids, want.ids) and torch.equal(got.logits, want.logits)


def _product(M=8, K=256, N=1000):
    g = torch.Generator("cuda").manual_seed(4)
    a, w = (b.dvp_quantize_fp8(torch.randn(r, K, device="cuda", generator=g), block_rows=n) for r, n in ((M, 1), (N, 128)))
    return a.q, a.scale, w.q, w.scale


@pytest.mark.parametrize("M", [8, 100])
def test_product_status_is_nobody_elses_while_the_stream_works(M):
    """The status word is let go of at once, and what takes its place on the current stream must stay as it is."""
    args = _product(M)
    want, _ = b.dvp_gemm_fp8(*args)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = _held()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got, status = b.dvp_gemm_fp8(*args, stream=side)
    del status
    held = _held() - before
    words = [torch.full((1,), 77, dtype=torch.int32, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert [int(v) for v in words] == [77] * 8
    assert held > 0
    assert torch.equal(got, want)


@pytest.mark.parametrize("M,N", [(0, 1000), (8, 0)])
def test_an_empty_product_says_so_on_the_named_stream(M, N):
    a, sa, w, sw = _product()
    side = torch.cuda.Stream()
    old = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    del old     # what the status word finds in its place
    torch.cuda._sleep(50_000_000)
    _, status = b.dvp_gemm_fp8(a[:M], sa[:M], w[:N], sw[:-(-N // 128)], stream=side)
    with torch.cuda.stream(side):
        said = status.to("cpu", non_blocking=False)
    torch.cuda.synchronize()
    assert int(said) == 0


def _behind_a_busy_stream(call):
    """Lets go of a call's results while its stream is held back, but for what `call` returns: the bytes that stay put for it, and new
    tensors of 77 that must stay as they are."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = _held()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    kept = call(side)
    held = _held() - before
    new = [torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (1 << 19, 1 << 19, 1 << 17, 1 << 17, 4096, 4096, 128, 128)]
    torch.cuda.synchronize()
    assert all((t == 77).all() for t in new)
    return kept, held


def test_norm_results_that_are_let_go_of():
    T, H = 4096, 512     # large enough for storages of their own
    g = torch.Generator("cuda").manual_seed(5)
    x, w = torch.randn(T, H, device="cuda", generator=g).bfloat16(), torch.ones(H, device="cuda")
    want = b.dvp_rms_norm(x, w, residual=x, out_dtype=torch.float8_e4m3fn)
    kept, held = _behind_a_busy_stream(lambda s: b.dvp_rms_norm(x, w, residual=x, out_dtype=torch.float8_e4m3fn, stream=s).y)
    assert held >= T * 4 + T * 4 * 4 + T * H * 2     # rstd, scale, residual
    assert torch.equal(kept.view(torch.uint8), want.y.view(torch.uint8))


@pytest.mark.parametrize("T", [2, 3000])
def test_rollout_head_whose_product_is_refused(T):
    H = 1024
    x, gamma = torch.randn(T, H, device="cuda").bfloat16(), torch.ones(H, device="cuda")
    q = b.dvp_quantize_fp8(torch.randn(500, H // 2, device="cuda"))     # of another width

    def call(side):
        try:
            b.dvp_rollout_head(x, gamma, q.q, q.scale, torch.rand(T, device="cuda"), stream=side)
        except ValueError:
            return True
    refused, held = _behind_a_busy_stream(call)
    assert refused and held >= T * H


def test_other_results_that_are_let_go_of():
    T, H, V = 4096, 1024, 2048
    g = torch.Generator("cuda").manual_seed(6)
    h, w = torch.randn(T, H, device="cuda", generator=g), torch.ones(H, device="cuda")
    rstd, u = h.square().mean(1).rsqrt(), torch.rand(T, device="cuda", generator=g)
    want = b.dvp_rms_norm_backward(h, h, w, rstd)
    kept, held = _behind_a_busy_stream(lambda s: b.dvp_rms_norm_backward(h, h, w, rstd, stream=s).d_weight)
    assert held >= T * H * 4 and torch.equal(kept, want.d_weight)
    kept, held = _behind_a_busy_stream(lambda s: b.dvp_quantize_fp8(h, stream=s).scale)
    assert held >= T * H and torch.equal(kept, b.dvp_quantize_fp8(h).scale)
    _, held = _behind_a_busy_stream(lambda s: (b.dvp_sample(h, u, stream=s), None)[1])
    assert held >= T * 20
    q = b.dvp_quantize_fp8(h, block_rows=1)
    k = b.dvp_quantize_fp8(torch.randn(V, H, device="cuda", generator=g))
    _, held = _behind_a_busy_stream(lambda s: (b.dvp_gemm_fp8(q.q, q.scale, k.q, k.scale, stream=s), None)[1])
    assert held >= T * V * 2
