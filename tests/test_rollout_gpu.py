"""The operators as a reinforcement-learning step uses them: a decoding step's end on the rollout's side, then the training step on
the drawn tokens, from the final norm through the fused LM head and back."""
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _model(T, H, V, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    x, r = normal(T, H).to(torch.bfloat16), (2 * normal(T, H)).to(torch.bfloat16)
    gamma = (1 + 0.2 * normal(H)).to(torch.bfloat16)
    w = (normal(V, H) * 0.1).to(torch.bfloat16)
    return x, r, gamma, w, torch.rand(T, generator=g, device="cuda"), normal(T)


@pytest.mark.parametrize("T", [1, 16, 130])
def test_rollout_head_is_its_parts(T):
    x, r, gamma, w, u, _ = _model(T, 384, 3001)
    q = b.dvp_quantize_fp8(w)
    got = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, residual=r, eps=EPS, rho=1e-3, top_p=0.95)
    h = x.double() + r.double()
    y = h * (h.square().mean(1, keepdim=True) + EPS).rsqrt() * gamma.double()
    # logits of the exact product: three block scales of a row, off by half an e4m3 step (2^-4) of every factor and bf16's 2^-8
    size = y.abs() @ w.double().abs().t()
    assert ((got.logits.double() - y @ w.double().t()).abs() <= size * (2 * 2.0 ** -4 + 2.0 ** -7)).all()
    assert int(got.status) == 0
    again = b.dvp_sample(got.logits, u, rho=1e-3, top_p=0.95)
    assert torch.equal(got.ids, again.ids) and torch.equal(got.logp_mp, again.logp_mp) and torch.equal(got.count, again.count)
    assert torch.equal(got.residual, h.to(torch.bfloat16))


def test_a_reinforcement_learning_step():
    T, H, V, rho = 96, 256, 2048, 1e-2
    x, r, gamma, w, u, advantage = _model(T, H, V)
    q = b.dvp_quantize_fp8(w)
    roll = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, residual=r, eps=EPS, rho=rho)
    # the inference side's values are those that the library's forward pass finds for the same logits and tokens
    fwd = b.dvp_forward(roll.logits, roll.ids, rho, infer_logits=roll.logits)
    assert ((fwd.flags & b.DVP_FLAG_IN_INFER) != 0).all() and torch.equal(fwd.infer.count, roll.count)
    assert (fwd.infer.logp_mp - roll.logp_mp).abs().max() < 1e-4
    # training: the norm in bfloat16, the fused LM head against the rollout's logits, and back through the norm
    norm = b.dvp_rms_norm(x, gamma, residual=r, eps=EPS)
    head = b.dvp_fused_lmhead_forward_backward(norm.y, w, roll.ids, rho, advantage, infer_logits=roll.logits)
    back = b.dvp_rms_norm_backward(head.d_hidden, norm.residual, gamma, norm.rstd)
    torch.cuda.synchronize()
    assert head.workspace[:4].view(torch.int32).item() == 0
    assert (head.infer.logp_mp - roll.logp_mp).abs().max() < 1e-4
    # the norm's step of the chain by autograd, in float64, from the head's own gradient
    h = norm.residual.double().requires_grad_()
    gd = gamma.double().requires_grad_()
    y = h * (h.square().mean(1, keepdim=True) + EPS).rsqrt() * gd
    y.backward(head.d_hidden.double())
    # The norm takes rstd of h before h is rounded to bfloat16.  Each h_j is off by 2^-8 of itself at most, so mean h^2 by twice
    # that and rstd = s by 2^-8: s g by as much, s^3 h mean(g h) by three times; float32 sums are far below.  One rounding
    # of the result.
    s = (h.detach().square().mean(1, keepdim=True) + EPS).rsqrt()
    g = head.d_hidden.double() * gd.detach()
    size = s * g.abs() + 3 * s ** 3 * h.detach().abs() * (g * h.detach()).abs().mean(1, keepdim=True)
    assert ((back.d_x.double() - h.grad).abs() <= (h.grad.abs() + size) * 2.0 ** -8 * 1.02).all()
    assert ((back.d_weight.double() - gd.grad).abs() <= 2.0 ** -8 * 1.02 * (head.d_hidden.double() * h.detach() * s).abs().sum(0)).all()
    # with that rstd itself the formula holds to float32's sums
    s = norm.rstd.double()[:, None]
    want = s * (g - h.detach() * s * s * (g * h.detach()).mean(1, keepdim=True))
    assert ((back.d_x.double() - want).abs() <= want.abs() * 2.0 ** -8 * 1.01 + 1e-5 * size).all()


def test_a_decoding_step_in_a_graph():
    x, r, gamma, w, u, _ = _model(8, 512, 5000)
    q = b.dvp_quantize_fp8(w)
    want = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, residual=r, top_k=20, temperature=0.8)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, residual=r, top_k=20, temperature=0.8)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got.ids, want.ids) and torch.equal(got.logits, want.logits)
    u.copy_(torch.rand(8, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    want = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, residual=r, top_k=20, temperature=0.8)
    assert torch.equal(got.ids, want.ids)


def test_a_padded_batch():
    """Rows without content, as a serving batch is padded with: zeros, and rows masked as a whole."""
    x, r, gamma, w, u, _ = _model(12, 256, 1000)
    x[8:], r[8:] = 0, 0
    q = b.dvp_quantize_fp8(w)
    got = b.dvp_rollout_head(x, gamma, q.q, q.scale, u, residual=r, top_p=0.9)
    alone = b.dvp_rollout_head(x[:8], gamma, q.q, q.scale, u[:8], residual=r[:8], top_p=0.9)
    assert torch.equal(got.ids[:8], alone.ids) and torch.equal(got.logits[:8], alone.logits)
    assert (got.logits[8:] == 0).all() and (got.count[8:] == 900).all()
    got.logits[9] = -float("inf")
    assert b.dvp_sample(got.logits, u, top_p=0.9).ids[9] == -1
