"""Sampling against its definition in float64, row by row: the token, its two log-probabilities and the number of tokens kept."""
import math

import numpy as np
import pytest
import torch

from paper_2512_23087_b200 import binding as b

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = {"f32": F32, "bf16": BF16, "f16": F16}


def _definition(z, u, temperature, top_k, top_p, rho):
    """One row of float64 logits: (a, ln pi(a), ln pi of the kept, |K2|) as the header states it."""
    if not (np.isfinite(z) | (z == -np.inf)).all() or not (z > -np.inf).any():
        return -1, math.nan, math.nan, 0
    greedy = temperature == 0
    t = 1.0 if greedy else temperature
    w = np.exp((z - z.max()) / t)
    order = np.lexsort((np.arange(z.size), -z))   # falling, equal ones by index
    n = int(((z > -np.inf) & (z >= z.max() + (t * math.log(rho) if rho > 0 else -np.inf))).sum())
    if greedy:
        n = 1
    elif top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        mass = w[order[:n]]
        before = np.concatenate([[0.0], np.cumsum(mass)[:-1]])
        n = max(1, int((before < top_p * mass.sum()).sum()))
    kept = np.sort(order[:n])
    run = np.cumsum(w[kept])
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    i = int(np.searchsorted(run, u * run[-1], side="right"))
    if i == n:
        i = int(np.flatnonzero(w[kept] > 0)[-1])
    a = int(kept[i])
    # the maximum's own term apart, so that logarithms near zero keep their digits
    top = int(z.argmax())
    rest = np.delete(w, top).sum()
    rest_kept = w[kept].sum() - 1.0 if n > 1 else 0.0
    if n > 1:
        rest_kept = np.delete(w[kept], int(np.flatnonzero(kept == top)[0])).sum()
    x = (z[a] - z[top]) / t
    return a, x - math.log1p(rest), x - math.log1p(rest_kept), n


def _per_row(v, T):
    return v.tolist() if isinstance(v, torch.Tensor) else [v] * T


def _check(z, u, hints=(0,), rows=None, **settings):
    T = z.shape[0]
    zd, ud = z.double().cpu().numpy(), u.double().cpu().numpy()
    s = {n: _per_row(settings.get(n, d), T) for n, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("rho", 0.0))}
    want = [_definition(zd[t], float(ud[t]), s["temperature"][t], s["top_k"][t], s["top_p"][t], s["rho"][t]) for t in range(T)]
    first = None
    for hint in hints:
        got = b.dvp_sample(z, u, launch_hint=hint, **settings)
        assert got.ids.tolist() == [w[0] for w in want], hint
        assert got.count.tolist() == [w[3] for w in want], hint
        for name, k in (("logp", 1), ("logp_mp", 2)):
            v, e = getattr(got, name).double().cpu().numpy(), np.array([w[k] for w in want])
            assert np.array_equal(np.isnan(v), np.isnan(e))
            # the sum over the row is formed in float32: exponents of up to 2^4 carry 2^-24 of themselves three times, products
            # and additions beside it some ten half steps: 4e-6 of the sum beside the maximum; one rounding of the result
            fine = ~np.isnan(e)
            # a term below 2^-126 is zero in float32, and a row has as many as it has logits; the result rounds to 2^-150 at the least
            lost = z.shape[1] * 2.0 ** -126 + 2.0 ** -150
            bound = 4e-6 * np.minimum(1.0, np.abs(e[fine])) + 2.0 ** -23 * np.abs(e[fine]) + lost
            assert (np.abs(v - e)[fine] <= bound).all(), (hint, name)
        if first is not None:
            assert torch.equal(got.ids, first.ids) and torch.equal(got.count, first.count)
        first = got
    return first


def _logits(T, V, dtype, seed, scale=3.0, boost=15.0, pad=0, offset=0):
    """Rows between open and decided; what lies behind a row is 30,000."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + T * (V + pad),), 3e4, dtype=dtype, device="cuda")
    z = buf[offset:].view(T, V + pad)[:, :V]
    v = scale * torch.randn(T, V, generator=g, device="cuda")
    at = torch.randint(0, V, (T, min(V, 8)), generator=g, device="cuda")
    v.scatter_add_(1, at, boost * torch.rand(T, 1, generator=g, device="cuda").expand(-1, min(V, 8)).contiguous())
    z.copy_(v.to(dtype))
    return z


def _uniform(T, seed=9):
    return torch.rand(T, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(rho=1e-4), dict(rho=1.0), dict(top_k=1), dict(top_k=7),
            dict(top_k=50, temperature=1.3), dict(top_p=0.9), dict(top_p=0.5, temperature=2.0), dict(top_p=0.0), dict(top_p=1e-9),
            dict(top_p=0.999999), dict(top_k=100, top_p=0.95, rho=0.01), dict(top_k=20000, top_p=0.99), dict(rho=0.3, top_p=0.8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("settings", SETTINGS, ids=str)
@pytest.mark.parametrize("V", [1, 2, 33, 1000, 50021])
def test_settings(dtype, settings, V):
    z = _logits(6, V, DTYPES[dtype], 1)
    _check(z, _uniform(6), hints=(0, 1, 2, 4, 8) if V > 33 else (0, 1, 8), **settings)


@pytest.mark.parametrize("dtype,V", [("bf16", 151936), ("f32", 262144), ("f32", 600011)])
@pytest.mark.parametrize("settings", [dict(), dict(rho=2.26e-6), dict(top_k=50), dict(top_p=0.95), dict(top_k=40000, top_p=0.999)], ids=str)
def test_long_vocabularies(dtype, V, settings):
    _check(_logits(3, V, DTYPES[dtype], 2), _uniform(3), hints=(0, 1, 2), **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (13, 3), (16, 1), (0, 5)])
def test_rows_at_any_alignment(dtype, pad, offset):
    z = _logits(9, 3001, DTYPES[dtype], 3, pad=pad, offset=offset)
    for settings in (dict(), dict(top_k=30), dict(top_p=0.9), dict(rho=0.01)):
        _check(z, _uniform(9), hints=(0, 1, 4), **settings)


def test_rows_with_settings_of_their_own():
    T, V = 300, 5000
    g = torch.Generator(device="cuda").manual_seed(4)

    def pick(values, dtype):
        return torch.tensor(values, dtype=dtype, device="cuda")[torch.randint(0, len(values), (T,), generator=g, device="cuda")]
    _check(_logits(T, V, BF16, 5), _uniform(T), hints=(0, 1, 2), temperature=pick([0.0, 0.5, 1.0, 1.5], F32),
           top_k=pick([-3, 0, 1, 2, 40, 4999, 5000, 100000], torch.int32), top_p=pick([0.0, 0.3, 0.9, 1.0, 1.5], F32),
           rho=pick([0.0, 1e-3, 0.5, 1.0], F32))


def test_settings_of_a_row_that_say_nothing():
    z, u = _logits(6, 200, F32, 1), _uniform(6)
    nan, inf = math.nan, math.inf
    bad = b.dvp_sample(z, u, temperature=torch.tensor([nan, -1.0, inf, 2e30, 1.0, 1e-35], device="cuda"))
    assert bad.ids.tolist()[:4] == [-1] * 4 and bad.count.tolist()[:4] == [0] * 4 and torch.isnan(bad.logp[:4]).all()
    assert bad.count[4] == 200 and bad.ids[5] == z[5].argmax() and bad.count[5] == 1
    bad = b.dvp_sample(z, u, top_p=torch.tensor([nan, -1.0, 2.0, 1.0, 0.0, inf], device="cuda"),
                       rho=torch.tensor([0.0, 0.0, 0.0, nan, 0.0, -1.0], device="cuda"))
    assert bad.ids[0] == -1 and bad.ids[3] == -1 and bad.count.tolist() == [0, 1, 200, 0, 1, 200]


@pytest.mark.parametrize("V", [64, 5000, 70001])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=3), dict(top_k=2500), dict(top_k=60000), dict(top_p=0.95), dict(top_p=0.3),
                                      dict(rho=1.0), dict(temperature=0.0), dict(rho=0.5, top_k=4000, top_p=0.5)], ids=str)
def test_equal_logits_stand_by_their_indices(V, settings):
    g = torch.Generator(device="cuda").manual_seed(V)
    same = torch.full((1, V), -2.5, device="cuda")
    two = torch.where(torch.rand(1, V, generator=g, device="cuda") < 0.5, 1.0, 1.25)
    few = torch.randint(0, 5, (1, V), generator=g, device="cuda") * 0.25 - 0.5     # on both sides of zero
    zeros = torch.where(torch.rand(1, V, generator=g, device="cuda") < 0.5, 0.0, -0.0)
    z = torch.cat([same, two, few, zeros])
    for dtype in (F32, BF16, F16):
        _check(z.to(dtype), _uniform(4), hints=(0, 1, 8), **settings)


@pytest.mark.parametrize("settings", [dict(top_k=5000), dict(top_p=0.5), dict(top_p=0.95, temperature=3.0)], ids=str)
@pytest.mark.parametrize("centre,scale", [(0.0, 1e-6), (0.0, 1e-38), (1000.0, 1e-3), (-7.0, 0.05), (0.0, 30.0)])
def test_dense_rows(settings, centre, scale):
    """Tens of thousands of logits around the cut, more than the list that is sorted holds."""
    g = torch.Generator(device="cuda").manual_seed(11)
    z = centre + scale * torch.randn(3, 100003, generator=g, device="cuda")
    _check(z, _uniform(3), hints=(0, 1, 4), **settings)
    _check(z.to(BF16), _uniform(3), hints=(0, 2), **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masked_rows(dtype):
    dt = DTYPES[dtype]
    V, inf = 5000, math.inf
    z = _logits(9, V, dt, 6)
    z[0] = -inf
    z[0, 4321] = -7.0                       # one token left
    z[1] = -inf                             # none
    z[2, ::2] = -inf
    z[3, 100:] = torch.finfo(dt).min        # the lowest value as the mask
    z[4] = torch.finfo(dt).min              # in the whole row: all equal
    z[5, 17] = math.nan
    z[6, 17] = inf
    z[7] = math.nan
    z[8, :4999] = -inf
    for settings in (dict(), dict(temperature=0.0), dict(temperature=0.25), dict(top_k=40), dict(top_k=4000), dict(top_p=0.9),
                     dict(rho=1e-3), dict(top_k=300, top_p=0.99, rho=1e-6)):
        got = _check(z, _uniform(9), hints=(0, 1, 4), **settings)
        assert got.ids.tolist()[1] == -1 and got.ids[0] == 4321 and got.ids[8] == 4999


def test_random_numbers_at_the_ends():
    z = _logits(8, 3000, BF16, 7)
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, math.inf, 2.0 ** -149], device="cuda")
    for settings in (dict(), dict(top_k=9), dict(top_p=0.9), dict(rho=1e-3)):
        _check(z, u, hints=(0, 1), **settings)


def test_draws_follow_the_distribution():
    """Random numbers on a fine grid: every token as often as its share, give or take one on each side."""
    n, V = 4096, 50
    row = _logits(1, V, F32, 8, boost=3.0)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    for settings in (dict(), dict(top_k=10), dict(top_p=0.8), dict(rho=0.1)):
        got = b.dvp_sample(row.expand(n, V).contiguous(), u, **settings)
        p = torch.softmax(row[0].double(), 0)
        kept = torch.zeros(V, dtype=torch.bool, device="cuda")
        kept[row[0].argsort(descending=True)[:int(got.count[0])]] = True
        p = torch.where(kept, p, 0.0) / p[kept].sum()
        assert ((torch.bincount(got.ids, minlength=V) - n * p).abs() <= 1.0 + 1e-6).all()


def test_a_draw_is_what_the_forward_pass_says_of_it():
    """ids, ln pi and ln pi^mp of a draw from the safe set are those that dvp_forward finds for the inference logits."""
    z = _logits(64, 20011, BF16, 10)
    rho = 1e-3
    got = b.dvp_sample(z, _uniform(64), rho=rho)
    fwd = b.dvp_forward(z, got.ids, rho, infer_logits=z)
    assert ((fwd.flags & b.DVP_FLAG_IN_INFER) != 0).all()
    assert torch.equal(fwd.infer.count, got.count)
    assert (fwd.infer.logp - got.logp).abs().max() < 1e-4 and (fwd.infer.logp_mp - got.logp_mp).abs().max() < 1e-4
    none = z.clone()
    none[5] = -math.inf
    assert b.dvp_sample(none, _uniform(64), rho=rho).ids[5] == -1


def test_id_types_and_reruns():
    z, u = _logits(40, 9000, F16, 12), _uniform(40)
    a, c = b.dvp_sample(z, u, top_p=0.9), b.dvp_sample(z, u, top_p=0.9, id_dtype=torch.int32)
    assert a.ids.dtype == torch.int64 and c.ids.dtype == torch.int32 and torch.equal(a.ids, c.ids.long())
    assert torch.equal(a.logp, c.logp) and torch.equal(a.logp_mp, c.logp_mp)


def test_captured_calls_and_two_streams():
    z, u = _logits(20, 30000, BF16, 13), _uniform(20)
    want = b.dvp_sample(z, u, top_p=0.9, top_k=500)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = b.dvp_sample(z, u, top_p=0.9, top_k=500)
    for _ in range(2):
        got.ids.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got.ids, want.ids) and torch.equal(got.logp_mp, want.logp_mp)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    pairs = [(b.dvp_sample(z, u, top_p=0.9, top_k=500, stream=stream), b.dvp_sample(z, u, rho=0.01, stream=other)) for _ in range(10)]
    torch.cuda.synchronize()
    alone = b.dvp_sample(z, u, rho=0.01)
    for x, y in pairs:
        assert torch.equal(x.ids, want.ids) and torch.equal(y.ids, alone.ids)


def test_empty_batch_and_refused_tensors():
    z, u = _logits(4, 100, F32, 1), _uniform(4)
    assert b.dvp_sample(z[:0], u[:0]).ids.shape == (0,)
    for bad in (lambda: b.dvp_sample(z, u[:3]), lambda: b.dvp_sample(z, u, top_p=u[:2]), lambda: b.dvp_sample(z.t(), u),
                lambda: b.dvp_sample(z, u.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: b.dvp_sample(z, u.double()), lambda: b.dvp_sample(z.double(), u), lambda: b.dvp_sample(z, u, top_k=u),
                lambda: b.dvp_sample(z, u, id_dtype=torch.int16)):
        with pytest.raises(TypeError):
            bad()
    for bad in (dict(temperature=-1.0), dict(rho=2.0), dict(top_p=-0.5), dict(launch_hint=5)):
        with pytest.raises(b.DvpError) as e:
            b.dvp_sample(z, u, **bad)
        assert e.value.status == b.DVP_ERR_INVALID_ARG
