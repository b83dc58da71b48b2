"""The operators of the rollout's last stage and of the norm before the LM head, and the calls that a program makes of them:
root-mean-square norm (forward with an output in 8 bits or in the model's type, and backward), the LM head's product in
8-bit floating point with a scale for each block of 128, and sampling with temperature, top-k, top-p and min-p.

``listed()`` are fixed workloads, ``draw()`` gives further ones from the same ranges.  With ``own`` false ``run`` computes the
operators in their plain form, elementary tensor operations; with ``own`` true it calls this library.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128          # columns (and rows of a weight) that share a scale
FP8_MAX = 448.0      # the largest value of e4m3
PAPER_RHO = math.exp(-13.0)
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2, "fp8": 1}


# ---- cases ---------------------------------------------------------------------------------------------------------

def _norm(T, H, dtype, out, residual=True):
    return {"kind": "norm", "T": T, "H": H, "dtype": dtype, "out": out, "residual": residual}


def _norm_backward(T, H, dtype, dy, d_residual=True):
    return {"kind": "norm_backward", "T": T, "H": H, "dtype": dtype, "dy": dy, "d_residual": d_residual}


def _product(T, H, V, out):
    return {"kind": "product", "T": T, "H": H, "V": V, "out": out}


def _sample(T, V, dtype, temperature=1.0, top_k=0, top_p=1.0, rho=0.0, mixed=False, pad=0):
    """``mixed``: every row has a temperature, top_k, top_p and rho of its own, as the requests of a serving batch."""
    return {"kind": "sample", "T": T, "V": V, "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
            "rho": rho, "mixed": mixed, "pad": pad}


def listed():
    return [
        # the final norm of a decoding step of eight rollouts: launch and latency
        dict(_norm(8, 4096, "bf16", "fp8"), name="decode_norm_fp8"),
        # the final norm when a batch of responses is scored with the rollout's 8-bit head
        dict(_norm(16384, 4096, "bf16", "fp8"), name="batch_norm_fp8"),
        # a width that no vector divides, rows back to back, without a residual, in the model's own type
        dict(_norm(1111, 5003, "f16", "f16", False), name="odd_norm_f16"),
        # the training step's way back through the final norm, from the LM head's float32 gradient
        dict(_norm_backward(16384, 4096, "bf16", "f32"), name="batch_norm_backward"),
        # the same for one response of a small model, all in float32
        dict(_norm_backward(512, 1024, "f32", "f32", False), name="small_norm_backward"),
        # logits of a decoding step of sixteen rollouts: every weight is read for little work
        dict(_product(16, 4096, 151936, "bf16"), name="decode_head_fp8"),
        # odd token and vocabulary counts, a short and ragged contraction
        dict(_product(163, 416, 45277, "f32"), name="odd_head_fp8"),
        # logits of a batch of responses
        dict(_product(4096, 4096, 151936, "bf16"), name="batch_head_fp8"),
        # the next token of one rollout from the paper's safe set
        dict(_sample(1, 151936, "bf16", rho=PAPER_RHO), name="one_token_min_p"),
        # a serving batch whose requests bring their own settings
        dict(_sample(64, 151936, "bf16", mixed=True), name="decode_mixed"),
        # rollouts of a reinforcement-learning step: temperature 1, nucleus of 0.95
        dict(_sample(1024, 151936, "bf16", top_p=0.95), name="rollout_top_p"),
        # float32 logits of a 262,144-token vocabulary, the fifty largest
        dict(_sample(128, 262144, "f32", temperature=0.7, top_k=50), name="long_vocabulary_top_k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "product", "sample", "sample"])
    if kind in ("norm", "norm_backward"):
        H = rng.choice([_log_int(rng, 64, 16384), 8 * _log_int(rng, 8, 2048), 128 * _log_int(rng, 1, 128)])
        T = max(1, min(_log_int(rng, 1, 32768), 16384 * 4096 // H))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if kind == "norm":
            return _norm(T, H, dtype, rng.choice(["fp8", "fp8", dtype]), rng.random() < 0.7)
        return _norm_backward(T, H, dtype, rng.choice(["f32", dtype]), rng.random() < 0.5)
    if kind == "product":
        H = rng.choice([_log_int(rng, 64, 8192), 128 * _log_int(rng, 1, 64)])
        V = min(152000, max(64, int(6.2e8 / H)), _log_int(rng, 1000, 152000))
        T = max(1, min(_log_int(rng, 1, 8192), int(2.5e12 / (H * V)), int(6.2e8 / V)))
        return _product(T, H, V, rng.choice(["bf16", "bf16", "f16", "f32"]))
    V = _log_int(rng, 1000, 262144)
    V = V // 64 * 64 if rng.random() < 0.5 else V
    T = max(1, min(_log_int(rng, 1, 2048), 1024 * 151936 // V))
    dtype, pad = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 16 - V % 16])
    if rng.random() < 0.4:
        return _sample(T, V, dtype, mixed=True, pad=pad)
    return _sample(T, V, dtype, rng.choice([1.0, 1.0, 0.6, 1.2, 0.0]), rng.choice([0, 0, 1, 20, _log_int(rng, 2, 1000)]),
                   rng.choice([1.0, 1.0, 0.9, 0.95, 0.99]), rng.choice([0.0, 1e-4, 0.05, PAPER_RHO]), pad=pad)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _round_fp8(v):
    return v.clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)


def _columns(scale, n):
    """A scale for each block of columns, at each of n columns."""
    return scale.repeat_interleave(BLOCK, dim=1)[:, :n]


def _fp8_rows(v):
    """Rows in 8 bits with a scale for each 128 columns; rows start on 16-byte boundaries."""
    T, H = v.shape
    n, ld = -(-H // BLOCK), -(-H // 16) * 16
    blocks = torch.nn.functional.pad(v, (0, n * BLOCK - H)).view(T, n, BLOCK)
    scale = blocks.abs().amax(2).clamp(min=2.0 ** -96) / FP8_MAX
    q = torch.zeros(T, ld, dtype=torch.float8_e4m3fn, device=v.device)
    q[:, :H] = _round_fp8((blocks / scale[:, :, None]).reshape(T, n * BLOCK)[:, :H])
    return q[:, :H], scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = _generator(seed, dev)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    state = {"case": case}
    if case["kind"] in ("norm", "norm_backward"):
        T, H, dt = case["T"], case["H"], _TYPES[case["dtype"]]
        state["weight"] = (1.0 + 0.2 * normal(H)).to(dt)
        if case["kind"] == "norm":
            state["x"] = normal(T, H).to(dt)
            state["residual"] = (3.0 * normal(T, H)).to(dt) if case["residual"] else None
        else:
            state["h"] = (3.0 * normal(T, H)).to(dt)
            state["rstd"] = torch.rsqrt(state["h"].float().square().mean(1) + 1e-6)
            state["dy"] = normal(T, H).to(_TYPES[case["dy"]])
            state["d_residual"] = normal(T, H).to(dt) if case["d_residual"] else None
    elif case["kind"] == "product":
        T, H, V = case["T"], case["H"], case["V"]
        # hidden states with a few large channels, as a norm's weight makes them; weights of the repository's LM head
        loud = torch.exp(normal(H))
        state["a"], state["a_scale"] = _fp8_rows(normal(T, H) * loud)
        rows, cols = -(-V // BLOCK), -(-H // BLOCK)
        state["b_scale"] = 0.02 * 4.5 / FP8_MAX * torch.exp(0.3 * normal(rows, cols))
        w = torch.zeros(V, -(-H // 16) * 16, dtype=torch.float8_e4m3fn, device=dev)
        for r in range(0, V, 16384):
            n = min(16384, V - r)
            w[r:r + n, :H] = _round_fp8(normal(n, H) * (FP8_MAX / 4.5))
        state["b"] = w[:, :H]
    else:
        T, V, dt = case["T"], case["V"], _TYPES[case["dtype"]]
        z = torch.empty(T, V + case["pad"], dtype=dt, device=dev)[:, :V]
        for r in range(0, T, 512):
            n = min(512, T - r)
            # between an open position (all of a wide distribution) and a decided one (a few tokens far above it)
            head = torch.randint(0, V, (n, 8), generator=g, device=dev)
            base = 3.0 * normal(n, V)
            boost = 15.0 * torch.rand(n, 1, generator=g, device=dev) + normal(n, 8)
            base.scatter_add_(1, head, boost)
            z[r:r + n] = base.to(dt)
            del base
        state["logits"] = z
        state["uniform"] = torch.rand(T, generator=g, device=dev)
        for name in ("temperature", "top_k", "top_p", "rho"):
            state[name] = case[name]
        if case["mixed"]:
            def pick(values, dtype):
                at = torch.randint(0, len(values), (T,), generator=g, device=dev)
                return torch.tensor(values, dtype=dtype, device=dev)[at]
            state["temperature"] = pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.2], torch.float32)
            state["top_k"] = pick([0, 0, 1, 20, 50, 200], torch.int32)
            state["top_p"] = pick([1.0, 1.0, 0.9, 0.95, 0.99], torch.float32)
            state["rho"] = pick([0.0, 0.0, 1e-4, 0.05], torch.float32)
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------

def _plain_norm(s):
    c = s["case"]
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = torch.rsqrt(h.square().mean(1) + 1e-6)
    y = h * rstd[:, None] * s["weight"].float()
    out = {"rstd": rstd}
    if s["residual"] is not None:
        out["residual"] = h.to(s["x"].dtype)
    if c["out"] == "fp8":
        out["y"], out["scale"] = _fp8_rows(y)
    else:
        out["y"] = y.to(_TYPES[c["out"]])
    return out


def _plain_norm_backward(s):
    h, rstd = s["h"].float(), s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["weight"].float()
    dh = rstd * (g - h * rstd.square() * (g * h).mean(1, keepdim=True))
    if s["d_residual"] is not None:
        dh = dh + s["d_residual"].float()
    return {"d_x": dh.to(s["h"].dtype), "d_weight": (dy * h * rstd).sum(0)}


def _plain_product(s):
    T, H = s["a"].shape
    a = s["a"].float() * _columns(s["a_scale"], H)
    b = s["b"].float() * _columns(s["b_scale"].repeat_interleave(BLOCK, dim=0)[:s["b"].shape[0]], H)
    return {"logits": (a @ b.t()).to(_TYPES[s["case"]["out"]])}


def _of_rows(v, z, dtype):
    """A setting, one for all rows or one a row, as a column."""
    v = v if torch.is_tensor(v) else torch.full((z.shape[0],), v, dtype=dtype, device=z.device)
    return v.to(dtype)[:, None]


def _plain_sample(s):
    z = s["logits"].float()
    T, V = z.shape
    f64 = torch.float64
    temperature, top_p, rho = (_of_rows(s[n], z, f64) for n in ("temperature", "top_p", "rho"))
    top_k = _of_rows(s["top_k"], z, torch.int64)
    greedy = temperature == 0
    temperature = torch.where(greedy, 1.0, temperature)
    top = z.amax(1, keepdim=True).to(f64)
    x = (z.to(f64) - top) / temperature
    w = torch.exp(x)
    total = w.sum(1)
    values, order = torch.sort(z, dim=1, descending=True, stable=True)
    values = values.to(f64)
    rank = torch.arange(V, device=z.device)
    keep = (values >= top + temperature * torch.log(rho)) & (values > -math.inf)
    keep &= (top_k <= 0) | (rank < top_k)
    keep &= ~greedy | (rank < 1)
    mass = torch.exp((values - top) / temperature) * keep
    del values
    before = torch.cumsum(mass, 1) - mass
    keep &= (top_p >= 1) | (before < top_p * mass.sum(1, keepdim=True)) | (rank == 0)
    del mass, before
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    del order
    reach = torch.cumsum(w * kept, 1)
    aim = s["uniform"].to(f64)[:, None] * reach[:, -1:]
    last = torch.where(kept, rank, -1).amax(1, keepdim=True)
    ids = torch.minimum(torch.searchsorted(reach, aim, right=True), last)
    at = x.gather(1, ids)[:, 0]
    return {"ids": ids[:, 0], "logp": (at - torch.log(total)).float(), "logp_mp": (at - torch.log(reach[:, -1])).float(),
            "count": keep.sum(1).to(torch.int32)}


_PLAIN = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "product": _plain_product, "sample": _plain_sample}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return _PLAIN[kind](state)
    from paper_2512_23087_b200 import binding
    if kind == "norm":
        r = binding.dvp_rms_norm(state["x"], state["weight"], residual=state["residual"], eps=1e-6,
                                 out_dtype=_TYPES[state["case"]["out"]])
        out = {"y": r.y, "rstd": r.rstd}
        if state["residual"] is not None:
            out["residual"] = r.residual
        if r.scale is not None:
            out["scale"] = r.scale
        return out
    if kind == "norm_backward":
        r = binding.dvp_rms_norm_backward(state["dy"], state["h"], state["weight"], state["rstd"],
                                          d_residual=state["d_residual"])
        return {"d_x": r.d_x, "d_weight": r.d_weight}
    if kind == "product":
        logits, _ = binding.dvp_gemm_fp8(state["a"], state["a_scale"], state["b"], state["b_scale"],
                                         out_dtype=_TYPES[state["case"]["out"]])
        return {"logits": logits}
    r = binding.dvp_sample(state["logits"], state["uniform"], temperature=state["temperature"], top_k=state["top_k"],
                           top_p=state["top_p"], rho=state["rho"])
    return {"ids": r.ids, "logp": r.logp, "logp_mp": r.logp_mp, "count": r.count}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    T = case["T"]
    if case["kind"] == "norm":
        H, z, o = case["H"], _BYTES[case["dtype"]], _BYTES[case["out"]]
        scales = 4.0 * T * -(-H // BLOCK) if case["out"] == "fp8" else 0.0
        return {"bytes": float(T) * H * (z * (3 if case["residual"] else 1) + o) + z * H + 4.0 * T + scales, "flops": 6.0 * T * H}
    if case["kind"] == "norm_backward":
        H, z, d = case["H"], _BYTES[case["dtype"]], _BYTES[case["dy"]]
        return {"bytes": float(T) * H * (d + z * (3 if case["d_residual"] else 2)) + (z + 4.0) * H + 4.0 * T,
                "flops": 10.0 * T * H}
    if case["kind"] == "product":
        H, V, n = case["H"], case["V"], -(-case["H"] // BLOCK)
        return {"bytes": float(T + V) * H + 4.0 * n * (T + -(-V // BLOCK)) + float(_BYTES[case["out"]]) * T * V,
                "flops": 2.0 * T * H * V}
    # a difference, a product, an exponential and an addition per logit
    return {"bytes": float(_BYTES[case["dtype"]]) * T * case["V"] + 24.0 * T, "flops": 4.0 * T * case["V"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def _exact_row(z, u, temperature, top_k, top_p, rho):
    """One row: (id, ln pi, ln pi of the kept set, kept tokens)."""
    z = z.double()
    t = temperature if temperature > 0 else 1.0
    y = z / t
    lse = torch.logsumexp(y, 0)
    order = torch.argsort(-z, stable=True)
    n = int((z >= z.max() + (t * math.log(rho) if rho > 0 else -math.inf)).sum())
    if temperature == 0:
        n = 1
    elif top_k > 0:
        n = min(n, top_k)
    p = torch.softmax(y[order[:n]], 0)
    if top_p < 1:
        # the fewest of the largest that reach top_p
        n = min(n, int((torch.cumsum(p, 0) < top_p).sum()) + 1)
    kept = torch.sort(order[:n]).values
    p = torch.softmax(y[kept], 0)
    i = min(int((torch.cumsum(p, 0) <= u).sum()), n - 1)
    a = kept[i]
    return a, y[a] - lse, torch.log(p[i]) if float(p[i]) < 0.5 else torch.log1p(-(p[:i].sum() + p[i + 1:].sum())), n


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        h = s["x"].double() + (s["residual"].double() if s["residual"] is not None else 0.0)
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / case["H"] + 1e-6)
        out = {"rstd": rstd}
        if s["residual"] is not None:
            out["residual"] = h
        y = torch.einsum("th,t,h->th", h, rstd, s["weight"].double())
        if case["out"] != "fp8":
            return dict(out, y=y)
        T, H = y.shape
        scale = torch.stack([b.abs().amax(1) for b in y.split(BLOCK, 1)], 1).clamp(min=2.0 ** -96) / FP8_MAX
        return dict(out, scale=scale, y=(y / _columns(scale, H)))
    if case["kind"] == "norm_backward":
        h, rstd, dy, w = (s[n].double() for n in ("h", "rstd", "dy", "weight"))
        unit = torch.einsum("th,t->th", h, rstd)
        g = dy * w
        dh = torch.einsum("th,t->th", g, rstd) - torch.einsum("th,t->th", unit, rstd * (g * unit).sum(1) / case["H"])
        if s["d_residual"] is not None:
            dh += s["d_residual"].double()
        return {"d_x": dh, "d_weight": torch.einsum("th,th->h", dy, unit)}
    if case["kind"] == "product":
        out = torch.zeros(case["T"], case["V"], dtype=torch.float64, device=s["a"].device)
        for j, k in enumerate(range(0, case["H"], BLOCK)):
            n = min(BLOCK, case["H"] - k)
            a = s["a"][:, k:k + n].double() * s["a_scale"][:, j:j + 1].double()
            rows = s["b_scale"][:, j].double().repeat_interleave(BLOCK)[:case["V"]]
            out += a @ (s["b"][:, k:k + n].double() * rows[:, None]).t()
        return {"logits": out}
    settings = {n: s[n].tolist() if torch.is_tensor(s[n]) else [s[n]] * case["T"] for n in ("temperature", "top_k", "top_p", "rho")}
    uniform = s["uniform"].tolist()
    rows = [_exact_row(s["logits"][t], uniform[t], settings["temperature"][t], settings["top_k"][t], settings["top_p"][t],
                       settings["rho"][t]) for t in range(case["T"])]
    dev = s["logits"].device
    return {"ids": torch.stack([r[0] for r in rows]), "logp": torch.stack([r[1] for r in rows]),
            "logp_mp": torch.stack([r[2] for r in rows]),
            "count": torch.tensor([r[3] for r in rows], dtype=torch.int32, device=dev)}
