"""Long rows with tokens that are not to be drawn, of which one random number after the other is drawn: every token against the
definition in float64.  The rows are so long that a warp keeps one sum for several of its pieces."""
import math

import numpy as np
import pytest
import torch

from paper_2512_23087_b200 import binding as b

from test_sample_gpu import DTYPES

pytestmark = pytest.mark.gpu
WARPS = 16
INF = math.inf


def _row(V, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (2.0 * torch.randn(V, generator=g, device="cuda")).to(DTYPES[dtype])


def _mask_fronts(z, blocks, lengths):
    """-inf in the first of the logits of each warp, where `blocks` blocks share the row."""
    piece = 32 * 32 // z.element_size()
    pieces = -(-z.numel() // piece)
    per_block = -(-pieces // blocks)
    for k in range(blocks):
        per_warp = -(-max(0, min(per_block, pieces - k * per_block)) // WARPS)
        for w in range(WARPS):
            at = (k * per_block + w * per_warp) * piece
            z[at:at + lengths[w % len(lengths)]] = -INF
    return z


def _only_runs(z, runs, length, seed):
    """-inf but for short runs of neighbouring tokens, as a grammar leaves them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    at = torch.randint(0, z.numel() - length, (runs, 1), generator=g, device="cuda")
    keep = torch.zeros(z.numel(), dtype=torch.bool, device="cuda")
    keep[(at + torch.arange(length, device="cuda")).flatten()] = True
    return z.masked_fill(~keep, -INF)


def _want(z, u, top_p):
    """The tokens that the random numbers draw from the row, and the number of tokens kept."""
    z = z.double().cpu().numpy()
    w = np.exp(z - z.max())
    kept = np.flatnonzero(z > -np.inf)
    if top_p < 1:
        order = kept[np.lexsort((kept, -z[kept]))]
        run = np.cumsum(w[order])
        kept = np.sort(order[:max(1, int((run - w[order] < top_p * run[-1]).sum()))])
    run = np.cumsum(w[kept])
    return kept[np.searchsorted(run, u.double().cpu().numpy() * run[-1], side="right")], kept.size


def _check(z, hints, n=200):
    u = (torch.arange(n, device="cuda") + 0.37) / n
    rows = z.expand(n, -1).contiguous()
    for top_p in (1.0, 0.9):
        ids, count = _want(z, u, top_p)
        for hint in hints:
            got = b.dvp_sample(rows, u, top_p=top_p, launch_hint=hint)
            assert (got.count == count).all(), (top_p, hint)
            wrong = int((got.ids.cpu() != torch.from_numpy(ids)).sum())
            assert wrong == 0, (top_p, hint, wrong)


@pytest.mark.parametrize("dtype,V", [("f32", 262208), ("f32", 600011), ("bf16", 600011), ("f16", 600016)])
@pytest.mark.parametrize("blocks", [1, 2])
def test_warps_that_begin_with_tokens_that_are_not_to_be_drawn(dtype, V, blocks):
    piece = 32 * 32 // DTYPES[dtype].itemsize
    lengths = (piece, 2 * piece, piece + piece // 2, 3 * piece)
    _check(_mask_fronts(_row(V, dtype, 1), blocks, lengths), hints=(blocks,))


@pytest.mark.parametrize("dtype,V", [("f32", 262208), ("f32", 600011), ("bf16", 600011)])
def test_short_runs_that_may_be_drawn(dtype, V):
    _check(_only_runs(_row(V, dtype, 2), 200, 50, 3), hints=(1, 2))


@pytest.mark.parametrize("dtype,V", [("f32", 262208), ("bf16", 600011)])
def test_one_warp_alone_may_be_drawn_from(dtype, V):
    z = _row(V, dtype, 4)
    z[:V // 2] = -INF
    z[V // 2 + 20000:] = -INF
    _check(z, hints=(1, 2))
