"""Backward passes of attention over key ranges where a token does see an infinity: which gradients are no numbers goes by the formulas
and by the query's (the key's) own range, not by where the tiles that it is worked on in end, or by whether others see all of a tile.
Nothing here has a tolerance: what the formulas leave finite has the bits that it has without the infinity."""
import numpy as np
import pytest
import torch

from paper_2603_22370_b200 import faar
from tests.test_gpu_scored_attention import Case, ctx  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu
INF = float("inf")


def broken(t):
    return (~torch.isfinite(t)).any(1)


def ranges_of_two_documents(S, cut):
    """Two documents: the second one's tiles have keys to mask on either side."""
    at = np.arange(S)
    return np.where(at < cut, 0, cut)[None], (at + 1)[None]


def runs(ctx, c, which, at, value):  # noqa: F811
    """outputs without and with one element of one token's row (of all heads) replaced"""
    B, S, H, HKV, D = c.dims
    c.run(ctx)
    clean = [t.clone() for t in c.outputs()]
    t = {"q": c.Q, "k": c.K, "v": c.V, "do": c.DO}[which]
    n = HKV if which in "kv" else H
    t[at, [h * D + 5 for h in range(n)]] = value
    c.new()
    c.run(ctx)
    torch.cuda.synchronize()
    faar.attention_status(ctx)
    return clean, [t.clone() for t in c.outputs()]


# tokens whose tiles are partly masked for some, and wholly seen by later ones; the second document begins within a tile of 64 and of 128
CUT, S = 150, 420
PLACES = [0, 70, 149, 150, 200, 419]


def who_sees(at):
    """queries that see key `at`, and the rest"""
    last = CUT if at < CUT else S
    return list(range(at, last)), [t for t in range(S) if not at <= t < last]


def whom_it_sees(at):
    first = 0 if at < CUT else CUT
    return list(range(first, at + 1)), [u for u in range(S) if not first <= u <= at]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("at", PLACES)
def test_an_infinite_key_leaves_no_gradient_to_those_who_see_it(ctx, D, cap, value, at):  # noqa: F811
    """dQ = dS K: whatever dS is there, 0 times an infinity is no number (a score of minus infinity, or a capped one, leaves the outputs
    themselves finite)."""
    c = Case(1, S, 2, 1, D, *ranges_of_two_documents(S, CUT), cap, pad=0)
    clean, got = runs(ctx, c, "k", at, value)
    see, rest = who_sees(at)
    for h in range(2):
        dq, dq0 = got[2][:, h * D:(h + 1) * D], clean[2][:, h * D:(h + 1) * D]
        assert broken(dq[see]).all()
        assert torch.equal(dq[rest], dq0[rest])
