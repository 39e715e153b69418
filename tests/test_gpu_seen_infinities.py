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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [INF, -INF, float("nan")])
@pytest.mark.parametrize("at", PLACES)
def test_values_do_not_enter_the_gradient_of_values(ctx, D, value, at):  # noqa: F811
    """dV = P^T dO: a v that is no number leaves it as it is, while the outputs, dQ and dK of those who see it are no numbers."""
    c = Case(1, S, 2, 1, D, *ranges_of_two_documents(S, CUT), 20.0, pad=0)
    clean, got = runs(ctx, c, "v", at, value)
    see, rest = who_sees(at)
    assert torch.equal(got[4], clean[4])
    assert broken(got[0][see]).all() and broken(got[2][see]).all()
    assert torch.equal(got[0][rest], clean[0][rest]) and torch.equal(got[2][rest], clean[2][rest])


@pytest.mark.parametrize("heads", [(2, 1, 1), (8, 2, 3), (2, 2, 80)])          # dealt over clusters, and whole key tiles
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [INF, float("nan")])
@pytest.mark.parametrize("at", PLACES)
def test_a_gradient_that_is_no_number_reaches_the_values_that_were_seen(ctx, D, value, at, heads):  # noqa: F811
    H, G, B = heads
    lo, hi = (np.repeat(a, B, 0) for a in ranges_of_two_documents(S, CUT))
    c = Case(B, S, H, G, D, lo, hi, 0.0, pad=0)
    clean, got = runs(ctx, c, "do", at, value)
    seen, rest = whom_it_sees(at)
    rest = rest + list(range(S, B * S))                          # and the other sequences
    for i in (3, 4):
        for g in range(G):
            cols = slice(g * D, (g + 1) * D)
            assert broken(got[i][seen][:, cols]).all() and torch.equal(got[i][rest][:, cols], clean[i][rest][:, cols])
    assert torch.equal(got[0], clean[0])


@pytest.mark.parametrize("heads", [(2, 1, 1), (8, 2, 3), (2, 2, 80)])          # dealt over clusters, and whole key tiles
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("at", PLACES)
def test_an_infinite_query_leaves_no_gradient_to_the_keys_that_it_sees(ctx, D, cap, value, at, heads):  # noqa: F811
    """dK = dS^T Q; with a cap its probabilities, and so dV and its own dQ, are finite."""
    H, G, B = heads
    lo, hi = (np.repeat(a, B, 0) for a in ranges_of_two_documents(S, CUT))
    c = Case(B, S, H, G, D, lo, hi, cap, pad=0)
    clean, got = runs(ctx, c, "q", at, value)
    seen, rest = whom_it_sees(at)
    rest = rest + list(range(S, B * S))
    for g in range(G):
        cols = slice(g * D, (g + 1) * D)
        assert broken(got[3][seen][:, cols]).all()
        for i in (3, 4):
            assert torch.equal(got[i][rest][:, cols], clean[i][rest][:, cols])
    if cap:
        assert torch.isfinite(got[4]).all() and torch.isfinite(got[2]).all() and torch.isfinite(got[0]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", ["k", "q", "do"])
@pytest.mark.parametrize("at", [2111, 2240, 4299])
def test_tiles_far_into_a_sequence(ctx, D, which, at):  # noqa: F811
    """The same beyond 32 tiles, with edge tiles in the middle and the diagonal's."""
    n, cut = 4300, 2139
    c = Case(1, n, 4, 2, D, *ranges_of_two_documents(n, cut), 20.0, pad=0)
    clean, got = runs(ctx, c, which, at, INF)
    first, last = (0, cut) if at < cut else (cut, n)
    heads, own = {"k": (4, 2), "q": (2, 3), "do": (2, 4)}[which]
    hit = list(range(at, last) if which == "k" else range(first, at + 1))
    rest = sorted(set(range(n)) - set(hit))
    for h in range(heads):
        cols = slice(h * D, (h + 1) * D)
        assert broken(got[own][hit][:, cols]).all() and torch.equal(got[own][rest][:, cols], clean[own][rest][:, cols])
