"""The backward pass of attention over key ranges takes delta = dout . out from the BF16 output, and its dQ kernel makes good what that
delta lacks: the lack is the sum along a row of P (dP - delta), dQ is corrected by it times the sum of P (times the cap's slope) K, and dK
is formed from the exact delta.  An `out` that is something else altogether has to give the same gradients, then, and a correction that
is left out or wrong shows at its full size instead of at half a step of `out`.

Bounds, carried through those formulas (an upright bar is a magnitude, `given` what delta is taken as): P is off by `err` of itself (its
score's error, 2^x and lse), P (dP - given) and P by another half step as operands, FP32 sums by 2^-18 of their magnitudes, tanh by 2^-20.
  lack   sum of P (|dP| + |given|) times (err + 2^-18), and dP's own error
  dQ     (what an operand of P (dP - given) is off by) |K| + |lack| (what one of P is off by) |K| + (the lack's error) P |K| + half a step
  dK     as with the exact delta, which is off by the lack's error
Products of two such errors are allowed for by a factor of 1.02 (all of them are below 2^-6)."""
import numpy as np
import pytest
import torch

from oracle import block_forms_oracle as bo
from paper_2603_22370_b200 import faar, inputs
from tests.gpu_helpers import DEV, dev_bf16, dev_f32, host

HALF_STEP, SUM, F32 = 2.0 ** -8, 2.0 ** -18, 2.0 ** -20
bf16 = lambda a: inputs.to_bf16_f32(a).astype(np.float64)
T = lambda x: x.transpose(0, 1, 3, 2)


class Problem:
    def __init__(self, B, S, H, G, D, cap, biased, q_scale, documents):
        self.dims, self.cap = (B, S, H, G, D), cap
        rng = np.random.default_rng(S + D)
        draw = lambda n, scale=1.0: inputs.to_bf16_f32(rng.standard_normal((B * S, n * D)) * scale)
        self.q, self.k, self.v, self.do, self.given = draw(H, q_scale), draw(G), draw(G), draw(H), draw(H, 4.0)
        self.slopes = [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)] if biased else None
        at = np.arange(S)
        self.lo = np.broadcast_to(at // documents * documents, (B, S))
        self.hi = np.broadcast_to(at + 1, (B, S))
        out, self.lse, saved = bo.scored_attention(self.q, self.k, self.v, *self.dims, self.lo, self.hi, cap, self.slopes)
        self.dq, self.dk, _ = bo.scored_attention_bwd(self.do, self.q, self.k, self.v, saved, *self.dims)
        self.P, self.tanh, self.scale, self.seen = saved
        heads = lambda x, n: bo._split(x, B, S, n).repeat(H // n, 1)
        self.qh, self.kh, self.vh, self.doh = heads(self.q, H), heads(self.k, G), heads(self.v, G), heads(self.do, H)
        self.dP = np.where(self.seen[:, None], self.doh @ T(self.vh), 0)
        self.delta, self.delta_given = ((self.doh * heads(o, H)).sum(3, keepdims=True) for o in (out, self.given))
        self.e_given = SUM * (np.abs(self.doh) * np.abs(heads(self.given, H))).sum(3, keepdims=True)
        self.slope = 1.0 if self.tanh is None else 1.0 - self.tanh ** 2

    def shared(self, g):
        B, S, H, G, D = self.dims
        return bo._rows(g.reshape(B, G, H // G, S, D).sum(2))

    def bounds(self):
        at, s, p, sl = np.arange(self.dims[1]), self.scale, self.P, self.slope
        es = SUM * np.abs(self.qh) @ T(np.abs(self.kh)) * s + F32 * self.cap
        if self.slopes is not None:
            es = es + F32 * np.asarray(self.slopes)[:, None, None] * np.abs(at[:, None] - at)
        es = np.where(self.seen[:, None], es, 0).max(3, keepdims=True)
        err = 2 * es + 4 * F32
        edp = SUM * np.abs(self.doh) @ T(np.abs(self.vh))
        given = np.abs(self.delta_given) + self.e_given
        e_lack = (p * (np.abs(self.dP) * (err + SUM) + edp)).sum(3, keepdims=True) + given * (err + SUM)
        lack = np.abs(self.delta - self.delta_given) + self.e_given
        off = np.abs(self.dP - self.delta_given)
        e_w = p * (sl * HALF_STEP + err + 4 * F32 + SUM)
        e_ds = p * s * ((err + 4 * F32 + SUM) * (np.abs(self.dP) + given) + edp + sl * HALF_STEP * off)
        k = np.abs(self.kh)
        tol_q = bo._rows(e_ds @ k + s * lack * (e_w @ k) + s * e_lack * ((p * sl) @ k)) + HALF_STEP * np.abs(self.dq)
        e_ds = p * s * ((err + 4 * F32 + SUM) * (np.abs(self.dP) + np.abs(self.delta)) + edp + e_lack + sl * HALF_STEP * np.abs(self.dP - self.delta))
        tol_k = self.shared(T(e_ds) @ np.abs(self.qh)) + HALF_STEP * np.abs(self.dk)
        return 1.02 * tol_q + 1e-30, 1.02 * tol_k + 1e-30

    def emulated(self, mistake=None):
        """dQ and dK as the kernels form them, with their roundings"""
        p, s, sl = self.P, self.scale, self.slope
        flat = p * (self.dP - self.delta_given) * s
        lack = (flat * (sl if mistake == "slope in the lack" else 1.0)).sum(3, keepdims=True)
        if mistake == "none":
            lack = 0 * lack
        if mistake == "sign":
            lack = -lack
        w = bf16(p if mistake == "no slope beside K" else p * sl)
        dq = bf16(bo._rows(bf16(flat * sl) @ self.kh - lack * (w @ self.kh)))
        delta = self.delta_given + (0 if mistake == "delta not left to dK" else lack / s)
        return dq, bf16(self.shared(T(bf16(p * (self.dP - delta) * s * sl)) @ self.qh))


PROBLEMS = [(2, 100, 4, 2, 64, 0.0, False, 1.5, 100), (1, 200, 2, 1, 64, 4.0, False, 4.0, 70), (2, 333, 2, 1, 128, 0.0, True, 1.5, 150),
            (1, 150, 4, 1, 128, 6.0, True, 5.0, 40), (1, 64, 2, 2, 64, 3.0, True, 3.0, 20)]


@pytest.mark.parametrize("args", PROBLEMS)
def test_the_bounds_hold_for_the_formula_and_for_no_mistake_in_it(args):
    problem = Problem(*args)
    tol = problem.bounds()
    over = lambda got: [(np.abs(g - r) / t).max() for g, r, t in zip(got, (problem.dq, problem.dk), tol)]
    assert max(over(problem.emulated())) <= 1
    both = ["none", "sign"] + (["slope in the lack"] if problem.cap else [])
    for mistake in both:
        assert min(over(problem.emulated(mistake))) > 4, mistake
    if problem.cap:
        assert over(problem.emulated("no slope beside K"))[0] > 4
    assert over(problem.emulated("delta not left to dK"))[1] > 4


@pytest.mark.gpu
@pytest.mark.parametrize("args", PROBLEMS)
def test_gradients_do_not_depend_on_the_output_that_delta_is_taken_from(args):
    from paper_2603_22370_b200 import build
    build.build()
    ctx = faar.Context(0)
    problem = Problem(*args)
    B, S, H, G, D = problem.dims
    q, k, v, do, given = (dev_bf16(a) for a in (problem.q, problem.k, problem.v, problem.do, problem.given))
    ranges = [torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV) for a in (problem.lo, problem.hi)]
    scores = faar.make_attention_scores(0.0, problem.cap, None if problem.slopes is None else dev_f32(problem.slopes), *ranges)
    out, lse = torch.empty_like(q), torch.empty((B, H, S), device=DEV)
    scratch = torch.empty(faar.attention_scored_scratch_size(B, S, H), dtype=torch.uint8, device=DEV)
    dq, dk, dv, dv2 = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k), torch.empty_like(k)
    faar.attention_scored_fwd(ctx, B, S, H, G, D, q, H * D, k, v, G * D, scores, out, H * D, lse)
    faar.attention_scored_bwd(ctx, B, S, H, G, D, q, H * D, k, v, G * D, scores, out, do, H * D, lse, scratch, dq, dk, dv2)
    faar.attention_scored_bwd(ctx, B, S, H, G, D, q, H * D, k, v, G * D, scores, given, do, H * D, lse, scratch, dq, dk, dv)
    torch.cuda.synchronize()
    faar.attention_status(ctx)
    for got, ref, tol, name in zip((dq, dk), (problem.dq, problem.dk), problem.bounds(), ("dq", "dk")):
        over = np.abs(host(got) - ref) / tol
        assert np.isfinite(host(got)).all() and over.max() <= 1, (name, over.max(), np.unravel_index(over.argmax(), over.shape))
    assert torch.equal(dv, dv2)                                # dV holds no delta
    ctx.close()
