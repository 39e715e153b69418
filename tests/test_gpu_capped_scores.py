"""The tanh of capped scores by itself: a sequence of one token has its own score as its lse, in FP32.

In units of the cap a score is t = q k / cap, formed exactly here (one product of two BF16 values, a cap and a scale that are powers of
two).  Where |t| <= sqrt(3)/2 its tanh is a polynomial that is off by 1.4e-7 of it (2^-22.8), evaluated in FP32: the last two multiply-adds
of the chain, t t, the product with t and the coefficients' own rounding are off by 2^-24 each, the inner ones by a third of that and
less: 1.4e-7 + 5 * 2^-24 < 2^-21.2.  Beyond, tanh = 1 - 2 r with r = 1 / (1 + 2^(2 t log2 e)) <= 0.151: 2^x is off by 2^-22 and by the
rounding of its argument, r by 2^-23, the cap's rounding and the last step by 2^-24 each: at t = 0.866, the least, 0.256 * 2^-21.4 + 0.3 *
2^-23 + 2 * 2^-24 of 0.699, below 2^-21.  2^-20 of the score is allowed for."""
import numpy as np
import pytest
import torch

from paper_2603_22370_b200 import faar, inputs
from tests.gpu_helpers import DEV, dev_bf16, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.5, 1.0, 32.0])
def test_the_score_of_a_single_token(cap, D):
    from paper_2603_22370_b200 import build
    build.build()
    ctx = faar.Context(0)
    rng = np.random.default_rng(int(cap * 2) + D)
    n = 20000
    t = np.concatenate([rng.uniform(-1, 1, n // 2), rng.uniform(-4, 4, n // 4), np.exp(rng.uniform(-60, 6, n // 4 - 2)), [0.0, 0.8660254]])
    t[::3] *= -1.0
    first = inputs.to_bf16_f32(rng.uniform(1, 2, n))
    q, k = np.zeros((n, D), np.float32), np.zeros((n, D), np.float32)
    q[:, 3], k[:, 3] = inputs.to_bf16_f32(t * cap / first), first
    Q, K = dev_bf16(q), dev_bf16(k)
    out, lse = torch.empty_like(Q), torch.empty((n, 1, 1), device=DEV)
    faar.attention_scored_fwd(ctx, n, 1, 1, 1, D, Q, D, K, K, D, faar.make_attention_scores(1.0, cap), out, D, lse)
    torch.cuda.synchronize()
    faar.attention_status(ctx)
    t = q[:, 3].astype(np.float64) * k[:, 3] / cap
    want = cap * np.tanh(t) * np.log2(np.e)
    near = np.abs(t) <= 0.866
    assert near.sum() > n / 2 and (~near).sum() > n / 8
    off = np.abs(host(lse).reshape(n) - want)
    assert np.all(off <= 2.0 ** -20 * np.abs(want)), (off[want != 0] / np.abs(want[want != 0])).max()
    assert torch.equal(out, K)
    ctx.close()
