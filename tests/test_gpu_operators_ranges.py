"""GPU parity of the group, rotary, cache and attention calls at the ends of their ranges, and on every kernel that a call may take,
against the plain 64-bit forms and bounds of operators_util."""
import numpy as np
import pytest

import operators_util as ou
from parity_util import dev, host
from test_gpu_operators import rng, rows, run_product, weights

pytestmark = pytest.mark.gpu


# ---- products --------------------------------------------------------------------------------------


@pytest.mark.parametrize("T,K,N,group", [(1, 256, 40, 32), (32, 512, 200, 128),           # a few tokens
                                         (64, 256, 8300, 32), (40, 512, 16500, 128),      # tiles of 64 x 128, K in two halves
                                         (300, 256, 8200, 64), (260, 512, 8200, 256),     # 128 x 128
                                         (100, 320, 8300, 32), (65, 192, 16400, 64),      # 128 x 256
                                         (3300, 192, 3900, 64)])                          # 256 x 256
def test_product_of_large_steps(T, K, N, group):
    """Steps up to the largest fp16, whose codes times the step are none, beside ordinary ones: a token's result does not depend on how
    many others there are.  Half the tokens are zero where the steps are large, so that what the ordinary ones give counts."""
    print(f"case product large steps {T} {K} {N} {group}", flush=True)
    g = rng(30, T, K, N, group)
    codes, steps = weights(g, N, K, group)
    large = g.random(steps.shape) < 0.3
    large[g.random(N) < 0.5] = False                        # half the channels have ordinary steps only
    steps[large] = g.choice([8184.0, 8192.0, -8192.0, 9000.0, 30000.0, -65504.0, 65504.0], int(large.sum())).astype(np.float16)
    X = (g.standard_normal((T, K)) * 2.0 ** -8).astype(np.float16)
    some = large.any(0)                                     # groups with a large step in any channel
    X.reshape(T, K // group, group)[1::2, some] = 0
    # the bound adds 16 |x| |step| over the channels; ou.product takes steps above 0, so the signs go to the codes: the same numbers
    want, bound = ou.product(X, codes * np.sign(steps).astype(int).repeat(group, 1), np.abs(steps), group, T > 32)
    if T > 32:
        # such a channel's codes * step / 8 are rounded to fp16 (below its normal range by 2^-25, so 2^-22) in place of codes * step
        beyond = (np.abs(steps.astype(np.float64)) >= 8192).any(1)
        bound = bound + (1 + ou.HALF) * (2.0 ** -22 - ou.TINY) * np.abs(X.astype(np.float64)).sum(1, keepdims=True) * beyond
    inside = np.abs(want) + bound < 65504.0
    assert inside.mean() > 0.9
    got = run_product(X, codes, steps, 8 * (T % 3), T % 2)
    ou.held(np.where(inside, got, 0), np.where(inside, want, 0), bound, f"{T} {K} {N} {group}")


def test_product_of_steps_that_are_not_finite():
    """A channel with an infinite step is not finite, and the others are what they are without it."""
    print("case product infinite steps", flush=True)
    for T, N in ((16, 100), (64, 8300)):
        g = rng(31, T)
        X = rows(g, T, 256)
        codes, steps = weights(g, N, 256, 64)
        want, bound = ou.product(X, codes, steps, 64, T > 32)
        steps[7, 1], steps[70, 3] = np.inf, np.nan
        got = run_product(X, codes, steps)
        there = np.isin(np.arange(N), (7, 70))
        assert not np.isfinite(got[:, there]).any()
        ou.held(got[:, ~there], want[:, ~there], bound[:, ~there], f"{T} {N}")
