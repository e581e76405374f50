"""Tokens drawn from the largest vocabularies that a row may have, against the
definition in 64 bits: as many pieces as there are bins, masses of up to 2^63."""
import numpy as np
import pytest
import torch

from gpu_util import dev, say
from test_gpu_sample import BF, F32, INF, check, logits, settings

pytestmark = pytest.mark.gpu

MOST = 1 << 19


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V", [MOST - 1, MOST])
def test_settings(V, dt):
    rng = np.random.RandomState(V % 1000)
    say("largest", dt, V)
    check(logits(V, 9, dt, V), rng.uniform(size=9), *settings(rng, 9))


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V", [MOST - 1, MOST])
def test_equal_logits_at_the_ends(V, dt):
    """A mass of V: the first token at u = 0, the last that is kept at the largest u."""
    say("equal", dt, V)
    x = torch.full((4, V), -2.5, device=dev()).to(dt)
    u = [0.0, 1 - 2.0 ** -24, 0.5, 2.0 ** -24]
    tokens = check(x, u)
    assert tokens[0] == 0 and tokens[1] == V - 1
    p = np.float32(0.75)
    tokens = check(x, u, p=np.full(4, p))                        # ends among equal logits: a list does not suffice
    assert tokens[0] == 0 and tokens[1] == int(np.ceil(float(p) * V)) - 1
    check(x, u, k=[V, V - 1, MOST // 2, 5000], p=[1.0, 0.9, 1 - 2.0 ** -24, 0.5])


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
def test_many_weights_below_the_least_that_counts(dt):
    """One token and 524,287 at 2^-45 or a little less of it: shares off by the header's bound and no more."""
    at = float(torch.tensor(-45.0 * np.log(2.0)).to(dt))
    x = torch.full((3, MOST), at, device=dev()).to(dt)
    x[1] = at * (1 + 2.0 ** -6)
    x[2] = -INF
    x[2, ::2] = at
    x[:, 77777] = 0.0
    say("least weights", dt, at)
    check(x, [0.5, 1 - 2.0 ** -24, 2.0 ** -24])
