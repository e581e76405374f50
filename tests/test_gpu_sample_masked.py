"""Tokens drawn from rows whose first logits are masked and whose others lie far
below 0, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import dev, say
from paper_2609_27233_amd import lib as sm
from test_gpu_sample import BF, F32, INF, check, sample

pytestmark = pytest.mark.gpu


def behind_a_mask(V, dt, first, seed):
    """Rows whose first `first` logits are -infinity and whose others lie around each of several low values, or are all
    equal to it."""
    rng = np.random.RandomState(seed)
    low = torch.finfo(dt).min
    x = np.full((14, V), -np.inf, np.float32)
    for r, at in enumerate((-80.0, -120.0, -500.0, -3e4, -1e6)):
        x[r, first:] = at + 2 * rng.randn(V - first)
        x[5 + r, first:] = at
    x[10, first:] = low
    x[11, first:] = low
    x[11, first + 3] = low / 2
    x[12, first:] = -1e30
    x[13, V - 1] = low                                           # a single token
    return torch.from_numpy(x).to(dt).to(dev())


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V,first", [(600, 512), (9000, 512), (9000, 5000), (40000, 1024)])
def test_low_logits_behind_a_mask(V, first, dt):
    x = behind_a_mask(V, dt, first, V + first)
    n, rng = len(x), np.random.RandomState(V)
    u = rng.uniform(size=n)
    u[:3] = [0.0, 1 - 2.0 ** -24, 0.5]
    for T in (0.25, 1.0, 3.0, 1e30):
        say("masked", dt, V, first, "T", T)
        for p in (0.0, 2.0 ** -149, 1e-6, 0.5, 1 - 2.0 ** -24):
            check(x, u, T=np.full(n, T), p=np.full(n, p))
        for k in (1, 2, 50, V - first, V - 1):
            check(x, u, T=np.full(n, T), k=np.full(n, k))
            check(x, u, T=np.full(n, T), k=np.full(n, k), p=np.full(n, 0.0))
            check(x, u, T=np.full(n, T), k=np.full(n, k), p=np.full(n, 0.7), m=np.full(n, 1e-3))
        check(x, u, T=np.full(n, T), p=np.full(n, 0.0), m=np.full(n, 0.5))


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
def test_no_mass_is_kept_but_the_likeliest_token(dt):
    """top_p = 0 keeps one token wherever the mask ends and whatever the rest is."""
    x = behind_a_mask(4000, dt, 700, 3)
    n = len(x)
    for u in (0.0, 0.999):
        tokens, logprobs, err = sample(x, np.full(n, u), p=np.zeros(n))
        assert err == 0 and not logprobs.any()
        assert np.array_equal(tokens, x.float().cpu().numpy().argmax(1))
    x[:] = -INF
    assert sample(x, np.full(n, 0.5), p=np.zeros(n))[2] == sm.ERR_EINVAL


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V", [2000, 30000])
def test_a_wide_k_takes_logits_past_the_largest_depth(V, dt):
    """Finite logits so low that their depth below the others passes fp32's range weigh like any others at a temperature as
    high: a k that reaches into them keeps its first."""
    rng = np.random.RandomState(V)
    big = torch.finfo(dt).max
    x = np.full((6, V), -big, np.float32)
    near = [600, 40, 1500, 600, 600, 3]
    for r, n in enumerate(near):
        x[r, rng.permutation(V)[:n]] = rng.randn(n)
    x[3, 0] = 0.0                                                # the bins' origin, with and without a near logit
    x[4, :512] = -big
    x = torch.from_numpy(x).to(dt).to(dev())
    u = np.array([0.99, 0.5, 0.9, 0.999, 0.7, 0.8])
    say("wide k", dt, V)
    for T in (3e38, 1e38):
        tokens = check(x, u, T=np.full(6, T), k=[V - 1, 1500, 1600, V - 1, 1900, 10])
        assert (x[torch.arange(6), torch.from_numpy(tokens).long()] < -1e30).any()
        check(x, u, T=np.full(6, T), k=np.full(6, 1700), p=np.full(6, 0.9))
        check(x, u, T=np.full(6, T), p=np.linspace(0.1, 0.95, 6))
