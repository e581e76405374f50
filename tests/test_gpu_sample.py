"""Tokens drawn from rows of logits against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")


def f32(a):
    return torch.as_tensor(np.asarray(a, np.float32)).to(dev())


def kept_and_mass(x, T, k, p, m):
    """(kept tokens in the order of the vocabulary, their weights) of one row x (fp64) by the definition."""
    V = len(x)
    order = np.argsort(-x, kind="stable")
    order = order[:1 if T == 0 else (V if k <= 0 else min(k, V))]
    z = (x[order] - x.max()) / (T or 1.0)
    # w >= m by logarithms: the exponential of -1e-30, which is below 1, rounds to 1
    keep = z >= (np.log(m) if m > 0 else -np.inf)
    order, w = order[keep], np.exp(z[keep])
    if p < 1 and T != 0:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        keep = before < p * w.sum()
        keep[0] = True
        order, w = order[keep], w[keep]
    at = np.argsort(order)
    return order[at], w[at]


def check_row(x, T, k, p, m, u, token, logprob):
    ids, w = kept_and_mass(x, T, k, p, m)
    cum = np.cumsum(w)
    # a weight is off by half of 2^-44 and by 2^-50 of itself, so a mass of n of them by n 2^-45 + 2^-50 of itself;
    # fp64's own sums here by about n 2^-53
    slack = len(w) * 2.0 ** -45 + 2.0 ** -40 * 1e-2 * cum[-1] + len(w) * 2.0 ** -53 * cum[-1]
    at = np.searchsorted(ids, token)
    assert at < len(ids) and ids[at] == token, ("not kept", token, len(ids))
    lo = cum[at] - w[at]
    assert lo - slack <= u * cum[-1] < cum[at] + slack, (token, lo, u * cum[-1], cum[at])
    # fp32's rounding of the logarithm, and the slack in the share
    ref = np.log(w[at] / cum[-1])
    assert abs(logprob - ref) <= 2.0 ** -23 * abs(ref) + 2.0 ** -30 + slack / max(w[at], 1e-300), (logprob, ref)


def sample(x, u, T=None, k=None, p=None, m=None, stream=None, ws=None):
    rows, V = x.shape
    tokens = torch.full((rows + 1,), -7, dtype=torch.int32, device=dev())
    logprob = torch.full((rows + 1,), 7.0, device=dev())
    err = torch.zeros(1, dtype=torch.int32, device=dev())
    ws = torch.zeros(sm.sample_workspace_bytes(rows, V), dtype=torch.uint8, device=dev()) if ws is None else ws
    sm.sample_tokens(x, f32(u), tokens, ws, temperature=None if T is None else f32(T), top_k=None if k is None else i32(k),
                     top_p=None if p is None else f32(p), min_p=None if m is None else f32(m), logprob=logprob, err=err)
    torch.cuda.synchronize()
    assert int(tokens[-1]) == -7 and float(logprob[-1]) == 7.0
    return tokens[:-1].cpu().numpy(), logprob[:-1].double().cpu().numpy(), int(err.item())


def check(x, u, T=None, k=None, p=None, m=None):
    rows, V = x.shape
    ws = torch.zeros(sm.sample_workspace_bytes(rows, V), dtype=torch.uint8, device=dev())
    tokens, logprobs, err = sample(x, u, T, k, p, m, ws=ws)
    assert err == 0
    # the workspace is ready for the next call, also after one of other sizes
    sample(torch.randn((1, 700), device=dev()), [0.5], [1.0], [30], [0.9], ws=ws)
    again = sample(x, u, T, k, p, m, ws=ws)
    assert np.array_equal(tokens, again[0]) and np.array_equal(logprobs, again[1])
    xd = x.double().cpu().numpy()
    one = lambda a, r, d: d if a is None else float(np.asarray(a, np.float32)[r])          # noqa: E731
    for r in range(rows):
        check_row(xd[r], one(T, r, 1.0), int(one(k, r, 0)), one(p, r, 1.0), one(m, r, 0.0), one(u, r, 0), int(tokens[r]),
                  logprobs[r])
    return tokens


def settings(rng, rows):
    """Every combination of the filters, tight and wide, and some greedy rows."""
    how = rng.randint(0, 8, rows)
    T = rng.choice([0.3, 0.7, 1.0, 1.5, 4.0], rows)
    T[rng.uniform(size=rows) < 0.1] = 0.0
    k = np.where(how & 1, rng.choice([1, 2, 7, 50, 1000], rows), 0)
    p = np.where(how & 2, rng.choice([0.0, 0.1, 0.5, 0.9, 0.99, 0.9999], rows), 1.0)
    m = np.where(how & 4, rng.choice([1e-6, 0.01, 0.1, 0.5, 1.0], rows), 0.0)
    return T, k, p, m


def logits(V, rows, dt, seed, std=2.5):
    g = torch.Generator().manual_seed(seed)
    x = std * torch.randn((rows, V), generator=g)
    x[:, torch.randint(V, (4,), generator=g)] += 9.0
    return x.to(dt).to(dev())


SIZES = [1, 2, 3, 7, 64, 511, 512, 513, 1000, 1025, 4097, 8192, 32000, 50257, 65536, 128256, 152064, 262144]


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V", SIZES)
def test_sizes_and_settings(V, dt):
    rows = 40 if V <= 50257 else 17
    rng = np.random.RandomState(V % 1000)
    say("sample", dt, rows, V)
    check(logits(V, rows, dt, V), rng.uniform(size=rows), *settings(rng, rows))


@pytest.mark.parametrize("rows", [1, 2, 16, 64, 257, 1000])
def test_numbers_of_rows(rows):
    rng = np.random.RandomState(rows)
    say("sample rows", rows)
    check(logits(3001, rows, BF, rows), rng.uniform(size=rows), *settings(rng, rows))


def test_no_filters_at_all_and_each_alone():
    x, rng = logits(20000, 12, BF, 5), np.random.RandomState(1)
    u = rng.uniform(size=12)
    check(x, u)
    check(x, u, T=np.full(12, 0.8))
    check(x, u, k=np.arange(12))
    check(x, u, p=np.linspace(0, 1.1, 12))
    check(x, u, m=np.linspace(0, 1, 12))


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
def test_ties_go_to_the_lower_index(dt):
    """Few distinct logits: whole pieces of equal ones, cut by each filter in the middle."""
    rng = np.random.RandomState(3)
    rows, V = 64, 5000
    x = torch.from_numpy(rng.randint(0, 3, (rows, V)).astype(np.float32)).to(dt).to(dev())
    x[5] = 1.5
    x[6, 1:] = -3.0
    x[7] = -0.0
    x[7, ::2] = 0.0                                              # equal to -0
    u = rng.uniform(size=rows)
    u[:8] = [0, 0.5, 1 - 2 ** -24, 0.1, 0.9, 0.3, 0.99, 0.75]
    tokens = check(x, u, k=rng.randint(0, 4000, rows))
    check(x, u, p=rng.uniform(size=rows), T=rng.choice([0.5, 1.0, 3.0], rows))
    check(x, u, *settings(rng, rows))
    greedy, _, _ = sample(x, u, T=np.zeros(rows))
    assert np.array_equal(greedy, x.float().cpu().numpy().argmax(1))
    assert int(tokens[0]) >= 0


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
def test_masked_vocabularies_and_far_logits(dt):
    rng = np.random.RandomState(4)
    rows, V = 30, 9000
    x = logits(V, rows, dt, 9)
    x[:10, torch.from_numpy(rng.permutation(V)[:8990])] = -INF   # ten tokens left
    x[10:15, 1:] = -INF                                          # one
    x[15:20] *= 30.0                                             # spread far past any weight that counts
    x[20] = -1e30
    x[20, 77], x[20, 99] = -3e4, -3e4
    x[21] = torch.finfo(dt).min
    x[21, 8999] = torch.finfo(dt).max
    x[22] *= 1e-30
    u = rng.uniform(size=rows)
    for _ in range(3):
        check(x, u, *settings(rng, rows))
    check(x, u, k=np.full(rows, 100), T=np.full(rows, 0.01))
    check(x, u, T=np.full(rows, 1e-30), p=np.full(rows, 0.7))
    check(x, u, T=np.full(rows, 3e38), p=np.full(rows, 0.7))
    check(x, u, k=np.full(rows, 2 ** 31 - 1), p=np.full(rows, 2.0))


def test_random_numbers_at_the_ends():
    x = torch.zeros((6, 1000), device=dev())
    x[:, :3] = -INF
    u = [0.0, 2.0 ** -149, 1 - 2.0 ** -24, 0.5, 1 / 3, 2.0 ** -24]
    tokens = check(x, u)
    assert tokens[0] == 3 and tokens[2] == 999 and tokens[3] == 3 + 498


def test_bad_rows_and_settings_alone_are_refused():
    x = logits(2000, 16, BF, 2)
    x[0, 5] = float("nan")
    x[1, 1999] = INF
    x[2] = -INF
    u, T, k, p, m = np.full(16, 0.4), np.ones(16), np.zeros(16, int), np.ones(16), np.zeros(16)
    u[3], u[4], u[5] = 1.0, -0.1, np.nan
    T[6], T[7], T[8] = -1.0, np.nan, np.inf
    k[9] = -1
    p[10], p[11] = -0.5, np.nan
    m[12], m[13] = 1.5, np.nan
    tokens, logprobs, err = sample(x, u, T, k, p, m)
    assert err == sm.ERR_EINVAL
    assert (tokens[:14] == -1).all() and np.isnan(logprobs[:14]).all()
    for r in (14, 15):
        check_row(x[r].double().cpu().numpy(), 1.0, 0, 1.0, 0.0, 0.4, int(tokens[r]), logprobs[r])
    # without an error word and log probabilities the call goes on the same way
    out = torch.empty(16, dtype=torch.int32, device=dev())
    ws = torch.zeros(sm.sample_workspace_bytes(16, 2000), dtype=torch.uint8, device=dev())
    sm.sample_tokens(x, f32(u), out, ws, temperature=f32(T), top_k=i32(k), top_p=f32(p), min_p=f32(m))
    assert np.array_equal(out.cpu().numpy(), tokens)


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_rows_with_a_stride_at_any_element(dt, shift):
    buf = logits(1301, 20, dt, 6)
    x, rng = buf[:, shift:shift + 1200], np.random.RandomState(6)
    u, s = rng.uniform(size=20), settings(rng, 20)
    tokens = check(x, u, *s)
    assert np.array_equal(tokens, check(x.contiguous(), u, *s))


def test_the_draws_follow_the_weights():
    """u on a grid: each token as often as its share, to one draw."""
    n, V = 4096, 300
    x = logits(V, 1, F32, 8)
    u = (np.arange(n) + 0.5) / n
    tokens, _, err = sample(x.expand(n, V).contiguous(), u, T=np.full(n, 0.9), p=np.full(n, 0.95))
    assert err == 0
    ids, w = kept_and_mass(x[0].double().cpu().numpy(), float(np.float32(0.9)), 0, float(np.float32(0.95)), 0.0)
    counts = np.bincount(tokens, minlength=V)
    assert set(np.nonzero(counts)[0]) <= set(ids)
    assert np.abs(counts[ids] - n * w / w.sum()).max() <= 1.0


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
def test_lists_that_do_not_suffice(dt):
    """A k of thousands and ends of the mass among thousands of near-equal logits: cut by passes over the row."""
    rng = np.random.RandomState(11)
    x = logits(128256, 8, dt, 12)
    x[4:6] *= 1e-3                                               # all in a bin or two
    x[6:] = torch.from_numpy(rng.choice([0.0, 0.5, 1.0], (2, 128256))).to(dt).to(dev())
    u = rng.uniform(size=8)
    check(x, u, k=[5000, 20000, 60000, 128255, 4097, 100000, 50000, 1])
    check(x, u, k=[5000, 20000, 60000, 128255, 4097, 100000, 50000, 9], p=np.full(8, 0.7), m=np.full(8, 1e-5))
    check(x, u, p=np.linspace(0.05, 0.9999, 8), T=[1.0, 0.3, 9.0, 1e-45, 1.0, 0.5, 1.0, 2.0])


def test_many_rows_each_with_its_own_settings():
    """More rows than the workspace holds at a time."""
    rng = np.random.RandomState(13)
    say("rows", 1500)
    check(logits(1030, 1500, BF, 14), rng.uniform(size=1500), *settings(rng, 1500))


def test_refused_rows_leave_the_workspace_as_any_do():
    rng = np.random.RandomState(15)
    x = logits(3000, 40, BF, 16)
    u, s = rng.uniform(size=40), settings(rng, 40)
    ws = torch.zeros(sm.sample_workspace_bytes(40, 3000), dtype=torch.uint8, device=dev())
    want = sample(x, u, *s, ws=ws)
    bad = x.clone()
    bad[::3, ::7] = float("nan")
    bad[1::3] = -INF
    for T in (s[0], np.full(40, -1.0)):
        assert sample(bad, u, T, *s[1:], ws=ws)[2] == sm.ERR_EINVAL
        got = sample(x, u, *s, ws=ws)
        assert got[2] == 0 and np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
