"""Token log probabilities, entropy and top alternatives against 64 bits."""
import math

import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def _rand(shape, dt, seed, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device=dev()).normal_(0, std, generator=g).to(dt)


def call(x, tokens, k, scale=1.0, want=True, ws=None, err=None, stream=None):
    rows, V = x.shape
    f = lambda *s: torch.full(s, -123.0, device=dev())                # noqa: E731
    lp, h = (f(rows), f(rows)) if want else (None, None)
    ids = torch.full((rows, k), -9, dtype=torch.int32, device=dev())
    tlp = f(rows, k)
    ws = torch.zeros(sm.token_logprobs_workspace_bytes(rows, V, k), dtype=torch.uint8, device=dev()) if ws is None else ws
    sm.token_logprobs(x, tokens, lp, h, ids, tlp, ws, scale=scale, err=err, stream=stream)
    return lp, h, ids, tlp


def reference(x, scale):
    """z - lse and entropy in 64 bits, and the order: the larger first, the lower index among equals, NaN last."""
    z = x.double() * float(torch.tensor(scale, dtype=F32))
    m = z.amax(1, keepdim=True).clamp(min=-1e300)
    e = torch.exp(z - m)
    S = e.sum(1, keepdim=True)
    logp = z - m - S.log()
    p = e / S
    H = -(p * torch.where(p > 0, logp, 0.0)).sum(1)
    order = torch.sort(torch.nan_to_num(x.float(), nan=-math.inf, posinf=math.inf, neginf=-3.4028235e38), dim=1,
                       descending=True, stable=True).indices if x.isnan().any() else \
        torch.sort(x.float(), dim=1, descending=True, stable=True).indices
    return logp, H, order


def assert_matches(x, tokens, k, scale, got):
    lp, H, ids, tlp = got
    V = x.shape[1]
    logp, Hr, order = reference(x, scale)
    torch.cuda.synchronize()
    assert torch.equal(ids.long(), order[:, :k])
    # S: fp32 additions one after another over a thread's share of the row, at least 64 threads to it, then the joins;
    # exponent and exponential 4 units of a term each.  A log probability moves by S's relative error and its own
    # roundings (scaled difference, logarithm, sum: 4 of each value).
    err_s = (V / 64 + 64) * U
    tol = lambda v: err_s + 6 * U * (v.abs() + 20)                     # noqa: E731
    tok = tokens.long().clamp(min=0)[:, None]
    ref = torch.where(tokens >= 0, logp.gather(1, tok)[:, 0], 0.0)
    fin = ref.isfinite()
    assert torch.equal(lp.double()[~fin], ref[~fin])
    assert ((lp.double() - ref).abs() <= tol(ref))[fin].all(), float((lp.double() - ref).abs()[fin].max())
    top = logp.gather(1, order[:, :k])
    fin = top.isfinite()
    assert torch.equal(tlp.double()[~fin], top[~fin])
    assert ((tlp.double() - top).abs() <= tol(top))[fin].all()
    # the entropy's sum is of terms of one sign, each at most exp(-1) times the largest e of a nat count below log V
    assert ((H.double() - Hr).abs() <= 3 * err_s * (1 + math.log(V)) + 20 * U).all(), float((H.double() - Hr).abs().max())


SIZES = [(1, 1), (1, 2), (3, 7), (2, 64), (5, 65), (1, 255), (4, 1000), (2, 4096), (3, 4097), (1, 32000), (7, 50257),
         (16, 128256), (1, 152064), (300, 1111), (2, 262144), (1200, 513)]


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_logprobs_match(dt, size):
    rows, V = size
    for k in sorted({0, 1, min(5, V), min(64, V)}):
        x = _rand((rows, V), dt, rows + V + k)
        tokens = torch.randint(-1, V, (rows,), generator=torch.Generator().manual_seed(k)).int().to(dev())
        scale = (1.0, 0.37, 2.5)[k % 3]
        say("logprobs", dt, size, "k", k, "scale", scale)
        assert_matches(x, tokens, k, scale, call(x, tokens, k, scale))


@pytest.mark.parametrize("dt,rows,V", [(BF, 1536, 33333), (F32, 1600, 20001), (BF, 4096, 70003), (F32, 4097, 33001),
                                       (BF, 511, 128256)], ids=str)
def test_many_long_rows(dt, rows, V):
    x = _rand((rows, V), dt, rows)
    x[5, 7:] = -math.inf
    tokens = torch.arange(rows, dtype=torch.int32, device=dev()) % V
    say("logprobs", dt, rows, V)
    got = call(x, tokens, 20)
    values, _ = torch.topk(x[6:].float(), 20, dim=1)
    assert torch.equal(x[6:].float().gather(1, got[2][6:].long()), values)
    some = torch.tensor([0, 1, 5, 6, rows // 2, rows - 2, rows - 1], device=dev())
    assert_matches(x[some], tokens[some], 20, 1.0, [t[some] for t in got])


def _orders(V):
    g = torch.Generator(device="cuda").manual_seed(V)
    up = torch.arange(V, device=dev(), dtype=F32) / V * 8
    few = torch.randint(0, 3, (V,), device=dev(), generator=g).float()
    return {"ascending": up, "descending": up.flip(0), "equal": torch.zeros(V, device=dev()), "few values": few,
            "equal but the last": torch.cat([torch.zeros(V - 1, device=dev()), torch.ones(1, device=dev())]),
            "zeros of both signs": torch.where(few > 0, 0.0, -0.0),
            "one far above": torch.where(torch.arange(V, device=dev()) == V // 2, 300.0, 0.0),
            "negative": -up - 5, "waves": torch.sin(torch.arange(V, device=dev()) * 0.01) * 5}


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("rows", [1, 600])
@pytest.mark.parametrize("V", [300, 33333])
def test_orders_and_ties(dt, rows, V):
    for name, row in _orders(V).items():
        x = row.to(dt).expand(rows, V).contiguous()
        tokens = torch.full((rows,), V - 1, dtype=torch.int32, device=dev())
        for k in (1, 20, 64):
            say("order", name, dt, rows, V, k)
            assert_matches(x, tokens, k, 1.0, call(x, tokens, k))


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V", [100, 20000])
def test_masked_rows(dt, V):
    x = _rand((6, V), dt, V)
    x[0, 10:] = -math.inf                                              # fewer left than alternatives asked for
    x[1, :] = -math.inf                                                # nothing left
    x[2, :] = torch.finfo(dt).min                                      # masked by the type's lowest value: all alike
    x[3, 1:] = torch.finfo(dt).min                                     # one left
    x[4, : V - 1] = -math.inf                                          # the last one left
    tokens = i32([3, 5, 7, 0, 0, V - 1])
    say("masked", dt, V)
    lp, h, ids, tlp = call(x, tokens, 20)
    keep = torch.tensor([0, 2, 3, 4, 5], device=dev())
    assert_matches(x[keep], tokens[keep], 20, 1.0, tuple(t[keep] for t in (lp, h, ids, tlp)))
    torch.cuda.synchronize()
    assert lp[1] == -math.inf and h[1] == 0 and (tlp[1] == -math.inf).all() and ids[1].tolist() == list(range(20))
    assert abs(float(lp[2]) + math.log(V)) <= 1e-4 and lp[3] == 0 and h[3] == 0 and lp[4] == -math.inf and h[4] == 0
    assert ids[0].tolist()[10:] == list(range(10, 20)) and (tlp[0, 10:] == -math.inf).all()


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("V", [64, 30000])
def test_nan_and_infinity(dt, V):
    x = _rand((4, V), dt, 3)
    x[0, 17], x[1, V - 1], x[2, 3], x[2, 4] = math.nan, math.inf, math.inf, math.nan
    tokens = i32([1, 1, 4, 1])
    say("nan", dt, V)
    lp, h, ids, tlp = call(x, tokens, 8)
    torch.cuda.synchronize()
    assert lp[:3].isnan().all() and h[:3].isnan().all() and tlp[:3].isnan().all()
    _, _, order = reference(x, 1.0)
    assert torch.equal(ids.long(), order[:, :8]) and ids[1, 0] == V - 1 and ids[2, 0] == 3
    assert_matches(x[3:], tokens[3:], 8, 1.0, (lp[3:], h[3:], ids[3:], tlp[3:]))
    y = torch.full((1, V), math.nan, dtype=dt, device=dev())
    y[0, V // 2] = -math.inf
    _, _, ids, _ = call(y, i32([0]), 3)
    assert ids[0].tolist() == [V // 2, 0, 1]                           # NaN below everything, the lower index first


def test_large_values():
    x = _rand((3, 5000), F32, 1, 1e30)
    x[1] = _rand((5000,), F32, 2) + 1e5
    x[2, 0], x[2, 1] = 3.4e38, -3.4e38
    tokens = torch.argmax(x, 1).int()
    lp, h, ids, tlp = call(x, tokens, 4, 2.0)
    torch.cuda.synchronize()
    assert lp[0] == 0 and h[0] == 0 and lp[2] == 0 and h[2] == 0
    assert torch.equal(ids[:, 0], tokens)
    assert_matches(x[1:2], tokens[1:2], 4, 2.0, (lp[1:2], h[1:2], ids[1:2], tlp[1:2]))


def test_tokens_out_of_range_and_parts_left_out():
    x = _rand((5, 900), BF, 1)
    err = torch.zeros(1, dtype=torch.int32, device=dev())
    tokens = i32([3, 900, -2, -1, 899])
    lp, h, ids, tlp = call(x, tokens, 2, err=err)
    logp, _, _ = reference(x, 1.0)
    torch.cuda.synchronize()
    assert int(err) == sm.ERR_EINVAL and lp[1:4].tolist() == [0, 0, 0]
    assert abs(float(lp[0]) - float(logp[0, 3])) < 1e-4 and abs(float(lp[4]) - float(logp[4, 899])) < 1e-4
    err.zero_()
    call(x, i32([0, -1, 899, -1, 2]), 2, err=err)
    call(x, tokens, 2)                                                  # no error word: nothing to report to
    torch.cuda.synchronize()
    assert int(err) == 0
    ws = torch.zeros(sm.token_logprobs_workspace_bytes(5, 900, 3), dtype=torch.uint8, device=dev())
    only = torch.empty((5, 3), dtype=torch.int32, device=dev())
    sm.token_logprobs(x, None, None, None, only, None, ws)
    assert torch.equal(only, call(x, i32([0] * 5), 3)[2])
    ent = torch.empty(5, device=dev())
    sm.token_logprobs(x, None, None, ent, None, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(ent, h)
    e = torch.empty((0, 900), dtype=BF, device=dev())
    sm.token_logprobs(e, i32([]), torch.empty(0, device=dev()), None, None, None, ws)


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("V", [777, 40000])
def test_strides_and_alignment(dt, shift, V):
    buf = _rand((5, V + 40), dt, shift)
    x = buf[:, shift:shift + V]
    tokens = i32([0, V - 1, 5, -1, 9])
    say("strides", dt, shift, V)
    got = call(x, tokens, 7)
    assert_matches(x, tokens, 7, 1.0, got)
    again = call(x.contiguous(), tokens, 7)
    assert torch.equal(got[2], again[2])


def test_same_inputs_same_bits_and_shared_workspace():
    """One workspace for calls of any shape, one after another; the same bits every time."""
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device=dev())
    cases = [(1, 128256, 8), (16, 50000, 64), (700, 3000, 4), (2, 100, 1), (1, 262144, 20)]
    xs = [_rand((r, V), BF, r) for r, V, _ in cases]
    first = None
    for rep in range(3):
        outs = [call(x, torch.zeros(x.shape[0], dtype=torch.int32, device=dev()), k, ws=ws) for x, (_, _, k) in zip(xs, cases)]
        torch.cuda.synchronize()
        assert (ws[:65536] == 0).all()
        flat = [t.clone() for o in outs for t in o]
        first = first or flat
        assert all(torch.equal(a, b) for a, b in zip(first, flat))


def test_captured_and_replayed():
    x = _rand((4, 30000), BF, 1)
    tokens = i32([1, 2, 3, 4])
    ws = torch.zeros(sm.token_logprobs_workspace_bytes(4, 30000, 5), dtype=torch.uint8, device=dev())
    outs = (torch.empty(4, device=dev()), torch.empty(4, device=dev()),
            torch.empty((4, 5), dtype=torch.int32, device=dev()), torch.empty((4, 5), device=dev()))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        sm.token_logprobs(x, tokens, *outs, ws, scale=0.5)
    for rep in range(4):
        x.copy_(_rand((4, 30000), BF, 10 + rep))
        g.replay()
        torch.cuda.synchronize()
        assert_matches(x, tokens, 5, 0.5, outs)
        eager = call(x, tokens, 5, 0.5)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


NANS = {BF: (0x7fc0, -0x40), F32: (0x7fc00000, -0x400000)}  # quiet, of both signs


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("rows,V", [(4, 4000), (3, 648), (4097, 9008)])
@pytest.mark.parametrize("k", [8, 33, 64])
def test_whole_vectors_of_nan(dt, rows, V, k):
    """16-byte vectors of nothing but NaN, one to all of a row's first ones: every number comes before them."""
    n = 16 // dt.itemsize
    for several, bits in enumerate(NANS[dt]):
        x = _rand((rows, V), dt, V + k, 0.01)
        raw = x.view(torch.int16 if dt == BF else torch.int32)
        peak = torch.arange(63, device=dev())
        x[0, peak * n + 3 + n * (peak >= 5)] += 20.0                    # 63 vectors with a peak each, the sixth one of NaN
        raw[0, 5 * n:6 * n] = bits
        raw[1, :7 * n] = bits
        raw[2, :(k + 2) * n] = bits                                     # more such vectors than alternatives
        raw[2, V - 1] = bits
        raw[rows - 1, 1::n] = bits                                      # one NaN in every vector
        tokens = torch.zeros(rows, dtype=torch.int32, device=dev())
        say("nan vectors", dt, rows, V, "k", k, hex(bits & 0xffffffff))
        lp, h, ids, tlp = call(x, tokens, k)
        some = torch.tensor([0, 1, 2, rows - 1], device=dev())
        _, _, order = reference(x[some], 1.0)
        assert torch.equal(ids[some].long(), order[:, :k]), (several, [int((a != b).sum()) for a, b in zip(ids[some], order[:, :k])])
        assert lp[some].isnan().all() and h[some].isnan().all() and tlp[some].isnan().all()
        if rows > 4:
            assert torch.equal(ids[3].long(), reference(x[3:4], 1.0)[2][0, :k]) and not lp[3:-1].isnan().any()


SIGNALING = {BF: (0x7f81, -0x7f), F32: (0x7f800001, -0x7fffff)}


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("rows,V", [(9, 648), (9, 40000), (600, 20000), (4097, 9008)])
@pytest.mark.parametrize("k", [1, 8, 64])
def test_signaling_nan(dt, rows, V, k):
    """A signaling NaN hides no number of its 16 bytes, wherever it stands in them."""
    n = 16 // dt.itemsize
    for bits in SIGNALING[dt]:
        x = _rand((rows, V), dt, V + k)
        raw = x.view(torch.int16 if dt == BF else torch.int32)
        for at in range(n):
            raw[at, at::n] = bits                                       # one in every vector
        raw[8, -3 * n + 1] = bits
        tokens = torch.zeros(rows, dtype=torch.int32, device=dev())
        say("signaling", dt, rows, V, "k", k, hex(bits & 0xffffffff))
        lp, h, ids, tlp = call(x, tokens, k)
        some = torch.tensor([*range(n), 8], device=dev())
        _, _, order = reference(x[some], 1.0)
        assert torch.equal(ids[some].long(), order[:, :k])
        assert lp[some].isnan().all() and h[some].isnan().all() and tlp[some].isnan().all()


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("rows,V", [(3, 262144), (600, 262144), (4096, 65536)])
def test_sums_to_their_counted_roundings(dt, rows, V):
    """Log probabilities and entropy of long rows, by the additions that a term of the sums passes."""
    n = 16 // dt.itemsize
    x = _rand((rows, V), dt, V, 2.5)
    x[1] = -0.5                                                         # sums of equal terms that are no power of two
    x[1, 0] = 0.0
    tokens = torch.arange(rows, dtype=torch.int32, device=dev()) * 7 % V
    say("counted", dt, rows, V)
    got = call(x, tokens, 4)
    some = torch.tensor([0, 1, 2, rows - 1], device=dev())
    z = x[some].double()
    d = (z - z.amax(1, keepdim=True)).abs()
    logp, H, order = reference(x[some], 1.0)
    p = logp.exp()
    # M and Q: the mean of |z - r| and its square under p; the reference r is within 3 of the maximum
    M, Q = (p * d).sum(1) + 3, (p * (d + 3).square()).sum(1)
    # A term passes a chunk's 4 vectors, at most V / (256 n) chunks and four joins of 6 steps.  The references that were
    # left (a factor each, with an exponential of their difference) lie in a range of 15, at least 2.7 apart: 3 of each and
    # 3 for every unit of the range, 60.  Its own exponent (difference, scale, product) is off by 3 |z - r|, the exponential by 2.
    depth = 4 * n + V / (256 * n) + 24 + 60
    err_s = (depth + 3 * M + 2) * U
    # the logarithm is off by a unit of itself and of the factor behind it, the difference, product and sum by one each
    def tol_lp(v):
        return err_s[:, None] + 6 * U * (v.abs() + math.log(V) + 3)
    lp, h, ids, tlp = (t[some] for t in got)
    assert torch.equal(ids.long(), order[:, :4])
    ref = logp.gather(1, tokens[some].long()[:, None])
    assert ((lp[:, None].double() - ref).abs() <= tol_lp(ref)).all()
    top = logp.gather(1, order[:, :4])
    assert ((tlp.double() - top).abs() <= tol_lp(top)).all()
    # E / S: the terms |p d| come to M, each off by what a term of S is and d's and the product's rounding
    tol = (M * (depth + 4) + 3 * Q) * U + (M + 1) * err_s + 6 * U * (math.log(V) + M)
    assert ((h.double() - H).abs() <= tol).all(), ((h.double() - H).abs() / tol).tolist()


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("rows,V", [(3, 900), (3, 40000), (2000, 9000)])
@pytest.mark.parametrize("scale", [1e-20, 1e-3, 0.4])
def test_differences_past_the_largest_number(dt, rows, V, scale):
    """Logits more than 3.4e38 apart: the scale brings their log probabilities back."""
    x = torch.linspace(-3.3e38, 3.3e38, V, dtype=torch.float64, device=dev()).to(dt).expand(rows, V).contiguous()
    x[1] = x[1].flip(0)
    x[2, 5] = -math.inf
    tokens = torch.arange(rows, dtype=torch.int32, device=dev()) % V
    tokens[2] = 5
    say("far apart", dt, rows, V, scale)
    lp, h, ids, tlp = call(x, tokens, 8, scale)
    some = torch.tensor([0, 1, 2, rows - 1], device=dev())
    logp, H, order = reference(x[some], scale)
    assert torch.equal(ids[some].long(), order[:, :8])
    ref = logp.gather(1, tokens[some].long()[:, None])[:, 0]
    top = logp.gather(1, order[:, :8])
    assert lp[2] == -math.inf and torch.equal(ref.isfinite(), some != 2)
    # a product with the scale and its rounding or a difference and its product, a sum: 4 units, of terms up to twice the
    # value (one of 6.6e38 x scale of two of 3.3e38 x scale); beside them the logarithm counts for the near ones
    for got, want in ((lp[some], ref), (tlp[some], top)):
        fin = want.isfinite()
        assert got.isfinite().eq(fin).all()
        assert ((got.double() - want).abs() <= 8 * U * (want.abs() + 20))[fin].all()
    assert ((h[some].double() - H).abs() <= 1e-4).all()
