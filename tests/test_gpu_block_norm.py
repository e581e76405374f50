"""The residual sum with the norms around it against the formula in 64 bits."""
import sys

import pytest
import torch

from gpu_util import dev, say
from paper_2609_27233_amd import lib as sm

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
# A row's sum: at most 16 chunks of 8 features added one after another in a thread, then 6 steps over a wave and 16
# waves: each term passes under 160 additions
SUM = 160 * U


def _rand(shape, dt, seed, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dt).to(dev())


def _norm(x, dx, n, eps):
    """(norm of x in 64 bits, what it may be off by) for x known to within dx."""
    kind, gain, bias = n
    eps = float(torch.tensor(eps))
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    # the mean: its sum's roundings, and the terms' own errors
    d_mean = (SUM * x.abs().mean(-1, keepdim=True) + dx.mean(-1, keepdim=True)) if kind == "layer" else 0.0
    c, dc = x - mean, dx + d_mean + U * (x.abs() + mean.abs())
    r = (c.square().mean(-1, keepdim=True) + eps).sqrt()
    # r: half the sum's relative error, the centred terms' errors (|d r| <= rms(dc)), and the divide, root and square
    dr = (SUM / 2 + 4 * U) * r + dc.square().mean(-1, keepdim=True).sqrt()
    g = torch.ones_like(x[0]) if gain is None else gain.double().cpu()
    b = torch.zeros_like(x[0]) if bias is None else bias.double().cpu()
    y = c / r * g
    # (first order in dr / r, which the cases keep below 1/10: doubled)
    dy = (dc / r * g.abs() + 2 * y.abs() * dr / r + 4 * U * y.abs())
    return y + b, dy + U * (y + b).abs()


def reference(h, y, post, gate, scale, pre, eps=1e-5):
    """h_out and n_out in 64 bits, each with what fp32 arithmetic may move it by."""
    d64 = lambda t: t.double().cpu()                                  # noqa: E731
    x, dx = d64(h), torch.zeros_like(d64(h))
    if y is not None:
        t, dt = d64(y), torch.zeros_like(x)
        if post is not None:
            t, dt = _norm(t, dt, post, eps)
        if gate is not None:
            t, dt = t * d64(gate), (dt + U * t.abs()) * d64(gate).abs()
        s = float(torch.tensor(scale, dtype=F32))
        x, dx = x + s * t, abs(s) * (dt + U * t.abs()) + U * (x.abs() + (s * t).abs() * 2)
    return (x, dx), (None if pre is None else _norm(x, dx, pre, eps))


def assert_near(got, ref, dt):
    val, slack = ref
    got = got.double().cpu()
    tol = slack + torch.finfo(dt).eps / 2 * (val.abs() + slack)          # rounding to the type: half a step
    over = (got - val).abs() - tol
    assert not got.isnan().any() and float(over.max()) <= 0, (float(over.max()), int((over > 0).sum()))


def _make(kind, d, dt, seed, gain=True, bias=None):
    if kind is None:
        return None, None
    g = _rand((d,), dt, seed, 0.2, 1.0) if gain else None
    b = _rand((d,), dt, seed + 1, 0.2) if (kind == "layer" if bias is None else bias) else None
    return sm.norm_params(kind, g, b, eps=1e-5), (kind, g, b)


WIDTHS = [1, 2, 7, 64, 65, 250, 256, 504, 1000, 1024, 1032, 2048, 2056, 3584, 4096, 4097, 5120, 8192, 8200, 16383, 16384]
FORMS = [(None, None, "rms"), ("rms", "channel", "rms"), ("layer", "row", "layer"), ("layer", None, "rms"),
         (None, "row", "layer")]


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("d", WIDTHS)
def test_block_norm_matches_formula(dt, d):
    for k, (post, gate, pre) in enumerate(FORMS):
        for rows in (1, 2, 5, 33):
            h, y = _rand((rows, d), dt, d + k, 2.0, 0.5), _rand((rows, d), dt, d + k + 7, 1.0, -0.3)
            g = None if gate is None else _rand((d,) if gate == "channel" else (rows, d), dt, k, 0.5)
            p, p_ref = _make(post, d, dt, 50 + k)
            q, q_ref = _make(pre, d, dt, 60 + k)
            ho, no = (torch.full_like(h, float("nan")) for _ in range(2))
            say("block_norm", dt, "d", d, "rows", rows, post, gate, pre)
            sm.block_norm(h, y, ho, no, post=p, gate=g, scale=0.75, pre=q)
            r = reference(h, y, p_ref, g, 0.75, q_ref)
            if d == 1 and "layer" in (post, pre):                        # (a row of one feature: nothing but its rounding is left)
                assert no.isfinite().all()
                continue
            assert_near(ho, r[0], dt)
            assert_near(no, r[1], dt)


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("d", [64, 1111, 4096])
def test_parts_left_out(dt, d):
    rows = 9
    h, y = _rand((rows, d), dt, 1), _rand((rows, d), dt, 2)
    n, n_ref = _make("rms", d, dt, 3, gain=False)                       # a gain folded into the next weight
    b, b_ref = _make("rms", d, dt, 4, bias=True)
    ho, no = torch.empty_like(h), torch.empty_like(h)
    say("parts", dt, d)
    sm.block_norm(h, None, None, no, pre=n)                             # the first block's norm
    assert_near(no, reference(h, None, None, None, 1.0, n_ref)[1], dt)
    sm.block_norm(h, None, ho, no, pre=b)
    assert torch.equal(ho, h)
    assert_near(no, reference(h, None, None, None, 1.0, b_ref)[1], dt)
    sm.block_norm(h, y, ho, None, post=b, scale=-2.0)                   # the last block's sum
    assert_near(ho, reference(h, y, b_ref, None, -2.0, None)[0], dt)
    sm.block_norm(h, y, None, no, scale=0.0, pre=n)
    assert_near(no, reference(h, y, None, None, 0.0, n_ref)[1], dt)


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("shift", [0, 8, 1])
def test_strides_and_in_place(dt, shift):
    """Rows inside wider buffers, both outputs in place; nothing beside them is touched."""
    rows, d = 13, 520
    hb, yb, gb = (_rand((rows, 560), dt, i) for i in range(3))
    h, y, g = (t[:, 16 + shift:16 + shift + d] for t in (hb, yb, gb))
    b4 = hb.clone(), yb.clone()
    p, p_ref = _make("layer", d, dt, 5)
    q, q_ref = _make("rms", d, dt, 6)
    r = reference(h, y, p_ref, g, 1.5, q_ref)
    say("in place", dt, shift)
    sm.block_norm(h, y, h, y, post=p, gate=g, scale=1.5, pre=q)
    assert_near(h, r[0], dt)
    assert_near(y, r[1], dt)
    keep = torch.ones(560, dtype=torch.bool)
    keep[16 + shift:16 + shift + d] = False
    assert torch.equal(hb[:, keep], b4[0][:, keep]) and torch.equal(yb[:, keep], b4[1][:, keep])


def test_far_from_zero_and_large_values():
    """Statistics of a row far from zero (LayerNorm's differences are taken before they are squared) and of large rows."""
    x = _rand((4, 4096), F32, 1, 1.0, 1000.0)
    n, ref = _make("layer", 4096, F32, 2)
    out = torch.empty_like(x)
    sm.block_norm(x, None, None, out, pre=n)
    assert_near(out, reference(x, None, None, None, 1.0, ref)[1], F32)
    x = _rand((4, 4096), BF, 3, 1e15)
    n, ref = _make("rms", 4096, BF, 4)
    out = torch.empty_like(x)
    sm.block_norm(x, None, None, out, pre=n)
    assert_near(out, reference(x, None, None, None, 1.0, ref)[1], BF)


def test_zero_rows_and_special_values():
    d = 512
    h = torch.zeros((4, d), dtype=BF, device=dev())
    h[1, 5], h[2, 7], h[3] = float("nan"), float("inf"), 2.0
    n, _ = _make("rms", d, BF, 1, gain=False)
    m, _ = _make("layer", d, BF, 1, gain=False, bias=False)
    out = torch.empty_like(h)
    sm.block_norm(h, None, None, out, pre=n)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and out[1].isnan().all() and (out[3] == 1).all()
    assert out[2, 7].isnan() and (out[2, :7] == 0).all()                # the others: over an infinite norm
    sm.block_norm(h, None, None, out, pre=m)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and (out[3] == 0).all() and out[1].isnan().all()
    e = torch.empty((0, d), dtype=BF, device=dev())
    sm.block_norm(e, e, e, e, pre=n)


def test_mean_squares_below_the_normal_numbers():
    d = 4096
    sign = torch.randint(0, 2, (3, d), generator=torch.Generator().manual_seed(1)) * 2.0 - 1
    x = (4e-20 * sign).to(dev())                                         # squares of 1.6e-39
    n = torch.empty_like(x)
    sm.block_norm(x, None, None, n, pre=sm.norm_params("rms", eps=0.0))
    # a square's rounding to steps of 2^-149, the sum's, the mean's; halved by the root, then that and the product
    tol = (2.0 ** -150 / 1.6e-39 + SUM + 2 ** -150 / 1.6e-39) / 2 + 4 * U
    assert float((n.double().cpu() - sign).abs().max()) <= tol


def test_many_rows():
    """More rows than a 16-bit grid, each its own."""
    rows, d = 300001, 16
    h = torch.arange(rows, device=dev(), dtype=F32)[:, None].expand(rows, d).contiguous() + 1
    out = torch.empty_like(h)
    n, _ = _make("rms", d, F32, 1, gain=False)
    sm.block_norm(h, None, None, out, pre=n)
    assert float((out - 1).abs().max()) <= 1e-5                         # every row is its own mean square


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("d", [512, 16384])
def test_sums_past_the_largest_number(dt, d):
    """Rows whose squares come to more than 3.4e38 are normed to 0, plus a bias; a LayerNorm is NaN where the features'
    plain sum (or a difference from their mean) does too."""
    sign = torch.randint(0, 2, (d,), generator=torch.Generator().manual_seed(1)) * 2.0 - 1
    sign[1::2] = -sign[::2]                                              # (their sum is 0)
    h = torch.stack([sign * 1e35, torch.full((d,), 3e38), torch.full((d,), 1e30)]).to(dt).to(dev())
    bias = _rand((d,), dt, 3)
    for b in (None, bias):
        want = torch.zeros_like(h[0]) if b is None else bias
        rms, layer = torch.full_like(h, 7.0), torch.full_like(h, 7.0)
        sm.block_norm(h, None, None, rms, pre=sm.norm_params("rms", None, b))
        sm.block_norm(h, None, None, layer, pre=sm.norm_params("layer", None, b))
        torch.cuda.synchronize()
        assert all(torch.equal(r, want) for r in rms)
        assert torch.equal(layer[0], want)
        assert layer[1].isnan().all()                                    # (512 x 3e38 is past the largest number)
        assert torch.equal(layer[2], want)                               # equal features: no difference, as the formula has it


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
@pytest.mark.parametrize("d", [64, 1111, 4096, 5120, 16384])
def test_sums_to_their_counted_roundings(monkeypatch, dt, d):
    """The same reference with the additions that a feature passes: 16 features of a thread, 6 steps over a wave, 16 waves,
    and its square or the mean's product."""
    monkeypatch.setattr(sys.modules[__name__], "SUM", (16 + 6 + 16 + 2) * U)
    for k, (post, gate, pre) in enumerate(FORMS):
        h, y = _rand((9, d), dt, 3 * d + k, 2.0, 0.5), _rand((9, d), dt, d + k + 5, 1.0, -0.3)
        g = None if gate is None else _rand((d,) if gate == "channel" else (9, d), dt, k, 0.5)
        p, p_ref = _make(post, d, dt, 70 + k)
        q, q_ref = _make(pre, d, dt, 80 + k)
        ho, no = (torch.full_like(h, float("nan")) for _ in range(2))
        say("counted", dt, "d", d, post, gate, pre)
        sm.block_norm(h, y, ho, no, post=p, gate=g, scale=0.75, pre=q)
        r = reference(h, y, p_ref, g, 0.75, q_ref)
        assert_near(ho, r[0], dt)
        assert_near(no, r[1], dt)
