"""Attention over 8-bit pages (one query a sequence, and a prompt's rows) against
the formula in 64 bits of the features that the pages stand for."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm
from test_gpu_e4m3_write import BF, E4, features, filled, slots_of, with_sequences
from test_gpu_rotary import _rand

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8  # half a step of bf16, relative


def attended(q, K, V, scale, seen=None):
    """(out [rows, Hq, D], what the roundings may move it by) of q over entries K, V [entries, H, D], all fp64.

    A probability is rounded to bf16 (2^-8 of itself) and so is the result (2^-8 of itself); the sums over at most 128 products
    and the exponentials are fp32: a score is off by 130 x 2^-24 of its products' sizes and 2 x 2^-24 of the distance that the
    exponent takes, the exponential itself by 2^-22, and a sum of n weights by the 2^-24 of up to n / 64 + 10 additions."""
    rows, Hq, D = q.shape
    n, G = K.shape[0], Hq // max(1, K.shape[1])
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    for h in range(Hq if n else 0):
        s = scale * (q[:, h] @ K[:, h // G].T)
        size = abs(scale) * (q[:, h].abs() @ K[:, h // G].abs().T)
        if seen is not None:
            s, size = torch.where(seen, s, -np.inf), torch.where(seen, size, 0.0)
        p = torch.softmax(s, 1)
        off = (2 * HALF + 2 * 134 * 2.0 ** -24 * size.amax(1, keepdim=True) + 2.0 ** -20 + (n / 32 + 20) * 2.0 ** -24)
        out[:, h] = p @ V[:, h // G]
        tol[:, h] = off * (p @ V[:, h // G].abs()) + HALF * out[:, h].abs()
    return out, tol


def assert_within(got, out, tol):
    got = got.double().cpu()
    over = (got - out).abs() - tol
    assert not got.isnan().any() and float(over.max()) <= 0, (float(over.max()), int((over > 0).sum()))


def poisoned(c, table, lens):
    """NaN in every byte that no entry holds, values and exponents."""
    k, v = c.k_pool.view(torch.uint8), c.v_pool.view(torch.uint8)
    free = torch.ones(c.num_blocks * c.bs, dtype=torch.bool)
    for s, L in enumerate(lens):
        free[slots_of(table, c.bs, s, np.arange(L))] = False
    free = free.view(c.num_blocks, c.bs).to(dev())
    k.masked_fill_(free[:, None, :, None], 0x7f)
    v.masked_fill_(free[:, None, None, :], 0x7f)
    c.k_exp.masked_fill_(free[:, None], 255)
    c.v_exp.masked_fill_(free[:, None], 255)


DECODES = [
    # Hq, Hkv, D, bs, lengths, listed sequences (None: each once), scale
    (32, 8, 128, 16, [300, 1, 0, 65], None, None),
    (16, 4, 64, 16, [307], None, None),
    (28, 4, 128, 64, [15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], [11, 0, 3, 3, 5, 7, 9, 1, 2, 10, 8, 6, 4], None),
    (4, 4, 64, 512, [1000, 513, 1], None, -0.3),                 # one head a group; a negative scale
    (16, 1, 128, 16, [20000], None, None),                       # many chunks, 16 heads a group
    (8, 2, 64, 32, [5000, 100, 0, 4097], [3, 0, 1, 2, 0], 0.0),  # scale 0: the mean
    (64, 8, 128, 16, [257 + 13 * i for i in range(70)], None, None),   # more pairs than compute units, in length order
    (4, 2, 64, 16, [1] * 300, None, None),
]


@pytest.mark.parametrize("case", range(len(DECODES)))
def test_decode_matches_formula(case):
    Hq, Hkv, D, bs, lens, ids, scale = DECODES[case]
    nb = sum(-(-x // bs) for x in lens) + 1
    c = filled(E4, Hkv, D, bs, nb, max_seqs=len(lens), max_blocks_per_seq=max(1, -(-max(lens) // bs)))
    table = with_sequences(c, lens, case)
    poisoned(c, table, lens)
    ids = list(np.random.RandomState(case).permutation(len(lens))) if ids is None else ids
    q = _rand((len(ids), Hq, D), BF, case)
    out = torch.full_like(q, float("nan"))
    max_len = max(lens)
    ws = torch.zeros(sm.decode_workspace_bytes(len(ids), Hq, D, max_len), dtype=torch.uint8, device=dev())
    say("e4m3 decode", case, Hq, Hkv, D, bs, "longest", max_len)
    for _ in range(2):                                           # the workspace is left ready for the next call
        out.fill_(float("nan"))
        sm.decode_attention(c, i32(ids), q, out, ws, max_len, scale=scale)
        torch.cuda.synchronize()
        assert c.error_bits() == 0
        K, V = features(c)
        for i, s in enumerate(ids):
            at = slots_of(table, bs, s, np.arange(lens[s]))
            assert_within(out[i:i + 1], *attended(q[i:i + 1].double().cpu(), K[at], V[at], D ** -0.5 if scale is None else scale))


def test_decode_errors_leave_zero_rows():
    c = filled(E4, 2, 64, 16, 40, max_seqs=5, max_blocks_per_seq=20)
    table = with_sequences(c, [40, 17, 300, 100, 30])
    K, V = features(c)
    q = _rand((5, 4, 64), BF, 1)
    ws = torch.zeros(sm.decode_workspace_bytes(5, 4, 64, 299), dtype=torch.uint8, device=dev())
    c.block_table[3, 2] = 40
    for ids, bits in (([0, 7, 1, 4, -1], sm.ERR_EINVAL), ([0, 2, 1, 4, 2], sm.ERR_ERANGE), ([0, 3, 1, 4, 3], sm.ERR_EINVAL)):
        out = torch.full_like(q, float("nan"))
        sm.decode_attention(c, i32(ids), q, out, ws, 299)
        torch.cuda.synchronize()
        assert c.error_bits() == bits
        c.clear_error()
        for i, s in enumerate(ids):
            if i in (1, 4):
                assert not out[i].any()
            else:
                at = slots_of(table, 16, s, np.arange([40, 17, 300, 100, 30][s]))
                assert_within(out[i:i + 1], *attended(q[i:i + 1].double().cpu(), K[at], V[at], 0.125))


def test_extreme_exponents():
    """Rows under the least and the largest exponents, V a wide range below: nothing is lost or overflows on the way."""
    c = filled(E4, 1, 64, 16, 8, max_seqs=2)
    lens = [70, 40]
    table = with_sequences(c, lens)
    c.k_exp[...], c.v_exp[...] = 119, 127 + 100          # K about 2^-8 x 60, V about 2^100 x 60
    s = slots_of(table, 16, 1, np.arange(40))
    page, at = torch.from_numpy(s // 16).to(dev()), torch.from_numpy(s % 16).to(dev())
    c.v_exp[page, 0, at] = 27                             # the least: 2^-100
    c.k_exp[page[:20], 0, at[:20]] = 27
    K, V = features(c)
    q = _rand((2, 4, 64), BF, 5)
    out = torch.full_like(q, float("nan"))
    ws = torch.zeros(sm.decode_workspace_bytes(2, 4, 64, 70), dtype=torch.uint8, device=dev())
    sm.decode_attention(c, i32([0, 1]), q, out, ws, 70)
    pre = torch.full((110, 4, 64), float("nan"), dtype=BF, device=dev())
    qp = _rand((110, 4, 64), BF, 6)
    sm.prefill_attention(c, i32([0, 1]), i32([0, 70, 110]), qp, pre, 70)
    torch.cuda.synchronize()
    assert c.error_bits() == 0
    for i, L in enumerate(lens):
        at = slots_of(table, 16, i, np.arange(L))
        assert_within(out[i:i + 1], *attended(q[i:i + 1].double().cpu(), K[at], V[at], 0.125))
        seen = torch.ones((L, L), dtype=torch.bool).tril()
        rows = slice(0, 70) if i == 0 else slice(70, 110)
        assert_within(pre[rows], *attended(qp[rows].double().cpu(), K[at], V[at], 0.125, seen))


PREFILLS = [
    # Hq, Hkv, D, bs, (rows, entries before them) of each request, scale
    (32, 8, 128, 16, [(100, 0)], None),
    (32, 8, 128, 16, [(1, 0), (1, 4000), (7, 60)], None),        # few rows, split or not by their length
    (4, 4, 64, 64, [(64, 0), (65, 1), (0, 50), (33, 300)], -0.2),
    (16, 4, 64, 16, [(300, 17), (255, 0), (256, 256)], None),
    (28, 4, 128, 32, [(500, 0), (130, 1000)], None),
    (8, 8, 128, 512, [(700, 0)], None),
    (16, 1, 128, 16, [(40, 900)], 0.0),
    (16, 4, 64, 16, [(1500, 0)] * 4, None),
    (32, 8, 128, 16, [(1100, 0)] * 3, None),
]


# The same with the form that the call takes: the waves apart, or the groups that they split a tile's keys into.
FORMS = [
    (32, 8, 128, 16, [(250, 700)], "apart"),
    (28, 4, 128, 64, [(61, 0), (3, 900), (1, 0), (17, 100)], "apart"),     # 4 rows of 7 heads, 4 vectors idle
    (16, 1, 64, 512, [(5, 1000), (0, 3), (2, 511)], "apart"),
    (4, 4, 128, 16, [(33, 31), (32, 32), (31, 33), (1, 255), (1, 256), (1, 257)], "apart"),
    (32, 8, 128, 32, [(8, 3 * i) for i in range(40)], "apart"),            # a request's rows are one workgroup's
    (32, 8, 128, 16, [(20, 100)] * 12, "few"),
    (32, 8, 128, 16, [(400, 50)], 4),
    (32, 8, 128, 64, [(1024, 0)], 2),
    (32, 8, 128, 16, [(700, 10)] * 3, 1),
    (16, 4, 64, 16, [(250, 100)], "apart"),
    (16, 4, 64, 16, [(20, 100)] * 23, "few"),
    (16, 4, 64, 32, [(1000, 20)], 4),
    (16, 4, 64, 16, [(2000, 0)], 2),
    (16, 4, 64, 16, [(1300, 0)] * 4, 1),
]


@pytest.mark.parametrize("case", range(len(PREFILLS) + len(FORMS)))
def test_prefill_matches_formula(case):
    Hq, Hkv, D, bs, reqs, scale = (PREFILLS + [(*f[:5], None) for f in FORMS])[case]
    lens = [m + past for m, past in reqs]
    c = filled(E4, Hkv, D, bs, sum(-(-x // bs) for x in lens) + 1, max_seqs=len(lens),
               max_blocks_per_seq=-(-max(lens) // bs))
    table = with_sequences(c, lens, case)
    poisoned(c, table, lens)
    K, V = features(c)
    offs = np.concatenate([[0], np.cumsum([m for m, _ in reqs])])
    q = _rand((offs[-1] + 2, Hq, D), BF, case)
    out = torch.full_like(q, 7.0)
    say("e4m3 prefill", case, Hq, Hkv, D, bs, reqs)
    sm.prefill_attention(c, i32(range(len(lens))), i32(offs), q, out, max(m for m, _ in reqs), scale=scale)
    torch.cuda.synchronize()
    assert c.error_bits() == 0 and bool((out[offs[-1]:] == 7).all())
    for i, (m, past) in enumerate(reqs):
        at, rows = slots_of(table, bs, i, np.arange(m + past)), slice(offs[i], offs[i + 1])
        seen = torch.ones((m, m + past), dtype=torch.bool).tril(past)
        if m:
            assert_within(out[rows], *attended(q[rows].double().cpu(), K[at], V[at], D ** -0.5 if scale is None else scale, seen))


def test_prefill_errors_leave_zero_rows():
    c = filled(E4, 2, 64, 16, 40, max_seqs=4, max_blocks_per_seq=20)
    table = with_sequences(c, [40, 17, 300, 30])
    c.block_table[2, 3] = -1
    K, V = features(c)
    q = _rand((60, 4, 64), BF, 1)
    for ids, offs in (([0, 9, 1], [0, 20, 43, 60]), ([0, 1, 3], [0, 20, 43, 60]), ([0, 2, 1], [0, 20, 43, 60])):
        out = torch.full_like(q, float("nan"))
        sm.prefill_attention(c, i32(ids), i32(offs), q, out, 30)
        torch.cuda.synchronize()
        assert c.error_bits() == sm.ERR_EINVAL
        c.clear_error()
        assert not out[20:43].any()
        at, seen = slots_of(table, 16, 0, np.arange(40)), torch.ones((20, 40), dtype=torch.bool).tril(20)
        assert_within(out[:20], *attended(q[:20].double().cpu(), K[at], V[at], 0.125, seen))


def test_queries_of_another_type_are_refused():
    c = sm.PagedCache(dtype=E4, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=4, max_seqs=2, max_blocks_per_seq=2)
    q = torch.zeros((1, 4, 64), device=dev())
    ws = torch.zeros(sm.decode_workspace_bytes(1, 4, 64, 32), dtype=torch.uint8, device=dev())
    for a, b in ((q, q), (q.to(BF), q), (q.to(E4), q.to(BF))):
        with pytest.raises(sm.SpanMergeError, match="q, out"):
            sm.decode_attention(c, i32([0]), a, b, ws, 32)
        with pytest.raises(sm.SpanMergeError, match="q, out"):
            sm.prefill_attention(c, i32([0]), i32([0, 1]), a, b, 1)
