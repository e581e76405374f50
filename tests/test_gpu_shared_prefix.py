"""Decode attention of requests behind entries that their group shares, against
the formula in 64 bits over the prefix's entries and then the request's own."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm
from test_gpu_e4m3_attention import assert_within, attended, poisoned
from test_gpu_e4m3_write import BF, E4, features, filled, slots_of, with_sequences
from test_gpu_rotary import _rand

pytestmark = pytest.mark.gpu


def shared(c, ids, prefixes, offs, q, max_len, max_prefix, scale=None, out=None, ws=None):
    n, Hq, D = q.shape
    out = torch.full_like(q, float("nan")) if out is None else out
    ws = torch.zeros(sm.decode_shared_workspace_bytes(n, Hq, D, max_len, max_prefix), dtype=torch.uint8, device=dev()) \
        if ws is None else ws
    sm.decode_attention_shared(c, i32(ids), i32(prefixes), i32(offs), q, out, ws, max_len, max_prefix, scale=scale)
    torch.cuda.synchronize()
    return out


def check(c, table, lens, ids, prefixes, offs, q, out, scale=None, skip=()):
    K, V = features(c)
    at = {s: slots_of(table, c.bs, s, np.arange(lens[s])) for s in set(ids) | set(prefixes) if 0 <= s < len(lens)}
    for p, prefix in enumerate(prefixes):
        before = at.get(prefix, np.zeros(0, np.int64))
        for i in range(offs[p], offs[p + 1]):
            if i in skip:
                assert not out[i].any()
                continue
            s = np.concatenate([before, at[ids[i]]])
            assert_within(out[i:i + 1], *attended(q[i:i + 1].double().cpu(), K[s], V[s], c.D ** -0.5 if scale is None else scale))


CASES = [
    # Hq, Hkv, D, bs, prefixes' lengths, requests of each group, own lengths (their range, or a list), scale
    (32, 8, 128, 16, [2048], [16], (1, 640), None),
    (28, 4, 128, 16, [1000, 3000, 17], [20, 31, 9], (0, 300), None),
    (16, 4, 64, 32, [1], [1], [1], None),
    (16, 4, 64, 16, [333, 0, 128, 129, 127, 5000], [3, 2, 0, 1, 7, 1], (0, 40), None),
    (4, 4, 64, 64, [700], [5], [0, 0, 3, 900, 1], -0.4),
    (8, 2, 64, 16, [0, 0], [2, 1], [0, 5, 0], None),             # nothing at all to attend to for two of them
    (16, 1, 128, 512, [9000], [40], (1, 100), None),             # more than one chunk of the longest, 640 vectors
    (64, 8, 128, 16, [400], [100], (100, 200), None),            # more pairs than compute units
    (32, 8, 128, 16, [300], [3], [5000, 1, 2600], 0.0),          # own entries in several chunks; scale 0
    (8, 8, 64, 16, [20, 50], [300, 260], (1, 3), None),
    (4, 2, 128, 16, [70] * 600, [0, 1, 0] * 200, (1, 20), None),  # more groups than threads of a workgroup
    (16, 1, 64, 16, [3700], [1000], (0, 2), None),               # chunks long enough for two workgroups a compute unit
]


@pytest.mark.parametrize("dt", [BF, E4], ids=str)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_shared_matches_formula(case, dt):
    Hq, Hkv, D, bs, plens, members, own, scale = CASES[case]
    rng, n, P = np.random.RandomState(case), sum(members), len(plens)
    mine = list(own) if isinstance(own, list) else rng.randint(own[0], own[1] + 1, n).tolist()
    lens = plens + mine
    c = filled(dt, Hkv, D, bs, sum(-(-x // bs) for x in lens) + 1, max_seqs=len(lens), max_blocks_per_seq=max(1, -(-max(lens) // bs)))
    table = with_sequences(c, lens, case)
    if dt == E4:
        poisoned(c, table, lens)
    ids, prefixes = (P + rng.permutation(n)).tolist(), rng.permutation(P).tolist()
    offs = np.concatenate([[0], np.cumsum(members)])
    q = _rand((n, Hq, D), BF, case)
    say("shared", dt, case, Hq, Hkv, D, bs, "requests", n, "longest", max(plens), max(mine))
    ws = torch.full((sm.decode_shared_workspace_bytes(n, Hq, D, max(mine), max(plens)),), 0xff, dtype=torch.uint8, device=dev())
    ws[:256 * 1024] = 0                                          # (the counters alone have to be zero)
    outs = []
    for _ in range(2):
        outs.append(shared(c, ids, prefixes, offs, q, max(mine), max(plens), scale, ws=ws))
        assert c.error_bits() == 0 and not ws[:256 * 1024].any()
    assert torch.equal(*outs)
    check(c, table, lens, ids, prefixes, offs, q, outs[0], scale)


@pytest.mark.parametrize("dt", [BF, E4], ids=str)
def test_one_prefix_for_several_groups_and_groups_without(dt):
    lens = [500, 3, 70, 40, 9]
    c = filled(dt, 2, 64, 16, 60, max_seqs=5, max_blocks_per_seq=40)
    table = with_sequences(c, lens)
    # a request may name a sequence that is another's prefix, and the same one twice
    ids, prefixes, offs = [1, 2, 2, 0, 3, 4], [0, -1, 0, 3], [0, 2, 4, 5, 6]
    q = _rand((6, 8, 64), BF, 3)
    out = shared(c, ids, prefixes, offs, q, 500, 600)
    assert c.error_bits() == 0
    check(c, table, lens, ids, prefixes, offs, q, out)
    # without any prefix: sm_decode_attention's rows
    alone = shared(c, ids, [-1], [0, 6], q, 500, 0)
    ws = torch.zeros(sm.decode_workspace_bytes(6, 8, 64, 500), dtype=torch.uint8, device=dev())
    plain = torch.empty_like(q)
    sm.decode_attention(c, i32(ids), q, plain, ws, 500)
    torch.cuda.synchronize()
    assert torch.equal(alone, plain) and c.error_bits() == 0


@pytest.mark.parametrize("dt", [BF, E4], ids=str)
def test_errors_leave_zero_rows(dt):
    lens = [200, 90, 40, 17, 300, 1]
    c = filled(dt, 2, 64, 16, 60, max_seqs=6, max_blocks_per_seq=30)
    table = with_sequences(c, lens)
    q = _rand((5, 4, 64), BF, 4)

    def call(ids, prefixes, offs, bits, skip, max_len=299, max_prefix=199):
        out = shared(c, ids, prefixes, offs, q, max_len, max_prefix)
        assert c.error_bits() == bits, (c.error_bits(), bits)
        c.clear_error()
        check(c, table, lens, ids, prefixes, offs, q, out, skip=skip)
    call([2, 3, 5, 2, 3], [1, -1], [0, 3, 5], 0, ())
    call([2, 3, 9, 2, 3], [1, -1], [0, 3, 5], sm.ERR_EINVAL, (2,))
    call([2, 3, 5, 2, 4], [1, -1], [0, 3, 5], sm.ERR_ERANGE, (4,))
    call([2, 3, 5, 2, 3], [6, 1], [0, 3, 5], sm.ERR_EINVAL, (0, 1, 2))
    call([2, 3, 5, 2, 3], [1, -2], [0, 3, 5], sm.ERR_EINVAL, (3, 4))
    call([2, 3, 5, 2, 3], [1, 0], [0, 3, 5], sm.ERR_ERANGE, (3, 4))
    for offs in ([0, 3, 4], [1, 3, 5], [0, 6, 5], [0, -1, 5], [0, 3, 6]):     # no list of the requests
        out = shared(c, [2, 3, 5, 2, 3], [1, -1], offs, q, 299, 199)
        assert c.error_bits() == sm.ERR_EINVAL and not out.any()
        c.clear_error()
    c.block_table[1, 2] = 60
    call([2, 3, 5, 2, 3], [1, -1], [0, 3, 5], sm.ERR_EINVAL, (0, 1, 2))
    c.lengths[1] = -5
    call([2, 3, 5, 2, 3], [1, -1], [0, 3, 5], sm.ERR_EINVAL, (0, 1, 2))
    c.lengths[1] = 2 ** 31 - 1
    call([2, 3, 5, 2, 3], [1, -1], [0, 3, 5], sm.ERR_EINVAL, (0, 1, 2))


def test_nan_reaches_the_rows_that_attend_to_it_alone():
    lens = [40, 20, 20]
    for dt in (BF, E4):
        c = filled(dt, 2, 64, 16, 12, max_seqs=3, max_blocks_per_seq=4)
        table = with_sequences(c, lens)
        page = int(table[1, 0])
        c.k_pool.view(torch.uint8)[page, 0, 3] = 0x7f                # e4m3's NaN; 0x7f7f in bf16 is 3.4e38
        if dt == BF:
            c.k_pool[page, 0, 3] = float("nan")
        q = _rand((2, 4, 64), BF, 4)
        out = shared(c, [1, 2], [0], [0, 2], q, 20, 40)
        assert bool(out[0, :2].isnan().all()) and not out[0, 2:].isnan().any() and not out[1].isnan().any()
        page = int(table[0, 1])
        c.v_pool.view(torch.uint8)[page, 1] = 0x7f
        if dt == BF:
            c.v_pool[page, 1] = float("nan")
        out = shared(c, [1, 2], [0], [0, 2], q, 20, 40)
        assert bool(out[:, 2:].isnan().all()) and not out[1, :2].isnan().any()


def test_refusals():
    c = sm.PagedCache(dtype=torch.float32, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=4, max_seqs=2,
                      max_blocks_per_seq=2)
    b = sm.PagedCache(dtype=BF, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=4, max_seqs=2, max_blocks_per_seq=2)
    q = torch.zeros((1, 4, 64), dtype=BF, device=dev())
    ws = torch.zeros(sm.decode_shared_workspace_bytes(1, 4, 64, 32, 32), dtype=torch.uint8, device=dev())

    def call(cache=b, ids=i32([0]), prefixes=i32([1]), offs=i32([0, 1]), q=q, out=q, ws=ws, L=32, P=32, **kw):
        sm.decode_attention_shared(cache, ids, prefixes, offs, q, out, ws, L, P, **kw)
    call()
    for kw in (dict(cache=c), dict(P=33), dict(L=33), dict(P=-1), dict(prefixes=i32([]), offs=i32([0])), dict(ws=ws[:-1]),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(q=q.float()), dict(out=q.float()), dict(offs=i32([0])),
               dict(ids=i32([])), dict(out=q[:, :2]), dict(ids=torch.zeros(1, dtype=torch.int64, device=dev()))):
        with pytest.raises(sm.SpanMergeError):
            call(**kw)
    call(ids=i32([]), q=q[:0], out=q[:0], offs=i32([0, 0]))
    torch.cuda.synchronize()
    assert b.error_bits() == 0
