"""kv_reserve against the oracle's rollback and append bookkeeping: the same
tables, lengths and free stack, and the slots that follow from them."""
import numpy as np
import pytest
import torch

from gpu_util import ERR_OF_STATUS, assert_same_state, dev, gpu_cache_like, i32, say
from paper_2609_27233_amd import lib as sm

pytestmark = pytest.mark.gpu

H, D = 1, 64


def _cache(orc, rng, bs, lens, spare, extra_blocks=3):
    n = len(lens)
    nb = sum(-(-int(x) // bs) for x in lens) + spare
    mb = max([-(-int(x) // bs) for x in lens] + [1]) + extra_blocks
    oc = orc.OracleCache(bf16=True, num_kv_heads=H, head_dim=D, block_size=bs, num_blocks=max(nb, 1), max_seqs=n + 1,
                         max_blocks_per_seq=mb, free_order=rng.permutation(max(nb, 1)).astype(np.int32))
    order = rng.permutation(n)
    for i in order:                                             # pages of a sequence in any order
        z = np.zeros((int(lens[i]), H, D), np.uint16)
        assert oc.append([i], [0, int(lens[i])], z, z) == orc.OK
    return oc, gpu_cache_like(oc, torch.bfloat16)


def _reserve(c, ids, crop, rows, room, stream=None):
    n = len(ids)
    out = [torch.full((k,), -77, dtype=torch.int32, device=dev()) for k in (n + 1, room, room)]
    sm.kv_reserve(c, i32(ids), i32(rows), *out, crop=None if crop is None else i32(crop), stream=stream)
    return out


def _check(orc, oc, c, ids, crop, rows, out):
    """The oracle's state after the same request, and the rows' places in it."""
    crop = np.zeros(len(ids), int) if crop is None else np.asarray(crop)
    rows = np.asarray(rows)
    offs = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    z = np.zeros((int(offs[-1]), H, D), np.uint16)
    st = oc.rollback(ids, crop)
    assert st == orc.OK
    assert oc.append(ids, offs, z, z) == orc.OK
    torch.cuda.synchronize()
    assert c.error_bits() == 0
    assert_same_state(c, oc, pools=False)
    ro, pos, slots = (t.cpu().numpy() for t in out)
    np.testing.assert_array_equal(ro, offs)
    want_pos, want_slot = np.zeros(len(pos), np.int64), np.full(len(pos), -1, np.int64)
    for i, s in enumerate(ids):
        p = int(oc.lengths[s]) - rows[i] + np.arange(rows[i], dtype=np.int64)
        want_pos[offs[i]:offs[i + 1]] = p
        want_slot[offs[i]:offs[i + 1]] = oc.block_table[s][p // oc.bs].astype(np.int64) * oc.bs + p % oc.bs
    np.testing.assert_array_equal(pos, want_pos)
    np.testing.assert_array_equal(slots, want_slot)


CASES = [
    # bs, lengths, crop (None: none), rows, room behind the rows
    (16, [0], None, [1], 0),
    (16, [0], None, [0], 3),
    (16, [16], [16], [16], 0),
    (16, [17, 15, 16, 1, 0], [1, 15, 0, 1, 0], [1, 1, 1, 33, 16], 5),
    (16, [40, 40], [40, 0], [0, 25], 0),                        # one request's freed blocks go to the other
    (32, [100, 3, 64], [70, 3, 64], [0, 0, 0], 2),              # rows of none
    (512, [700, 511, 513], [3, 511, 513], [900, 2, 1], 1),
    (16, [300] * 7, [299] * 7, [298] * 7, 4000),                # padded far behind
    (16, [0] * 3, None, [4095, 1, 0], 0),                       # 4096 rows: placed by the one workgroup
    (16, [5, 0, 31], None, [4096, 7, 900], 11),                 # more: by a second launch
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("order", ["listed", "mixed"])
def test_reserve_matches_rollback_then_append(orc, case, order):
    bs, lens, crop, rows, room = CASES[case]
    rng = np.random.RandomState(case)
    oc, c = _cache(orc, rng, bs, lens, spare=sum(-(-r // bs) for r in rows) + 2, extra_blocks=max(rows) // bs + 2)
    at = np.arange(len(lens)) if order == "listed" else rng.permutation(len(lens))
    rows = [rows[i] for i in at]
    crop = None if crop is None else [crop[i] for i in at]
    say("reserve", case, order)
    _check(orc, oc, c, at.astype(np.int32), crop, rows, _reserve(c, at, crop, rows, sum(rows) + room))


@pytest.mark.parametrize("n,top_len,top_rows", [(1, 5000, 3000), (33, 200, 40), (256, 90, 8), (1024, 40, 3), (1000, 33, 60),
                                                (500, 60, 2), (200, 50, 1), (40, 70, 1)])
def test_reserve_random_batches(orc, n, top_len, top_rows):
    rng = np.random.RandomState(n)
    lens = rng.randint(0, top_len + 1, n)
    oc, c = _cache(orc, rng, 16, lens, spare=n * (top_rows // 16 + 2), extra_blocks=3 * (top_rows // 16 + 2))
    for step in range(3):
        m = max(1, int(n * (1, 0.5, 1)[step]))
        ids = rng.permutation(n)[:m].astype(np.int32)
        crop = np.minimum(rng.randint(0, top_rows + 1, m), oc.lengths[ids])
        rows = rng.randint(0, top_rows + 1, m) if step else rng.randint(0, 2, m)
        say("reserve", n, "step", step)
        _check(orc, oc, c, ids, crop, rows, _reserve(c, ids, crop, rows, int(rows.sum()) + step))


def test_reserve_equals_rollback_and_append_calls(orc):
    """The library's own two calls on a twin cache: the same state, stack entries past the top among it."""
    rng = np.random.RandomState(5)
    lens = rng.randint(1, 100, 20)
    oc, a = _cache(orc, rng, 16, lens, spare=60)
    b = gpu_cache_like(oc, torch.bfloat16)
    ids = rng.permutation(20).astype(np.int32)
    crop, rows = np.minimum(rng.randint(0, 60, 20), lens[ids]), rng.randint(0, 50, 20)
    _reserve(a, ids, crop, rows, int(rows.sum()))
    offs = np.concatenate([[0], np.cumsum(rows)])
    z = torch.zeros((int(offs[-1]), H, D), dtype=torch.bfloat16, device=dev())
    sm.kv_rollback(b, i32(ids), i32(crop))
    sm.kv_append(b, i32(ids), i32(offs), z, z)
    torch.cuda.synchronize()
    assert a.error_bits() == 0 and b.error_bits() == 0
    for name in ("block_table", "lengths", "free_stack", "free_top"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_no_request(orc):
    oc, c = _cache(orc, np.random.RandomState(0), 16, [20], spare=2)
    for room in (0, 5, 5000):
        out = _reserve(c, [], None, [], room)
        torch.cuda.synchronize()
        assert out[0].tolist() == [0] and (out[1] == 0).all() and (out[2] == -1).all() and c.error_bits() == 0
    assert_same_state(c, oc, pools=False)


def _refused(c, oc, out, bit):
    torch.cuda.synchronize()
    assert c.error_bits() == bit
    assert (out[0] == 0).all() and (out[1] == 0).all() and (out[2] == -1).all()
    assert_same_state(c, oc, pools=False)


BAD = [
    # lengths, ids, crop, rows, room, spare blocks, error
    ([20, 20], [0, 0], None, [1, 1], 2, 4, sm.ERR_EINVAL),       # the same sequence twice
    ([20, 20], [0, 3], None, [1, 1], 2, 4, sm.ERR_EINVAL),       # max_seqs is 3
    ([20, 20], [-1, 0], None, [1, 1], 2, 4, sm.ERR_EINVAL),
    ([20, 20], [0, 1], [-1, 0], [1, 1], 2, 4, sm.ERR_EINVAL),
    ([20, 20], [0, 1], None, [1, -1], 2, 4, sm.ERR_EINVAL),
    ([20, 20], [0, 1], None, [2, 1], 2, 4, sm.ERR_EINVAL),       # more rows than room
    ([20, 20], [0, 1], None, [2 ** 31 - 1, 2 ** 31 - 1], 2, 4, sm.ERR_EINVAL),
    ([20, 20], [0, 1], [21, 0], [1, 1], 2, 4, sm.ERR_ERANGE),
    ([20, 20], [0, 1], [2 ** 31 - 1, 0], [1, 1], 2, 4, sm.ERR_ERANGE),
    ([20, 20], [0, 1], None, [70, 1], 71, 40, sm.ERR_ERANGE),    # 5 blocks of 16 at most
    ([20, 20], [0, 1], None, [13, 13], 26, 1, sm.ERR_ENOMEM),    # 2 blocks, 1 free
    ([20, 20], [0, 1], [0, 21], [-5, 1], 2, 4, sm.ERR_EINVAL),   # both: EINVAL comes first
]


@pytest.mark.parametrize("case", range(len(BAD)))
@pytest.mark.parametrize("pad", [0, 5000])                      # (with the rows in a second launch, too)
def test_refusals_leave_everything(orc, case, pad):
    lens, ids, crop, rows, room, spare, bit = BAD[case]
    if pad and sum(r for r in rows if r > 0) > room:
        pad = 0                                                  # (padding would make room)
    oc, c = _cache(orc, np.random.RandomState(case), 16, lens, spare=spare)
    say("refusal", case, "pad", pad)
    out = _reserve(c, ids, crop, rows, room + pad)
    _refused(c, oc, out, bit)
    out = _reserve(c, [0], None, [1], 3)                          # sticky: frozen until cleared
    _refused(c, oc, out, bit)
    c.clear_error()
    _check(orc, oc, c, np.array([0], np.int32), None, [1], _reserve(c, [0], None, [1], 3))


@pytest.mark.parametrize("what", ["stack", "table-freed", "table-tail", "top-low", "top-high", "full"])
def test_corrupt_tables_are_refused(orc, what):
    oc, c = _cache(orc, np.random.RandomState(9), 16, [40, 24], spare=4)
    top = int(oc.free_top[0])
    ids, crop, rows, bit = [0, 1], [0, 0], [20, 20], sm.ERR_EINVAL
    if what == "stack":
        oc.free_stack[top - 2] = oc.num_blocks
    elif what == "table-freed":
        oc.block_table[0][2] = -1
        crop, rows = [10, 0], [0, 0]
    elif what == "table-tail":
        oc.block_table[1][1] = oc.num_blocks + 7
        rows = [0, 1]
    elif what == "top-low":
        oc.free_top[0] = -1
    elif what == "top-high":
        oc.free_top[0] = oc.num_blocks + 1
    else:                                                        # more blocks free than there is room to push
        oc.free_top[0] = oc.num_blocks
        crop, rows, bit = [40, 24], [0, 0], sm.ERR_ERANGE
    c = gpu_cache_like(oc, torch.bfloat16)
    say("corrupt", what)
    out = _reserve(c, ids, crop, rows, sum(rows))
    torch.cuda.synchronize()
    assert c.error_bits() == bit and (out[2] == -1).all() and (out[0] == 0).all()
    for name in ("block_table", "lengths", "free_stack", "free_top"):
        np.testing.assert_array_equal(getattr(c, name).cpu().numpy(), getattr(oc, name))


@pytest.mark.parametrize("room", [40, 6000])
def test_captured_and_replayed(orc, room):
    """A step's reserve in a graph, its counts changed between replays."""
    rng = np.random.RandomState(3)
    lens = rng.randint(20, 60, 12)
    oc, c = _cache(orc, rng, 16, lens, spare=60, extra_blocks=6)
    ids = rng.permutation(12).astype(np.int32)
    t_ids, t_crop, t_rows = i32(ids), i32(np.zeros(12)), i32(np.zeros(12))
    out = [torch.empty(k, dtype=torch.int32, device=dev()) for k in (13, room, room)]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        sm.kv_reserve(c, t_ids, t_rows, *out, crop=t_crop)       # (no rows: nothing moves)
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        sm.kv_reserve(c, t_ids, t_rows, *out, crop=t_crop)
    for step in range(4):
        crop, rows = rng.randint(0, 4, 12), rng.randint(0, 4, 12)
        t_crop.copy_(i32(crop))
        t_rows.copy_(i32(rows))
        say("replay", step)
        g.replay()
        _check(orc, oc, c, ids, crop, rows, out)
