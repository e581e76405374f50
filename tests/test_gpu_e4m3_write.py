"""K and V written into 8-bit pages, and cached entries of every page type read
back, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm
from test_gpu_rotary import _rand, _runs, assert_near, turned

pytestmark = pytest.mark.gpu

BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def rounded(y):
    """y (fp64, at most 448 in size) to the nearest e4m3 value, ties to even, by its steps."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def row_exps(x, factor=1.0):
    """Exponent of each row: the least e with factor max|x| <= 2^(e + 8), over its finite features."""
    m = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1) * factor
    e = torch.where(m > 0, torch.ceil(torch.log2(m.clamp(min=2.0 ** -140))) - 8, -1000.0)
    return e.clamp(-100, 119)


def filled(dt, H, D, bs, nb, seed=100, **kw):
    """A cache with something in every byte."""
    c = sm.PagedCache(dtype=dt, num_kv_heads=H, head_dim=D, block_size=bs, num_blocks=nb,
                      **{**dict(max_seqs=4, max_blocks_per_seq=nb), **kw})
    for i, pool in enumerate((c.k_pool, c.v_pool)):
        pool.copy_((_rand(pool.shape, F32, seed + i) * (60 if dt == E4 else 1)).to(dt))
    if dt == E4:
        for i, e in enumerate((c.k_exp, c.v_exp)):
            e.copy_(torch.randint(115, 125, e.shape, generator=torch.Generator().manual_seed(seed + 2 + i)).to(torch.uint8))
    return c


def by_slot(c):
    """(K values, V values [slots, H, D], K exponents, V exponents [slots, H]) of the pages, fp64 on the host."""
    k = c.k_pool.float().cpu().double().transpose(1, 2).flatten(0, 1)
    v = c.v_pool.float().cpu().double().permute(0, 3, 1, 2).flatten(0, 1)
    if c.k_exp is None:
        return k, v, None, None
    return k, v, c.k_exp.cpu().transpose(1, 2).flatten(0, 1).long(), c.v_exp.cpu().transpose(1, 2).flatten(0, 1).long()


def check_write(c, before, slots, pos, k, v, a, q=None, q_out=None):
    """The pages after a write of these rows over `before`."""
    k0, v0, ke0, ve0 = before
    k1, v1, ke1, ve1 = by_slot(c)
    there = torch.from_numpy(np.asarray(slots) >= 0)
    s = torch.from_numpy(np.asarray(slots)[np.asarray(slots) >= 0].astype(np.int64))
    factor = max(1.0, abs(float(np.float32(a.get("attn_scale", 1.0)))))
    ek, ev = (row_exps(x.double().cpu()[there], f) for x, f in ((k, factor), (v, 1.0)))
    ref, slack = turned(k, pos, a)
    ref, slack = ref[there] * torch.exp2(-ek)[..., None], slack[there] * torch.exp2(-ek)[..., None]
    # the turn is off by its slack before it is rounded, and rounding keeps the order of values
    assert bool(((k1[s] >= rounded(ref - slack)) & (k1[s] <= rounded(ref + slack))).all())
    v0[s], ke0[s], ve0[s], k0[s] = rounded(v.double().cpu()[there] * torch.exp2(-ev)[..., None]), ek.long() + 127, \
        ev.long() + 127, k1[s]
    for got, want in ((k1, k0), (v1, v0), (ke1, ke0), (ve1, ve0)):
        assert torch.equal(got, want)
    if q is not None:
        assert_near(q_out, *turned(q, pos, a), BF)


WRITES = [
    # Hq, Hkv, D, bs, rows of each sequence, padded rows, kind of slots
    (32, 8, 128, 16, [1] * 16, 0, "runs"),
    (28, 4, 128, 16, [1], 0, "runs"),
    (32, 8, 128, 16, [100, 3, 17, 64], 5, "runs"),
    (4, 1, 64, 64, [200, 1, 1, 90], 0, "runs"),
    (0, 2, 64, 32, [33, 40], 3, "runs"),                    # K and V alone
    (8, 8, 128, 512, [600, 30], 0, "runs"),
    (3, 2, 128, 32, [50], 0, "runs"),
    (4, 3, 64, 16, [90], 0, "any"),                         # slots in any order
    (4, 2, 64, 16, [90], 0, "down"),                        # counted down
    (2, 2, 64, 16, [300], 40, "holes"),                     # padded rows between the others
    (2, 1, 128, 16, [700], 0, "runs"),
    (32, 8, 128, 16, [2000, 2001, 1999], 0, "runs"),
]


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("case", range(len(WRITES)))
def test_write_matches_definition(case, packed):
    Hq, Hkv, D, bs, lens, pad, kind = WRITES[case]
    rng = np.random.RandomState(case)
    nb = sum(-(-x // bs) + 1 for x in lens) + 2
    c = filled(E4, Hkv, D, bs, nb)
    n = sum(lens)
    slots = _runs(rng, nb, bs, lens)
    if kind == "any":
        slots = rng.permutation(nb * bs)[:n]
    if kind == "down":
        slots = nb * bs - 1 - np.arange(n)
    slots = np.concatenate([slots, np.full(pad, -1)])
    if kind == "holes":
        order = np.sort(np.concatenate([np.arange(n), rng.choice(n, pad)]), kind="stable")
        slots = slots[:n][order]
        slots[1:][order[1:] == order[:-1]] = -1                  # each repeat becomes a hole
    rows = len(slots)
    pos = torch.from_numpy(rng.randint(0, 40000, rows).astype(np.int32))
    a = dict(rot_dim=D if case % 3 else D // 2, layout="interleaved" if case % 2 else "half", scaling="bands", factor=8.0,
             attn_scale=(1.0, 1.3, -2.0, 0.5)[case % 4])
    if packed:
        buf = _rand((rows, (Hq + 2 * Hkv) * D), BF, case)
        q, k, v = (t.unflatten(1, (-1, D)) for t in buf.split([Hq * D, Hkv * D, Hkv * D], 1))
    else:
        q, k, v = (_rand((rows, h, D), BF, 3 * case + i) for i, h in enumerate((Hq, Hkv, Hkv)))
        k *= torch.exp2(torch.randint(-20, 20, (rows, Hkv, 1), generator=torch.Generator().manual_seed(case)).to(dev()))
    before = by_slot(c)
    say("e4m3 write", case, "packed", packed, "rows", rows)
    q_out = torch.full((rows, Hq, D), float("nan"), dtype=BF, device=dev()) if Hq else None
    sm.kv_write_rotary(c, pos.to(dev()), i32(slots), q if Hq else None, k, v, sm.rope_params(**a), q_out)
    torch.cuda.synchronize()
    assert c.error_bits() == 0
    check_write(c, before, slots, pos, k, v, a, q if Hq else None, q_out)


@pytest.mark.parametrize("R,layout", [(64, "half"), (6, "half"), (62, "interleaved"), (2, "half"), (50, "half")])
def test_write_unaligned_columns_and_narrow_turns(R, layout):
    Hq, Hkv, D, bs = 2, 1, 64, 16
    c = filled(E4, Hkv, D, bs, 4)
    buf = _rand((37, 400), BF, 8)
    q, k, v = buf[:, 1:129].view(37, 2, D), buf[:, 131:195].view(37, 1, D), buf[:, 203:267].view(37, 1, D)
    pos = torch.arange(37, dtype=torch.int32) * 11
    a = dict(rot_dim=R, layout=layout)
    before, q_out = by_slot(c), torch.zeros((37, 2, D), dtype=BF, device=dev())
    slots = np.arange(37) + 5
    say("e4m3 write unaligned", R, layout)
    sm.kv_write_rotary(c, pos.to(dev()), i32(slots), q, k, v, sm.rope_params(**a), q_out)
    torch.cuda.synchronize()
    check_write(c, before, slots, pos, k, v, a, q, q_out)


@pytest.mark.parametrize("shift", [0, 1])
def test_special_values(shift):
    """Zeros, the smallest and largest rows, powers of two and what lies beside them, NaN and infinities."""
    D, n = 64, 20
    buf = torch.zeros((n, 1, 2 * D + shift), dtype=BF, device=dev())
    x = buf[..., shift:shift + D]
    x.copy_(_rand((n, 1, D), BF, 3).clamp(-0.99, 0.99))
    tops = [0.0, 1.0, 256.0, 257.0, 258.0, 2.0 ** -100, 2.0 ** -133, 2.0 ** 127, 1.99 * 2.0 ** 127, 2.0 ** 119, 448.0, 464.0]
    for r, t in enumerate(tops):
        x[r] *= t
        x[r, 0, 5] = -t
    x[12, 0, 3], x[13, 0, 3], x[14, 0, 63], x[15] = float("inf"), float("nan"), -float("inf"), float("nan")
    x[16] = float("inf")
    c = filled(E4, 1, D, 16, 2)
    say("e4m3 special values", shift)
    # position 0 turns nothing; V goes the same way in a transposed page
    sm.kv_write_rotary(c, i32([0] * n), i32(range(n)), None, x, x, sm.rope_params(D), None)
    torch.cuda.synchronize()
    k, v, ke, ve = by_slot(c)
    xd = x.double().cpu()
    e = row_exps(xd)
    want = torch.where(xd.isfinite(), rounded((xd * torch.exp2(-e)[..., None]).clamp(-448, 448)), float("nan"))
    assert torch.equal(ke[:n], e.long() + 127) and torch.equal(ve[:n], e.long() + 127)
    # a pair with a NaN or an infinity turns into two NaN (0 times infinity is one)
    bad = want.isnan() | want.isnan().roll(D // 2, -1)
    for got, want in ((k[:n], torch.where(bad, float("nan"), want)), (v[:n], want)):
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def test_slots_out_of_range_are_refused_alone():
    c = filled(E4, 2, 64, 16, 4)
    before, n = by_slot(c), 20
    k, v = (_rand((n, 2, 64), BF, i) for i in range(2))
    pos, slots = torch.zeros(n, dtype=torch.int32), np.arange(n) + 8
    slots[[2, 11, 19]] = [64, -2, 2 ** 31 - 1]
    sm.kv_write_rotary(c, pos.to(dev()), i32(slots), None, k, v, sm.rope_params(64), None)
    torch.cuda.synchronize()
    assert c.error_bits() == sm.ERR_EINVAL
    slots[[2, 11, 19]] = -1
    check_write(c, before, slots, pos, k, v, dict(rot_dim=64))


@pytest.mark.parametrize("D,R,layout", [(128, 128, "half"), (64, 64, "half"), (128, 64, "half"), (128, 128, "interleaved")])
def test_a_row_has_the_same_bits_however_it_comes(D, R, layout):
    """Rows one element off a 16-byte address, alone and in full tiles, with and without neighbours."""
    rows, H = 70, 5
    k, v = (_rand((rows, H, D), BF, s).to(dev()) for s in (5, 6))
    pos, slots = i32(np.arange(rows) * 37 + 1000), i32(np.random.RandomState(2).permutation(96)[:rows])
    rope = sm.rope_params(R, layout=layout)
    caches = [filled(E4, H, D, 16, 6) for _ in range(4)]
    odd = [torch.empty((rows, H * D + 8), dtype=BF, device=dev())[:, 1:1 + H * D].unflatten(1, (H, D)) for _ in range(2)]
    for o, x in zip(odd, (k, v)):
        o.copy_(x)
    say("same bits", D, R, layout)
    sm.kv_write_rotary(caches[0], pos, slots, None, k, v, rope, None)
    sm.kv_write_rotary(caches[1], pos, slots, None, *odd, rope, None)
    order = slots.argsort()
    sm.kv_write_rotary(caches[2], pos[order], slots[order], None, k[order], v[order], rope, None)
    for r in range(rows):
        sm.kv_write_rotary(caches[3], pos[r:r + 1], slots[r:r + 1], None, k[r:r + 1], v[r:r + 1], rope, None)
    torch.cuda.synchronize()
    for c in caches[1:]:
        for name in ("k_pool", "v_pool", "k_exp", "v_exp"):
            assert torch.equal(getattr(c, name).view(torch.uint8), getattr(caches[0], name).view(torch.uint8)), name


# --------------------------------------------------------------------------
# entries read back

def features(c):
    """K, V [slots, H, D] in fp64 on the host, what the pages stand for."""
    k, v, ke, ve = by_slot(c)
    if ke is None:
        return k, v
    return k * torch.exp2(ke.double() - 127)[..., None], v * torch.exp2(ve.double() - 127)[..., None]


def with_sequences(c, lens, seed=0):
    """Sequences of these lengths on pages in any order."""
    order = np.random.RandomState(seed).permutation(c.num_blocks)
    table, at = np.full((c.max_seqs, c.max_blocks), -1, np.int32), 0
    for s, L in enumerate(lens):
        m = -(-L // c.bs)
        table[s, :m] = order[at:at + m]
        at += m
    c.block_table.copy_(torch.from_numpy(table))
    c.lengths[:len(lens)] = i32(lens)
    return table


def slots_of(table, bs, s, p):
    return table[s, np.asarray(p) // bs].astype(np.int64) * bs + np.asarray(p) % bs


READS = [
    # H, D, bs, lengths, requests (sequence, start, rows)
    (8, 128, 16, [300, 5, 77, 16], [(0, 0, 300), (2, 3, 70), (1, 0, 5)]),
    (4, 64, 32, [61, 517, 1, 40], [(1, 456, 61), (1, 0, 1), (2, 0, 1), (3, 7, 0), (0, 17, 13), (1, 400, 117)]),
    (1, 64, 512, [1000, 0, 0, 3], [(0, 999, 1), (3, 0, 3), (1, 0, 0), (0, 0, 1000)]),
    (3, 128, 64, [129, 64, 65, 1], [(0, 0, 0), (0, 0, 129), (1, 0, 64), (2, 64, 1), (3, 0, 1), (2, 0, 0)]),
    (2, 64, 16, [2000, 1, 1, 1], [(0, 5, 1990)]),
]


@pytest.mark.parametrize("dt", [E4, BF, F32], ids=str)
@pytest.mark.parametrize("case", range(len(READS)))
def test_read_matches_pages(case, dt):
    H, D, bs, lens, reqs = READS[case]
    c = filled(dt, H, D, bs, sum(-(-x // bs) for x in lens) + 1)
    table = with_sequences(c, lens, case)
    K, V = features(c)
    ids, start, rows = (np.array(x) for x in zip(*reqs))
    offs, total = np.concatenate([[0], np.cumsum(rows)]), int(rows.sum())
    at = np.concatenate([slots_of(table, bs, s, f + np.arange(m)) for s, f, m in reqs]).astype(np.int64)
    for shift in (0, 1):                                         # rows at any element, with more behind the last
        buf = torch.full((total + 3, 2 * H * D + 8), 7.0, dtype=c.row_dtype, device=dev())
        k_out, v_out = (buf[:, o:o + H * D].view(total + 3, H, D) for o in (shift, H * D + 8 - shift))
        say("read", dt, case, "shift", shift)
        sm.kv_read(c, i32(ids), i32(offs), k_out, v_out, start=i32(start))
        torch.cuda.synchronize()
        assert c.error_bits() == 0
        assert torch.equal(k_out[:total].double().cpu(), K[at]) and torch.equal(v_out[:total].double().cpu(), V[at])
        beside = torch.ones(2 * H * D + 8, dtype=torch.bool)
        beside[shift:shift + H * D] = beside[H * D + 8 - shift:2 * H * D + 8 - shift] = False
        assert bool((buf[total:] == 7).all()) and bool((buf[:, beside] == 7).all())
    one = torch.full((total, H, D), 7.0, dtype=c.row_dtype, device=dev())
    sm.kv_read(c, i32(ids), i32(offs), None, one, start=i32(start))
    assert torch.equal(one.double().cpu(), V[at])
    sm.kv_read(c, i32(ids), i32(offs), one, None, start=i32(start))
    assert torch.equal(one.double().cpu(), K[at])


def test_read_without_starts_and_of_nothing():
    c = filled(E4, 2, 64, 16, 9)
    table = with_sequences(c, [40, 17, 0, 1])
    K, V = features(c)
    out = torch.full((60, 2, 64), 7.0, dtype=BF, device=dev())
    sm.kv_read(c, i32([1, 2, 0]), i32([0, 17, 17, 57]), out, None)
    at = np.concatenate([slots_of(table, 16, 1, np.arange(17)), slots_of(table, 16, 0, np.arange(40))])
    assert torch.equal(out[:57].double().cpu(), K[at]) and bool((out[57:] == 7).all())
    sm.kv_read(c, i32([]), i32([0]), out, out)
    sm.kv_read(c, i32([1]), i32([0, 0]), out[:0], out[:0])
    torch.cuda.synchronize()
    assert c.error_bits() == 0


def test_read_refuses_row_by_row():
    """Bad ids and pages, entries outside a sequence: those rows are zero, the others come; the word says why."""
    c = filled(E4, 2, 64, 16, 9)
    table = with_sequences(c, [40, 17, 33, 1])
    K, V = features(c)

    def read(ids, start, rows, bits):
        offs = np.concatenate([[0], np.cumsum(rows)])
        k, v = (torch.full((offs[-1] + 1, 2, 64), 7.0, dtype=BF, device=dev()) for _ in range(2))
        sm.kv_read(c, i32(ids), i32(offs), k, v, start=i32(start))
        torch.cuda.synchronize()
        assert c.error_bits() == bits
        c.clear_error()
        assert bool((k[-1] == 7).all())
        return k[:-1].double().cpu(), v[:-1].double().cpu()
    k, v = read([0, 9, 1], [0, 0, 0], [40, 5, 17], sm.ERR_EINVAL)
    assert torch.equal(k[:40], K[slots_of(table, 16, 0, np.arange(40))]) and not k[40:45].any() and not v[40:45].any()
    assert torch.equal(v[45:], V[slots_of(table, 16, 1, np.arange(17))])
    k, v = read([2, 1], [-3, 10], [6, 9], sm.ERR_ERANGE)
    assert not k[:3].any() and torch.equal(k[3:6], K[slots_of(table, 16, 2, np.arange(3))])
    assert torch.equal(v[6:13], V[slots_of(table, 16, 1, np.arange(10, 17))]) and not v[13:].any()
    c.block_table[2, 1] = 9
    k, v = read([2], [0], [33], sm.ERR_EINVAL)
    assert not k[16:32].any() and torch.equal(k[:16], K[slots_of(table, 16, 2, np.arange(16))]) and k[32:].any()
    c.block_table[2, 1] = -1
    k, v = read([2], [0], [33], sm.ERR_EINVAL)
    assert not v[16:32].any() and v[:16].any()
    c.lengths[3] = 2 ** 31 - 1
    k, v = read([3], [2 ** 30], [3], sm.ERR_ERANGE)
    assert not k.any()
    for offs in ([0, 5, 4], [1, 5, 9], [0, 5, 11], [0, -1, 3]):  # not a row list: nothing is written
        out = torch.full((10, 2, 64), 7.0, dtype=BF, device=dev())
        sm.kv_read(c, i32([0, 1]), i32(offs), out, out)
        torch.cuda.synchronize()
        assert c.error_bits() == sm.ERR_EINVAL and bool((out == 7).all())
        c.clear_error()


def test_write_then_read_then_append_elsewhere():
    """A sequence written in 8 bits and moved into a bf16 cache: the same features, bit for bit."""
    kw = dict(num_kv_heads=2, head_dim=128, block_size=16, num_blocks=12, max_seqs=2, max_blocks_per_seq=6)
    a, b = sm.PagedCache(dtype=E4, **kw), sm.PagedCache(dtype=BF, **kw)
    n = 50
    k, v = _rand((n, 2, 128), BF, 1), _rand((n, 2, 128), BF, 2)
    ro, pos, slots = (torch.empty(m, dtype=torch.int32, device=dev()) for m in (3, n, n))
    sm.kv_reserve(a, i32([1, 0]), i32([20, 30]), ro, pos, slots)
    sm.kv_write_rotary(a, pos, slots, None, k, v, sm.rope_params(128), None)
    K, V = torch.empty_like(k), torch.empty_like(v)
    sm.kv_read(a, i32([1, 0]), ro, K, V)
    sm.kv_append(b, i32([1, 0]), ro, K, V)
    K2, V2 = torch.empty_like(k), torch.empty_like(v)
    sm.kv_read(b, i32([1, 0]), ro, K2, V2)
    torch.cuda.synchronize()
    assert a.error_bits() == 0 and b.error_bits() == 0
    assert torch.equal(K, K2) and torch.equal(V, V2)
    # each feature off by half a step: 2^-4 of itself, or 2^-17 of its row's largest
    for x, y in ((v, V),):
        tol = torch.maximum(x.abs().double() * 2 ** -4, x.abs().amax(-1, keepdim=True).double() * 2 ** -17)
        assert bool(((x.double() - y.double()).abs() <= tol).all())
    # a crop and another reservation move the tables as those of any cache
    sm.kv_rollback(a, i32([0, 1]), i32([14, 3]))
    torch.cuda.synchronize()
    assert a.lengths.tolist() == [16, 17] and int(a.free_top.item()) == 12 - 3 and a.error_bits() == 0


def test_eight_bit_pages_are_refused_elsewhere():
    c = sm.PagedCache(dtype=E4, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=4, max_seqs=2, max_blocks_per_seq=2)
    k = torch.zeros((1, 2, 64), dtype=BF, device=dev())
    q = torch.zeros((1, 4, 64), dtype=BF, device=dev())
    ws = torch.zeros(sm.decode_workspace_bytes(1, 4, 64, 32), dtype=torch.uint8, device=dev())
    for call in (lambda: sm.kv_append(c, i32([0]), i32([0, 1]), k, k), lambda: sm.decode_step(c, i32([0]), k, k, q, q, ws, 32),
                 lambda: sm.decode_merge_step(c, i32([0]), i32([0]), k, k, q, q, ws, 32),
                 lambda: sm.decode_step_noalloc(c, i32([0]), k, k, q, q, 32)):
        with pytest.raises(sm.SpanMergeError):
            call()
    with pytest.raises(sm.SpanMergeError, match="k: expected"):
        sm.kv_write_rotary(c, i32([0]), i32([0]), None, k.to(E4), k, sm.rope_params(64), None)
    with pytest.raises(sm.SpanMergeError, match="K: expected"):
        sm.kv_read(c, i32([0]), i32([0, 0]), k.to(E4), None)
