"""The calls around a backbone's projections beyond the sizes of their own
tests: offsets past 32 bits, other streams, a captured step."""
import math

import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm
from test_gpu_rotary import assert_near, turned

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _rand(shape, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, device=dev()).normal_(0, 1, generator=g).to(dt)


def test_pages_past_32_bits():
    """A cache of 140,000 pages of 16 x 8 x 128: 2.3 x 10^9 elements in each pool."""
    H, D, bs, nb = 8, 128, 16, 140_000
    c = sm.PagedCache(dtype=BF, num_kv_heads=H, head_dim=D, block_size=bs, num_blocks=nb, max_seqs=2, max_blocks_per_seq=8)
    n = 40
    ro, pos, slots = (torch.empty(m, dtype=torch.int32, device=dev()) for m in (2, n, n))
    say("large pools", c.k_pool.numel())
    # the stack hands out the last pages first when it is turned round
    c.free_stack.copy_(torch.arange(nb, dtype=torch.int32))
    sm.kv_reserve(c, i32([1]), i32([n]), ro, pos, slots)
    assert slots.tolist() == [(nb - 1 - j // bs) * bs + j % bs for j in range(n)]
    k, v = _rand((n, H, D), BF, 1), _rand((n, H, D), BF, 2)
    sm.kv_write_rotary(c, torch.zeros_like(pos), slots, None, k, v, sm.rope_params(D), None)
    torch.cuda.synchronize()
    assert c.error_bits() == 0
    for j in (0, 15, 16, 39):
        blk, s = nb - 1 - j // bs, j % bs
        assert torch.equal(c.k_pool[blk, :, s], k[j]) and torch.equal(c.v_pool[blk, :, :, s], v[j])
    assert int((c.k_pool[: nb - 3] != 0).any(-1).any(-1).any(-1).sum()) == 0


def test_rows_past_32_bits():
    rows, d = 600_000, 4096
    h = _rand((1, d), BF, 3).expand(rows, d).contiguous()                # 2.5 x 10^9 elements
    out = torch.empty_like(h)
    n = sm.norm_params("rms", None)
    say("large rows", h.numel())
    sm.block_norm(h, None, None, out, pre=n)
    assert torch.equal(out[0], out[rows - 1]) and torch.equal(out[0], out[rows // 2]) and float(out[0].abs().sum()) > 0
    x = out.view(rows, 32, 128)
    pos = torch.full((rows,), 77, dtype=torch.int32, device=dev())
    sm.rotary(x, pos, sm.rope_params(128), x)
    assert torch.equal(x[0], x[rows - 1]) and torch.equal(x[0], x[rows // 2])
    del x, out
    V = 128_256
    x = h.view(-1)[: 19_000 * V].view(19_000, V)
    lp, ent = torch.empty(19_000, device=dev()), torch.empty(19_000, device=dev())
    ids = torch.empty((19_000, 2), dtype=torch.int32, device=dev())
    ws = torch.zeros(sm.token_logprobs_workspace_bytes(19_000, V, 2), dtype=torch.uint8, device=dev())
    tok = torch.full((19_000,), V - 1, dtype=torch.int32, device=dev())
    sm.token_logprobs(x, tok, lp, ent, ids, None, ws)
    for r in (0, 16_743, 18_999):                                        # the middle one begins behind 2^31 elements
        z = x[r].double()
        assert abs(float(lp[r]) - float(torch.log_softmax(z, 0)[V - 1])) <= 1e-4
        assert int(ids[r, 0]) == int(torch.argmax(x[r].float()))


def test_rows_of_several_launches():
    """More rows than one launch has threads for (counted in 32 bits), or takes."""
    rows = (1 << 26) + 5                                     # 64 threads a row
    x = torch.zeros((rows, 1), dtype=torch.bfloat16, device=dev())
    lp = torch.full((rows,), -1.0, device=dev())
    ws = torch.zeros(sm.token_logprobs_workspace_bytes(rows, 1, 1), dtype=torch.uint8, device=dev())
    say("logprobs", rows)
    ids = torch.full((rows, 1), -1, dtype=torch.int32, device=dev())
    sm.token_logprobs(x, ids + 1, lp, None, ids, None, ws)
    assert not lp.any() and not ids.any()
    del x, lp, ids
    for rows, d in (((1 << 29) + 70, 1), ((1 << 21) + 33, 64)):  # 256 threads for 32 rows
        say("block_norm", rows, d)
        x = torch.ones((rows, d), dtype=torch.bfloat16, device=dev())
        x[rows - 2] = -3.0
        n = torch.zeros_like(x)
        sm.block_norm(x, None, None, n, pre=sm.norm_params("rms", eps=0.0))
        assert (n[:-2] == 1).all() and (n[-2] == -1).all() and (n[-1] == 1).all()
        del x, n
    rows = (1 << 28) + 70                                    # 256 threads for 16 rows
    say("rotary", rows)
    x = torch.ones((rows, 1, 2), dtype=torch.bfloat16, device=dev())
    pos = torch.zeros(rows, dtype=torch.int32, device=dev())
    p = sm.rope_params(2)
    pos[-1] = 1
    out = torch.zeros_like(x)
    sm.rotary(x, pos, p, out)
    turn = torch.tensor([math.cos(1) - math.sin(1), math.cos(1) + math.sin(1)]).bfloat16().to(dev())
    assert (out[:-1] == 1).all() and torch.equal(out[-1, 0], turn)
    del x, out, pos
    rows = (1 << 24) + 21                                    # the last 22 rows have slots
    say("write", rows)
    c = sm.PagedCache(dtype=torch.bfloat16, num_kv_heads=1, head_dim=64, block_size=16, num_blocks=4, max_seqs=1,
                      max_blocks_per_seq=4)
    slots = torch.full((rows,), -1, dtype=torch.int32, device=dev())
    slots[-22:] = torch.arange(7, 29, dtype=torch.int32, device=dev())
    k = torch.zeros((rows, 1, 64), dtype=torch.bfloat16, device=dev())
    k[-22:] = torch.arange(1.0, 23.0, device=dev())[:, None, None].bfloat16()
    sm.kv_write_rotary(c, torch.zeros_like(slots), slots, None, k, k, sm.rope_params(64), None)
    got_k = c.k_pool[:2, 0].reshape(32, 64)
    got_v = c.v_pool[:2, 0].transpose(1, 2).reshape(32, 64)
    want = torch.zeros((32, 64), device=dev())
    want[7:29] = torch.arange(1.0, 23.0, device=dev())[:, None]
    assert torch.equal(got_k.float(), want) and torch.equal(got_v.float(), want) and c.error_bits() == 0


def test_host_tensors_are_refused():
    x, pos, rope = _rand((3, 2, 8), BF, 1), i32([0, 1, 2]), sm.rope_params(8)
    out = torch.empty_like(x)
    for pinned in (False, True):
        host = torch.zeros((3, 2, 8), dtype=BF, pin_memory=pinned)
        host_pos = torch.zeros(3, dtype=torch.int32, pin_memory=pinned)
        for bad in ((host, pos, out), (x, host_pos, out), (x, pos, host)):
            with pytest.raises(sm.SpanMergeError, match="current device"):
                sm.rotary(bad[0], bad[1], rope, bad[2])
        gain = torch.ones(8, dtype=BF, pin_memory=pinned)
        with pytest.raises(sm.SpanMergeError, match="pre: expected"):
            sm.block_norm(x[:, 0], None, None, out[:, 0], pre=sm.norm_params("rms", gain))


def test_other_streams():
    """Each call on a stream of its own, beside work on the current one."""
    side = torch.cuda.Stream()
    x, big = _rand((3000, 8, 64), BF, 1), _rand((4096, 4096), F32, 2)
    pos, rope = torch.arange(3000, dtype=torch.int32, device=dev()), sm.rope_params(64)
    want, got = torch.empty_like(x), torch.zeros_like(x)
    logits, ids, got_ids = _rand((9, 40_000), BF, 5), *(torch.zeros((9, 4), dtype=torch.int32, device=dev()) for _ in range(2))
    ws = [torch.zeros(sm.token_logprobs_workspace_bytes(9, 40_000, 4), dtype=torch.uint8, device=dev()) for _ in range(2)]
    n = sm.norm_params("rms", None)
    h, a, b = _rand((500, 512), BF, 3), *(torch.zeros((500, 512), dtype=BF, device=dev()) for _ in range(2))
    sm.rotary(x, pos, rope, want)
    sm.block_norm(h, h, None, a, pre=n)
    sm.token_logprobs(logits, None, None, None, ids, None, ws[0])
    torch.cuda.synchronize()
    for _ in range(5):
        big @ big
    side.wait_stream(torch.cuda.current_stream())
    sm.rotary(x, pos, rope, got, stream=side)
    sm.block_norm(h, h, None, b, pre=n, stream=side)
    sm.token_logprobs(logits, None, None, None, got_ids, None, ws[1], stream=side)
    side.synchronize()
    assert torch.equal(want, got) and torch.equal(a, b) and torch.equal(ids, got_ids)


def test_captured_decode_step():
    """A step's calls in one graph (padded to a fixed number of rows), its inputs and counts changed between replays,
    against the same calls one by one on a twin cache."""
    H, Hq, D, bs, n, room, V = 2, 8, 64, 16, 5, 9, 5000
    rng = np.random.RandomState(3)
    order = rng.permutation(60)
    kw = dict(dtype=BF, num_kv_heads=H, head_dim=D, block_size=bs, num_blocks=60, max_seqs=n, max_blocks_per_seq=12,
              free_order=order)
    rope, norm = sm.rope_params(D, scaling="linear", factor=2.0), sm.norm_params("rms", _rand((512,), BF, 9))
    head = _rand((512, V), F32, 10) * 0.05
    ids = i32(rng.permutation(n))

    class Side:
        def __init__(self):
            self.c = sm.PagedCache(**kw)
            e = lambda *s, dt=BF: torch.zeros(s, dtype=dt, device=dev())             # noqa: E731
            self.ro, self.pos, self.slots = e(n + 1, dt=torch.int32), e(room, dt=torch.int32), e(room, dt=torch.int32)
            self.qkv, self.q_out, self.att = e(room, (Hq + 2 * H) * D), e(room, Hq, D), e(room, Hq, D)
            self.h, self.nrm, self.crop, self.rows = e(room, 512), e(room, 512), e(n, dt=torch.int32), e(n, dt=torch.int32)
            self.ws = torch.zeros(sm.decode_workspace_bytes(n, Hq, D, 192), dtype=torch.uint8, device=dev())
            self.lws = torch.zeros(sm.token_logprobs_workspace_bytes(n, V, 3), dtype=torch.uint8, device=dev())
            self.top, self.ent = e(n, 3, dt=torch.int32), e(n, dt=F32)

        def step(self):
            sm.kv_reserve(self.c, ids, self.rows, self.ro, self.pos, self.slots, crop=self.crop)
            q, k, v = (t.unflatten(1, (-1, D)) for t in self.qkv.split([Hq * D, H * D, H * D], 1))
            sm.kv_write_rotary(self.c, self.pos, self.slots, q, k, v, rope, self.q_out)
            sm.decode_attention(self.c, ids, self.q_out[:n], self.att[:n], self.ws, 192)
            sm.block_norm(self.h, self.att.flatten(1), self.h, self.nrm, scale=0.5, pre=norm)
            sm.token_logprobs(self.nrm[:n].float() @ head, None, None, self.ent, self.top, None, self.lws)

        def state(self):
            return [self.ro, self.pos, self.slots, self.q_out, self.att[:n], self.h[:n], self.nrm[:n], self.top, self.ent,
                    self.c.k_pool, self.c.v_pool, self.c.block_table, self.c.lengths, self.c.free_top]

    a, b = Side(), Side()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.step()                                                          # (no rows: the caches stay empty)
    a.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        b.step()
    for rep in range(8):
        crop = np.minimum(rng.randint(0, 3, n), a.c.lengths.cpu().numpy()[ids.cpu().numpy()])
        rows = np.ones(n, int) if rep % 2 else rng.randint(1, 3, n).clip(max=1 + (rep == 0))
        rows = rows if rows.sum() <= room else np.ones(n, int)
        for s in (a, b):
            s.crop.copy_(i32(crop))
            s.rows.copy_(i32(rows))
            s.qkv.copy_(_rand(s.qkv.shape, BF, 100 + rep))
            s.h.copy_(_rand(s.h.shape, BF, 200 + rep))
        say("replay", rep)
        a.step()
        g.replay()
        torch.cuda.synchronize()
        assert a.c.error_bits() == 0 and b.c.error_bits() == 0
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)


def test_rows_past_32_bits_match_the_formula():
    """Rows on both sides of 2^31 elements and the last ones, against the formula in 64 bits; the others are zeros."""
    rows, d = 600_000, 4096                                              # 2.5 x 10^9 elements
    first = (1 << 31) // d
    some = torch.cat([torch.arange(3), torch.arange(first - 3, first + 4), torch.arange(rows - 5, rows)]).to(dev())
    h = torch.zeros((rows, d), dtype=BF, device=dev())
    h[some] = _rand((some.numel(), d), BF, 11)
    out = torch.full_like(h, 7.0)
    say("far rows", h.numel())
    sm.block_norm(h, None, None, out, pre=sm.norm_params("rms", None))
    x = h[some].double()
    want = x / (x.square().mean(1, keepdim=True) + float(np.float32(1e-5))).sqrt()
    got = out[some].double()
    # 40 additions of the mean square, halved by the root, with that, the mean and the product: 26 x 2^-24; then half a step
    assert ((got - want).abs() <= want.abs() * (26 * 2.0 ** -24 + 2.0 ** -8)).all()
    out[some] = 0
    assert not out.any()
    pos = torch.zeros(rows, dtype=torch.int32, device=dev())
    pos[some] = torch.arange(some.numel(), dtype=torch.int32, device=dev()) * 1013
    x = h.view(rows, 32, 128)
    want, slack = turned(x[some], pos[some], dict(rot_dim=128))
    sm.rotary(x, pos, sm.rope_params(128), out.view(rows, 32, 128))
    assert_near(out[some].view(-1, 32, 128), want, slack, BF)
    out[some] = 0
    assert not out.any()
