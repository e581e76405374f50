"""The serving calls together as a decoder uses them: room in the cache, entries
turned and written, prompts, requests behind a shared prefix, tokens drawn, a
crop, entries read back; captured, on other streams and far into a large pool."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm
from test_gpu_e4m3_attention import assert_within, attended
from test_gpu_e4m3_write import BF, E4, F32, features, filled, slots_of
from test_gpu_rotary import _rand
from test_gpu_sample import check_row, f32

pytestmark = pytest.mark.gpu

HQ, H, D, BS, VOCAB = 8, 2, 64, 16, 600
PREFIX, PROMPTS = 150, [40, 1, 33, 90, 16]       # sequence 0, and requests 1 ..
GROUPS, OFFS = [0, -1], [0, 3, 5]                # three behind the prefix, two on their own
ROPE = dict(theta=10000.0)


def to_ints(*shape):
    return torch.empty(shape, dtype=torch.int32, device=dev())


def fresh(dt, nb=60, blocks=None):
    """A cache whose free pages are `blocks`, the last first."""
    c = sm.PagedCache(dtype=dt, num_kv_heads=H, head_dim=D, block_size=BS, num_blocks=nb, max_seqs=6, max_blocks_per_seq=16)
    if blocks is not None:
        c.free_stack[:len(blocks)] = i32(blocks)
        c.free_top.fill_(len(blocks))
    return c


class Run:
    """A decoder's layer over one cache; tables of rows stand for its products."""

    def __init__(self, c):
        self.c, self.n = c, len(PROMPTS)
        self.q, self.k, self.v = (_rand((VOCAB, h, D), BF, s).to(dev()) for s, h in ((1, HQ), (2, H), (3, H)))
        self.W = _rand((HQ * D, VOCAB), F32, 4).cpu()
        self.rope = sm.rope_params(D, **ROPE)
        self.ids = i32(range(1, self.n + 1))
        self.ws = torch.zeros(sm.decode_shared_workspace_bytes(self.n, HQ, D, 256, 256), dtype=torch.uint8, device=dev())
        self.sample_ws = torch.zeros(sm.sample_workspace_bytes(self.n, VOCAB), dtype=torch.uint8, device=dev())

    def rows(self, ids, counts, tokens, before, crop=None):
        """Room for the tokens' entries, written: (row offsets, turned queries)."""
        total = len(tokens)
        offs, pos, slots = to_ints(len(counts) + 1), to_ints(total), to_ints(total)
        sm.kv_reserve(self.c, ids, i32(counts), offs, pos, slots, crop=crop)
        pos += before
        t = tokens.long()
        q = torch.empty((total, HQ, D), dtype=BF, device=dev())
        sm.kv_write_rotary(self.c, pos, slots, self.q[t], self.k[t], self.v[t], self.rope, q)
        return offs, q

    def prompt(self, ids, counts, tokens):
        offs, q = self.rows(ids, counts, tokens, 0)
        out = torch.empty_like(q)
        sm.prefill_attention(self.c, ids, offs, q, out, max(counts))
        return q, out

    def step(self, tokens, u, before, crop=None):
        """One token for each request: attention, and the next ones drawn."""
        _, q = self.rows(self.ids, [1] * self.n, tokens, before, crop)
        out = torch.empty_like(q)
        sm.decode_attention_shared(self.c, self.ids, i32(GROUPS), i32(OFFS), q, out, self.ws, 256, 256)
        logits = (out.flatten(1).float().cpu() @ self.W).to(BF).to(dev())
        drawn, logprob = to_ints(self.n), torch.empty(self.n, device=dev())
        err = torch.zeros(1, dtype=torch.int32, device=dev())
        sm.sample_tokens(logits, u, drawn, self.sample_ws, temperature=f32([0.7] * self.n), top_k=i32([40] * self.n),
                         top_p=f32([0.9] * self.n), logprob=logprob, err=err)
        assert int(err.item()) == 0
        return q, out, logits, drawn, logprob


def serve(c, look=None):
    """Every output of a run, in order; look(run, kind, q, out) after each attention."""
    run, rng = Run(c), np.random.RandomState(5)
    got = []
    tokens = i32(rng.randint(0, VOCAB, PREFIX))
    got += run.prompt(i32([0]), [PREFIX], tokens)
    look and look(run, "prefix", *got[-2:])
    tokens = i32(rng.randint(0, VOCAB, sum(PROMPTS)))
    got += run.prompt(run.ids, PROMPTS, tokens)
    look and look(run, "prompts", *got[-2:])
    tokens = i32(rng.randint(0, VOCAB, run.n))
    before = i32([PREFIX] * OFFS[1] + [0] * (run.n - OFFS[1]))
    for step in range(4):
        u = rng.uniform(size=run.n)
        crop = i32([0, 0, 3, 1, 0]) if step == 2 else None       # a span's entries go, the merged one's comes
        res = run.step(tokens, f32(u), before, crop)
        if look:
            look(run, "step", *res[:2])
            for r in range(run.n):
                check_row(res[2][r].double().cpu().numpy(), float(np.float32(0.7)), 40, float(np.float32(0.9)), 0.0,
                          float(np.float32(u[r])), int(res[3][r]), float(res[4][r]))
        got += res
        tokens = res[3]
    lens = c.lengths.cpu().numpy()
    offs = np.concatenate([[0], np.cumsum(lens)])
    K, V = (torch.full((int(offs[-1]), H, D), 5.0, dtype=BF, device=dev()) for _ in "KV")
    sm.kv_read(c, i32(range(6)), i32(offs), K, V)
    torch.cuda.synchronize()
    assert c.error_bits() == 0 and lens.tolist() == [PREFIX] + [p + 4 - x for p, x in zip(PROMPTS, (0, 0, 3, 1, 0))]
    return got + [K, V]


@pytest.mark.parametrize("dt", [E4, BF], ids=str)
def test_a_run_of_the_calls(dt):
    c = fresh(dt)

    def look(run, kind, q, out):
        torch.cuda.synchronize()
        K, V = features(c)
        table, lens = c.block_table.cpu().numpy(), c.lengths.cpu().numpy()
        at = [slots_of(table, BS, s, np.arange(lens[s])) for s in range(6)]
        q = q.double().cpu()
        if kind == "step":
            for i in range(run.n):
                s = np.concatenate([at[0], at[i + 1]]) if i < OFFS[1] else at[i + 1]
                assert_within(out[i:i + 1], *attended(q[i:i + 1], K[s], V[s], D ** -0.5))
            return
        r = 0
        for s in [0] if kind == "prefix" else range(1, run.n + 1):
            m = int(lens[s])
            seen = torch.ones((m, m), dtype=torch.bool).tril()
            assert_within(out[r:r + m], *attended(q[r:r + m], K[at[s]], V[at[s]], D ** -0.5, seen))
            r += m
    say("serving run", dt)
    got = serve(c, look)
    K, V = features(c)
    table, lens = c.block_table.cpu().numpy(), c.lengths.cpu().numpy()
    s = np.concatenate([slots_of(table, BS, i, np.arange(lens[i])) for i in range(6)])
    assert torch.equal(got[-2].double().cpu(), K[s]) and torch.equal(got[-1].double().cpu(), V[s])
    for a, b in zip(got, serve(fresh(dt))):                      # and the same bits again
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [E4, BF], ids=str)
def test_far_into_a_large_pool(dt):
    """Pages whose elements lie behind 2^31 and 2^32 give what the first pages give."""
    small = list(range(60))
    nb = 2 ** 32 // (H * BS * D) + 64
    half = 2 ** 31 // (H * BS * D)
    far = [half - 3 + i if i % 2 else nb - 1 - i for i in small]
    want = serve(fresh(dt, 60, small))
    say("large pool", dt, nb, "pages")
    c = fresh(dt, nb, far)
    for a, b in zip(want, serve(c)):
        assert torch.equal(a, b)
    used = c.block_table[c.block_table >= 0].cpu().numpy()
    assert int(used.max()) * H * BS * D > 2 ** 32 - 2 ** 20


def test_rows_read_and_drawn_behind_the_first_two_gibielements():
    c = filled(E4, 2, 64, 16, 40)
    c.block_table[0, :20] = i32(range(20))
    c.lengths[0] = 320
    stride = 2 ** 31 // 300 + 77
    big = torch.empty(300 * stride + 128, dtype=BF, device=dev())
    K = big.as_strided((300, 2, 64), (stride, 64, 1))
    plain = torch.empty((300, 2, 64), dtype=BF, device=dev())
    say("wide read", stride)
    for out in (K, plain):
        sm.kv_read(c, i32([0]), i32([0, 300]), out, None, start=i32([9]))
    torch.cuda.synchronize()
    assert c.error_bits() == 0 and torch.equal(K, plain)
    x = big.as_strided((300, 999), (stride, 1))
    x.copy_(2 * _rand((300, 999), BF, 3))
    tokens = [to_ints(300) for _ in range(2)]
    ws = torch.zeros(sm.sample_workspace_bytes(300, 999), dtype=torch.uint8, device=dev())
    u, p = f32(np.random.RandomState(1).uniform(size=300)), f32([0.8] * 300)
    say("wide logits")
    for t, rows in zip(tokens, (x, x.contiguous())):
        sm.sample_tokens(rows, u, t, ws, top_p=p)
    torch.cuda.synchronize()
    assert torch.equal(*tokens) and int(tokens[0].min()) >= 0


class Step:
    """A decoder's step over fixed buffers: both attentions, a prompt row's, the last entries read, tokens drawn."""

    def __init__(self, ws=None):
        self.n, self.rope = 5, sm.rope_params(D, **ROPE)
        self.c = fresh(E4)
        run = Run(self.c)
        rng = np.random.RandomState(7)
        run.prompt(i32([0]), [PREFIX], i32(rng.randint(0, VOCAB, PREFIX)))
        run.prompt(run.ids, PROMPTS, i32(rng.randint(0, VOCAB, sum(PROMPTS))))
        self.ids, self.one, self.start = run.ids, i32([1] * 5), self.c.lengths[1:].clone()
        self.offs, self.pos, self.slots = to_ints(6), to_ints(5), to_ints(5)
        self.q, self.k, self.v = (torch.empty((5, h, D), dtype=BF, device=dev()) for h in (HQ, H, H))
        self.logits, self.u = torch.empty((5, VOCAB), dtype=BF, device=dev()), torch.empty(5, device=dev())
        self.prefixes, self.groups = i32(GROUPS), i32(OFFS)
        self.T, self.kk, self.p = f32([0.8, 0, 1, 1, 2]), i32([0, 0, 30, 0, 100]), f32([0.9, 1, 1, 0.5, 0.95])
        self.out = [torch.empty((5, HQ, D), dtype=BF, device=dev()) for _ in range(4)]
        self.read = [torch.empty((5, H, D), dtype=BF, device=dev()) for _ in range(2)]
        self.tokens, self.logprob = to_ints(5), torch.empty(5, device=dev())
        sizes = (sm.decode_workspace_bytes(5, HQ, D, 256), sm.decode_shared_workspace_bytes(5, HQ, D, 256, 256),
                 sm.sample_workspace_bytes(5, VOCAB))
        self.ws = ws or [torch.zeros(b, dtype=torch.uint8, device=dev()) for b in sizes]
        torch.cuda.synchronize()

    def load(self, seed):
        for i, (t, s) in enumerate(((self.q, 1), (self.k, 1), (self.v, 1), (self.logits, 2))):
            t.copy_(s * _rand(t.shape, BF, 10 * seed + i))
        self.u.copy_(f32(np.random.RandomState(seed).uniform(size=5)))

    def __call__(self):
        turned, decoded, shared, pre = self.out
        sm.kv_reserve(self.c, self.ids, self.one, self.offs, self.pos, self.slots)
        sm.kv_write_rotary(self.c, self.pos, self.slots, self.q, self.k, self.v, self.rope, turned)
        sm.decode_attention(self.c, self.ids, turned, decoded, self.ws[0], 256)
        sm.decode_attention_shared(self.c, self.ids, self.prefixes, self.groups, turned, shared, self.ws[1], 256, 256)
        sm.prefill_attention(self.c, self.ids, self.offs, turned, pre, 1)
        sm.kv_read(self.c, self.ids, self.offs, *self.read, start=self.start)
        sm.sample_tokens(self.logits, self.u, self.tokens, self.ws[2], temperature=self.T, top_k=self.kk, top_p=self.p,
                         logprob=self.logprob)

    def results(self):
        torch.cuda.synchronize()
        assert self.c.error_bits() == 0
        pools = [t.clone() for t in (self.c.k_pool.view(torch.uint8), self.c.v_pool.view(torch.uint8), self.c.k_exp, self.c.v_exp)]
        return [t.clone() for t in self.out + self.read + [self.tokens, self.logprob, self.c.lengths]] + pools


def captured(step, stream):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        step()
    return g


def test_captured_and_replayed():
    """Replays with other inputs and eager work between; two graphs that share their workspaces."""
    stream = torch.cuda.Stream()
    eager = [Step(), Step()]
    first = Step()
    graphed = [first, Step(ws=first.ws)]
    for s in eager + graphed:
        s.load(99)
    torch.cuda.synchronize()
    graphs = [captured(s, stream) for s in graphed]
    for i in range(5):
        for e, s, g in zip(eager, graphed, graphs):
            say("replay", i)
            e.load(2 * i + (s is first))
            s.load(2 * i + (s is first))
            g.replay()
            e()
            for a, b in zip(s.results(), e.results()):
                assert torch.equal(a, b)
        torch.randn(1000, device=dev()).sum().item()             # eager work between the replays


def test_two_streams_at_once():
    steps, alone = [Step(), Step()], [Step(), Step()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, s in enumerate(steps):
        s.load(i)
        alone[i].load(i)
    torch.cuda.synchronize()
    say("two streams")
    for _ in range(10):
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s()
    torch.cuda.synchronize()
    for _ in range(10):
        for s in alone:
            s()
    for s, a in zip(steps, alone):
        for x, y in zip(s.results(), a.results()):
            assert torch.equal(x, y)


def test_the_same_sequence_more_than_once():
    """A sequence listed twice is read twice, by every call that reads."""
    s = Step()
    s.load(3)
    s()
    s.results()
    ids, q, ws = i32([2, 2, 4]), s.out[0][:3].contiguous(), s.ws
    q[1] = q[0]
    dec, sh, pre = (torch.empty_like(q) for _ in range(3))
    say("the same twice")
    sm.decode_attention(s.c, ids, q, dec, ws[0], 256)
    sm.decode_attention_shared(s.c, ids, i32([2, 2]), i32([0, 2, 3]), q, sh, ws[1], 256, 256)
    sm.prefill_attention(s.c, ids, i32([0, 1, 2, 3]), q, pre, 1)
    K, V = (torch.empty((6, H, D), dtype=BF, device=dev()) for _ in "KV")
    sm.kv_read(s.c, ids, i32([0, 2, 4, 6]), K, V)
    torch.cuda.synchronize()
    assert s.c.error_bits() == 0
    for out in (dec, sh, pre):
        assert torch.equal(out[0], out[1])
    assert torch.equal(K[:2], K[2:4]) and torch.equal(V[:2], V[2:4])
    # behind itself as a prefix a sequence's entries count twice: the same weights, the same mean
    Kf, Vf = features(s.c)
    at = slots_of(s.c.block_table.cpu().numpy(), BS, 2, np.arange(int(s.c.lengths[2])))
    at = np.concatenate([at, at])
    assert_within(sh[:1], *attended(q[:1].double().cpu(), Kf[at], Vf[at], D ** -0.5))


def test_layers_of_both_page_types_share_their_tables():
    """One reservation a step for a bf16 layer and an 8-bit one of other head counts; a span's crop moves both."""
    kw = dict(head_dim=D, block_size=BS, num_blocks=20, max_seqs=3, max_blocks_per_seq=8)
    a = sm.PagedCache(dtype=BF, num_kv_heads=2, **kw)
    b = sm.PagedCache(dtype=E4, num_kv_heads=1, tables=a, **kw)
    rng, ids, rope = np.random.RandomState(6), i32([2, 0]), sm.rope_params(D, **ROPE)
    ws = torch.zeros(sm.decode_workspace_bytes(2, 4, D, 128), dtype=torch.uint8, device=dev())
    say("both page types")
    for counts, crop in (([30, 17], [0, 0]), ([1, 1], [0, 0]), ([1, 2], [3, 0]), ([1, 0], [2, 17])):
        total = sum(counts)
        offs, pos, slots = to_ints(3), to_ints(total), to_ints(total)
        sm.kv_reserve(a, ids, i32(counts), offs, pos, slots, crop=i32(crop))
        for c in (a, b):
            k, v = (_rand((total, c.H, D), BF, int(rng.randint(1000))).to(dev()) for _ in "kv")
            sm.kv_write_rotary(c, pos, slots, None, k, v, rope, None)
    sm.kv_rollback(a, i32([0]), i32([1]))
    torch.cuda.synchronize()
    lens = a.lengths.cpu().numpy()
    assert lens.tolist() == [17 + 1 + 2 - 17 - 1, 0, 30 + 1 - 3 + 1 - 2 + 1]
    table = a.block_table.cpu().numpy()
    assert a.error_bits() == 0 and torch.equal(a.lengths, b.lengths)
    q = _rand((2, 4, D), BF, 9).to(dev())
    for c in (a, b):
        out = torch.empty_like(q)
        sm.decode_attention(c, ids, q, out, ws, 128)
        torch.cuda.synchronize()
        K, V = features(c)
        for i, s in enumerate((2, 0)):
            at = slots_of(table, BS, s, np.arange(lens[s]))
            assert_within(out[i:i + 1], *attended(q[i:i + 1].double().cpu(), K[at], V[at], D ** -0.5))
    assert a.error_bits() == 0
