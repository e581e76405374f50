"""A small backbone of two layers served through the library: prompt, decode
steps and decode-time merges, with the calls around its projections (norms,
reserved rows, rotated K/V writes, token log probabilities) beside the ones
they feed (attention over pages, rule check, surrogate rows).  Compared with
the same backbone in 64 bits over plain lists of K and V rows, fed the same
tokens."""
import math

import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm

pytestmark = pytest.mark.gpu

d, Hq, H, D, VOCAB, LAYERS, BS, NSEQ = 256, 4, 2, 64, 600, 2, 16, 3
ROPE = dict(rot_dim=48, theta=10000.0, layout="half", scaling="bands", factor=4.0, low=1.0, high=4.0, context=64)
EPS = 1e-5


class Weights:
    def __init__(self, dt, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0, mean=0.0: (torch.randn(s, generator=g) * std + mean).to(dt)   # noqa: E731
        self.emb, self.lut = r(VOCAB, d), r(40, d)
        self.layers = [dict(g1=r(d, std=0.1, mean=1.0), g2=r(d, std=0.1, mean=1.0), gate=r(d, std=0.1, mean=0.8),
                            qkv=r((Hq + 2 * H) * D, d, std=d ** -0.5), o=r(d, Hq * D, std=(Hq * D) ** -0.5))
                       for _ in range(LAYERS)]
        self.g_out, self.head = r(d, std=0.1, mean=1.0), r(VOCAB, d, std=2 * d ** -0.5)


class Plain:
    """The backbone in 64 bits: a list of K and V rows per layer and sequence."""

    def __init__(self, w):
        self.w = w
        self.kv = [[[] for _ in range(NSEQ)] for _ in range(LAYERS)]
        j = torch.arange(24, dtype=torch.float64)
        f = 10000.0 ** (-2 * j / 48)
        u = ((64 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
        self.f = u * f + (1 - u) * f / 4

    def norm(self, x, g):
        return x / (x.square().mean() + EPS).sqrt() * g.double()

    def turn(self, x, p):
        c, s, y = (p * self.f).cos(), (p * self.f).sin(), x.clone()
        u, v = x[:, :24], x[:, 24:48]
        y[:, :24], y[:, 24:48] = u * c - v * s, u * s + v * c
        return y

    def row(self, s, x):
        """One input row at the end of sequence s: its logits."""
        w = self.w
        for l, m in enumerate(w.layers):
            kv = self.kv[l][s]
            q, k, v = (m["qkv"].double() @ self.norm(x, m["g1"])).view(-1, D).split([Hq, H, H])
            p = len(kv)
            kv.append((self.turn(k, p), v))
            q = self.turn(q, p)
            K, V = torch.stack([a for a, _ in kv]), torch.stack([b for _, b in kv])
            out = [torch.softmax(K[:, h // (Hq // H)] @ q[h] * D ** -0.5, 0) @ V[:, h // (Hq // H)] for h in range(Hq)]
            y = m["o"].double() @ torch.cat(out)
            x = x + 0.5 * m["gate"].double() * self.norm(y, m["g2"])
        return w.head.double() @ self.norm(x, w.g_out)

    def crop(self, s, n):
        for l in range(LAYERS):
            if n:
                del self.kv[l][s][-n:]


class Served:
    """The same through the library."""

    def __init__(self, w, dt):
        self.dt = dt
        self.w = w
        self.g = lambda t: t.to(dev())                                        # noqa: E731
        kw = dict(dtype=dt, num_kv_heads=H, head_dim=D, block_size=BS, num_blocks=40, max_seqs=NSEQ + 1, max_blocks_per_seq=12)
        first = sm.PagedCache(**kw, free_order=np.random.RandomState(1).permutation(40))
        self.caches = [first] + [sm.PagedCache(**kw, tables=first) for _ in range(LAYERS - 1)]
        self.rope = sm.rope_params(**ROPE)
        self.layers = [dict(pre=sm.norm_params("rms", self.g(m["g1"]), eps=EPS), post=sm.norm_params("rms", self.g(m["g2"]), eps=EPS),
                            gate=self.g(m["gate"]), qkv=self.g(m["qkv"]).float(), o=self.g(m["o"]).float()) for m in w.layers]
        self.out_norm, self.head = sm.norm_params("rms", self.g(w.g_out), eps=EPS), self.g(w.head).float()
        self.ws = torch.zeros(sm.decode_workspace_bytes(NSEQ, Hq, D, 192), dtype=torch.uint8, device=dev())

    def rows(self, ids, crop, counts, x, prompt):
        """Input rows x of the listed sequences (all of them counts[i] long): their logits."""
        n, room = len(ids), x.shape[0] + 3                                     # (a padded batch)
        e = lambda *s, dt=self.dt: torch.empty(s, dtype=dt, device=dev())      # noqa: E731
        ro, pos, slots = e(n + 1, dt=torch.int32), e(room, dt=torch.int32), e(room, dt=torch.int32)
        t_ids = i32(ids)
        sm.kv_reserve(self.caches[0], t_ids, i32(counts), ro, pos, slots, crop=None if crop is None else i32(crop))
        h = torch.zeros((room, d), dtype=self.dt, device=dev())
        h[:x.shape[0]] = x
        y, nrm = None, torch.empty_like(h)
        post = gate = None
        for c, m in zip(self.caches, self.layers):
            sm.block_norm(h, y, h, nrm, post=post, gate=gate, scale=0.5, pre=m["pre"])
            qkv = (nrm.float() @ m["qkv"].t()).to(self.dt)
            q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, H * D, H * D], 1))
            q_out, att = e(room, Hq, D), torch.zeros((room, Hq, D), dtype=self.dt, device=dev())
            sm.kv_write_rotary(c, pos, slots, q, k, v, self.rope, q_out)
            if prompt:
                sm.prefill_attention(c, t_ids, ro, q_out, att, max(counts))
            else:
                sm.decode_attention(c, t_ids, q_out[:n], att[:n], self.ws, 192)
            y = (att.flatten(1).float() @ m["o"].t()).to(self.dt)
            post, gate = m["post"], m["gate"]
        sm.block_norm(h, y, h, nrm, post=post, gate=gate, scale=0.5, pre=self.out_norm)
        return (nrm[:x.shape[0]].float() @ self.head.t()).to(self.dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=str)
def test_prompt_then_merging_decode(dt):
    w = Weights(dt, 7)
    plain, served = Plain(w), Served(w, dt)
    rng = np.random.RandomState(2)
    emb, lut = w.emb.to(dev()), w.lut.to(dev())
    # Rounding to bf16 between the stages: 8 roundings a layer (norm, projection, turned rows, probabilities, attention,
    # output projection, sum, and the weights' products of them) and 3 behind, each at most 2^-8 of its row:
    # (2 x 8 + 3) x 2^-8.  In fp32 the attention's own sums, at 1e-5 a layer, and the norms lead.
    tol = 19 * 2.0 ** -8 if dt == torch.bfloat16 else 1e-4
    lens = [21, 1, 40]
    prompts = [rng.randint(0, VOCAB, n) for n in lens]
    worst = 0.0

    def compare(logits, want):
        nonlocal worst
        ref = torch.stack(want)
        worst = max(worst, float(((logits.double().cpu() - ref).norm(dim=1) / ref.norm(dim=1)).max()))
        assert worst <= tol, worst

    # the prompts (fp32 caches have no prefill: a row of each sequence at a time)
    say("prompt", dt)
    if dt == torch.bfloat16:
        tokens = np.concatenate(prompts)
        got = served.rows([0, 1, 2], None, lens, emb[torch.from_numpy(tokens).to(dev())], True)
        compare(got, [plain.row(s, w.emb[t].double()) for s in range(3) for t in prompts[s]])
        last = got[torch.tensor([20, 21, 61], device=dev())]
    else:
        rows_of = {}
        for t in range(max(lens)):
            ids = [s for s in (2, 0, 1) if t < lens[s]]
            got = served.rows(ids, None, [1] * len(ids), emb[[int(prompts[s][t]) for s in ids]], False)
            compare(got, [plain.row(s, w.emb[int(prompts[s][t])].double()) for s in ids])
            rows_of.update({s: got[i] for i, s in enumerate(ids)})
        last = torch.stack([rows_of[s] for s in range(3)])

    # rules: pairs and triples that the sequences are then led through now and then
    rules = [(10, 11, -1, -1), (12, 13, 14, -1), (20, 21, 22, 23), (11, 12, -1, -1)]
    table = sm.RuleTable(16)
    sm.rules_build(table, i32(rules))
    state = torch.zeros((NSEQ + 1, 4), dtype=torch.int32, device=dev())
    script = {2: [10, None, 20], 3: [11, None, 21], 4: [12, 12, 22], 5: [13, 13, 23], 6: [14, 14, None]}
    ids = [0, 1, 2]
    ws = torch.zeros(sm.token_logprobs_workspace_bytes(3, VOCAB, 4), dtype=torch.uint8, device=dev())
    length = list(lens)
    merges = 0
    for step in range(9):
        say("step", step)
        f = lambda *s: torch.empty(s, device=dev())                            # noqa: E731
        top, top_lp, ent = torch.empty((3, 4), dtype=torch.int32, device=dev()), f(3, 4), f(3)
        sm.token_logprobs(last, None, None, ent, top, top_lp, ws)
        logp = torch.log_softmax(last.double(), 1)
        assert torch.equal(top[:, 0].long(), last.float().argmax(1))
        assert float((top_lp.double() - logp.gather(1, top.long())).abs().max()) <= 1e-5
        assert float((ent.double() + (logp.exp() * logp).sum(1)).abs().max()) <= 1e-4
        new = [int(t) if f is None else f for t, f in zip(top[:, 0], script.get(step, [None] * 3))]
        t_new, crop, rule = i32(new), i32([0] * 3), i32([0] * 3)
        sm.match_decode(table, state, i32(ids), t_new, crop, rule)
        x = torch.empty((3, d), dtype=dt, device=dev())
        err = torch.zeros(1, dtype=torch.int32, device=dev())
        sm.gather_surrogates(lut, rule, x, err, emb=emb, token_ids=t_new)
        crop, rule = crop.tolist(), rule.tolist()
        merges += sum(r >= 0 for r in rule)
        last = served.rows(ids, crop, [1] * 3, x, False)
        want = []
        for s in range(3):
            plain.crop(s, crop[s])
            length[s] += 1 - crop[s]
            want.append(plain.row(s, (w.lut[rule[s]] if rule[s] >= 0 else w.emb[new[s]]).double()))
        compare(last, want)
        assert served.caches[0].lengths.tolist()[:3] == length and int(err) == 0
    torch.cuda.synchronize()
    assert merges >= 4 and served.caches[0].error_bits() == 0
    # every page of the shared table is taken once, in each layer's pools
    used = served.caches[0].block_table[served.caches[0].block_table >= 0].tolist()
    assert len(used) == len(set(used)) == sum(-(-n // BS) for n in length)
    assert int(served.caches[0].free_top) == 40 - len(used)
