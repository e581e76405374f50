"""The operators between a backbone's projections and the paged cache, and from its logits to a token, as cases that
can be timed and compared.

  reserve   block tables, positions and slots of the rows that a batch's requests are about to write
  rotary    rotary positions of rows of heads
  write     a packed projection's rows: q and k turned, K and V put into their pages by slot
  norm      residual sum with the norms after one block and before the next
  logprobs  log probabilities of given tokens, entropy and top alternatives of rows of logits
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA = 500000.0


# --------------------------------------------------------------------------
# the cases

def listed():
    return [
        # one decode step of the benchmark batch whose last row was a draft: the smallest call
        dict(name="reserve-step", kind="reserve", n=16, bs=16, lo=2458, hi=2842, rlo=1, rhi=1, pad=0),
        # the 7B-shaped serving batch, up to 8 draft rows for each session, some with none
        dict(name="reserve-drafts", kind="reserve", n=128, bs=16, lo=512, hi=4096, rlo=0, rhi=8, pad=96),
        # the benchmark's compacted prompt batch, 16 x 2458 rows from empty
        dict(name="reserve-prompts", kind="reserve", n=16, bs=16, lo=2458, hi=2458, rlo=2458, rhi=2458, pad=0),
        # gradient of half a head's rotation, pairs side by side, a prompt of the small fp32 model
        dict(name="rotary-f32-back", kind="rotary", dtype="f32", rows=512, H=4, D=64, R=32, layout="interleaved",
             scaling="none", at=0, transpose=True, packed=False),
        # query heads of a long document's chunk far behind the trained context, out of a packed projection
        dict(name="rotary-far", kind="rotary", dtype="bf16", rows=4096, H=64, D=128, R=128, layout="half",
             scaling="bands", at=120000, transpose=False, packed=True),
        # one decode step of the benchmark batch, 8B-shaped layer
        dict(name="write-step", kind="write", dtype="bf16", n=16, lo=1, hi=1, past=2650, Hq=32, Hkv=8, D=128, R=128, bs=16,
             layout="half", scaling="none", pad=0),
        # prefill of the benchmark's compacted prompt batch
        dict(name="write-prompts", kind="write", dtype="bf16", n=16, lo=2458, hi=2458, past=0, Hq=32, Hkv=8, D=128, R=128,
             bs=16, layout="half", scaling="bands", pad=0),
        # ragged chunks of 33 sessions in mid-page, half of each head turned, fp32 cache, padded rows
        dict(name="write-f32-ragged", kind="write", dtype="f32", n=33, lo=1, hi=61, past=517, Hq=4, Hkv=4, D=64, R=32, bs=32,
             layout="interleaved", scaling="ramp", pad=13),
        # one decode step: residual sum and the next block's norm
        dict(name="norm-step", kind="norm", dtype="bf16", rows=16, d=4096, post="none", gate="none", pre="rms", scale=1.0),
        # the compacted prompt batch with a norm behind the block, its channel gate and a residual scale
        dict(name="norm-prompts", kind="norm", dtype="bf16", rows=39328, d=4096, post="rms", gate="channel", pre="rms",
             scale=0.7),
        # one decode step of the benchmark batch: the token and its alternatives
        dict(name="logprobs-step", kind="logprobs", dtype="bf16", rows=16, V=128256, k=8, temperature=0.8, masked=0.0),
        # a prompt batch of the benchmark's vocabulary scored: 4096 positions
        dict(name="logprobs-prompts", kind="logprobs", dtype="bf16", rows=4096, V=128256, k=20, temperature=1.0, masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (query heads, kv heads, head dim) of the layers the library is configured and tested with
_LAYERS = ((32, 8, 128), (28, 4, 128), (64, 8, 128), (16, 4, 64), (4, 4, 64))
_SCALINGS = ("none", "none", "linear", "bands", "ramp")


def draw(rng):
    kind = rng.choice(("reserve", "rotary", "write", "norm", "logprobs"))
    if kind == "reserve":
        n = _log_int(rng, 1, 1024)
        rhi = _log_int(rng, 1, min(8192, 65536 // n))
        rlo = rng.choice((0, 1, rhi))
        hi = rhi + _log_int(rng, 1, min(16384, 1 + (1 << 21) // n))
        return dict(kind=kind, n=n, bs=rng.choice((16, 16, 32, 64, 256)), lo=max(rhi, int(hi * rng.uniform(0.1, 1))), hi=hi,
                    rlo=rlo, rhi=rhi, pad=rng.choice((0, 0, 7, 256)))
    if kind == "rotary":
        dtype = rng.choice(("bf16", "bf16", "f32"))
        H, D = rng.choice((1, 4, 7, 8, 28, 32, 64)), rng.choice((64, 72, 80, 96, 128, 128, 256))
        return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, min(65536, (1 << (28 if dtype == "bf16" else 27)) // (H * D))),
                    H=H, D=D, R=rng.choice((D, D, D // 2, 2 * (D // 8))), layout=rng.choice(("half", "interleaved")),
                    scaling=rng.choice(_SCALINGS), at=rng.choice((0, 0, _log_int(rng, 1, 1000000))),
                    transpose=rng.random() < 0.3, packed=rng.random() < 0.5)
    if kind == "write":
        Hq, Hkv, D = rng.choice(_LAYERS)
        dtype = "f32" if D == 64 and rng.random() < 0.4 else "bf16"
        n = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, max(1, min(8192, 39328 * 32 // (n * max(Hq, 16)))))
        return dict(kind=kind, dtype=dtype, n=n, lo=rng.choice((1, hi)), hi=hi, past=rng.choice((0, _log_int(rng, 1, 2048))),
                    Hq=Hq, Hkv=Hkv, D=D, R=rng.choice((D, D, D // 2)), bs=rng.choice((16, 16, 32, 64)),
                    layout=rng.choice(("half", "half", "interleaved")), scaling=rng.choice(_SCALINGS),
                    pad=rng.choice((0, 0, 5, 64)))
    if kind == "norm":
        dtype = rng.choice(("bf16", "bf16", "f32"))
        d = rng.choice((64, 250, 256, 1000, 1111, 2048, 3584, 4096, 5120, 8192, 16384))
        return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, min(65536, (1 << (27 if dtype == "bf16" else 26)) // d)), d=d,
                    post=rng.choice(("none", "rms", "layer")), gate=rng.choice(("none", "channel", "row")),
                    pre=rng.choice(("rms", "rms", "layer")), scale=rng.choice((1.0, round(rng.uniform(0.1, 2.0), 3))))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    V = rng.choice((1000, 32000, 50257, 128256, 152064, _log_int(rng, 64, 262144)))
    return dict(kind=kind, dtype=dtype, rows=_log_int(rng, 1, min(8192, (1 << (29 if dtype == "bf16" else 28)) // V)), V=V,
                k=rng.choice((0, 1, 1, 5, 8, 20, 64)), temperature=rng.choice((1.0, round(rng.uniform(0.3, 2.0), 2))),
                masked=rng.choice((0.0, 0.0, 0.5, 0.99)))


# --------------------------------------------------------------------------
# inputs (plain torch and numpy)

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)


def _i32(a):
    return torch.as_tensor(np.array(a, dtype=np.int32, order="C")).cuda()


def _rope_args(c):
    """The arguments of a case's rotation: factor 8 over a trained context of 8192 where it is scaled."""
    a = dict(rot_dim=c["R"], theta=THETA, layout=c["layout"])
    if c["scaling"] != "none":
        a.update(scaling=c["scaling"], factor=8.0)
    if c["scaling"] == "bands":
        a.update(low=1.0, high=4.0, context=8192)
    if c["scaling"] == "ramp":
        a.update(low=1.0, high=32.0, context=8192, attn_scale=0.1 * math.log(8.0) + 1.0)
    return a


def _tables(rng, lens, bs, spare):
    """Block table of sequences of these lengths on pages in any order, and the stack of the free ones."""
    blocks = -(-np.asarray(lens) // bs)
    nb = int(blocks.sum()) + spare
    order = rng.permutation(nb).astype(np.int32)
    table = np.full((len(lens), max(1, int(blocks.max()))), -1, np.int32)
    at = 0
    for i, b in enumerate(blocks):
        table[i, :b] = order[at:at + b]
        at += int(b)
    stack = np.full(nb, -1, np.int32)
    stack[:nb - at] = order[at:]
    return table, stack, nb - at, nb


def _prepare_reserve(c, seed):
    rng, n, bs = np.random.RandomState(seed % (1 << 32)), c["n"], c["bs"]
    sizes = np.random.RandomState(n)  # lengths are the case's own, pages and order the seed's
    rows = sizes.randint(c["rlo"], c["rhi"] + 1, n)
    lens = np.maximum(sizes.randint(c["lo"], c["hi"] + 1, n), rows)
    table, stack, top, nb = _tables(rng, lens, bs, 8)
    ids = rng.permutation(n)
    cap = int(rows.sum()) + c["pad"]
    # each request drops its last rows and reserves as many again, so that a pass leaves the lengths as it found them
    s = dict(kind="reserve", ids=_i32(ids), rows=_i32(rows[ids]), crop=_i32(rows[ids]), bs=bs, nb=nb,
             tables=dict(block_table=_i32(table), lengths=_i32(lens), free_stack=_i32(stack), free_top=_i32([top])),
             row_offsets=torch.empty(n + 1, dtype=torch.int32, device="cuda"),
             pos=torch.empty(cap, dtype=torch.int32, device="cuda"), slots=torch.empty(cap, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2609_27233_amd import lib as sm
        s["cache"] = sm.PagedCache(dtype=torch.bfloat16, num_kv_heads=1, head_dim=64, block_size=bs, num_blocks=nb, max_seqs=n,
                                   max_blocks_per_seq=table.shape[1])
        for name, t in s["tables"].items():
            s["tables"][name] = getattr(s["cache"], name).copy_(t)
    return s


def _prepare_rotary(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    rows, H, D = c["rows"], c["H"], c["D"]
    buf = _randn(g, (rows, H * D + (2 * D if c["packed"] else 0)), dt)
    s = dict(kind="rotary", x=buf[:, :H * D].view(rows, H, D), out=torch.empty((rows, H, D), dtype=dt, device="cuda"),
             pos=_i32(c["at"] + np.random.RandomState(seed % (1 << 32)).permutation(rows)), args=_rope_args(c),
             transpose=c["transpose"])
    if own:
        from paper_2609_27233_amd import lib as sm
        s["rope"] = sm.rope_params(**s["args"])
    return s


def _prepare_write(c, seed):
    g, dt, rng = _gen(seed), DTYPES[c["dtype"]], np.random.RandomState(seed % (1 << 32))
    n, bs, Hq, Hkv, D = c["n"], c["bs"], c["Hq"], c["Hkv"], c["D"]
    sizes = np.random.RandomState(n)
    new = sizes.randint(c["lo"], c["hi"] + 1, n)
    past = sizes.randint(c["past"] // 2, c["past"] + 1, n) if c["past"] else np.zeros(n, np.int64)
    table, _, _, nb = _tables(rng, past + new, bs, 4)
    pos = np.concatenate([np.arange(p, p + m) for p, m in zip(past, new)])
    req = np.repeat(np.arange(n), new)
    slots = table[req, pos // bs] * bs + pos % bs
    pos, slots = np.concatenate([pos, np.zeros(c["pad"], int)]), np.concatenate([slots, np.full(c["pad"], -1)])
    rows = len(pos)
    qkv = _randn(g, (rows, (Hq + 2 * Hkv) * D), dt)
    s = dict(kind="write", q=qkv[:, :Hq * D].view(rows, Hq, D), k=qkv[:, Hq * D:(Hq + Hkv) * D].view(rows, Hkv, D),
             v=qkv[:, (Hq + Hkv) * D:].view(rows, Hkv, D), pos=_i32(pos), slots=_i32(slots), args=_rope_args(c), bs=bs,
             q_out=torch.empty((rows, Hq, D), dtype=dt, device="cuda"))
    k_pool, v_pool = _randn(g, (nb, Hkv, bs, D), dt), _randn(g, (nb, Hkv, D, bs), dt)
    if own:
        from paper_2609_27233_amd import lib as sm
        s["rope"] = sm.rope_params(**s["args"])
        s["cache"] = sm.PagedCache(dtype=dt, num_kv_heads=Hkv, head_dim=D, block_size=bs, num_blocks=nb, max_seqs=n,
                                   max_blocks_per_seq=table.shape[1])
        k_pool, v_pool = s["cache"].k_pool.copy_(k_pool), s["cache"].v_pool.copy_(v_pool)
    s.update(k_pool=k_pool, v_pool=v_pool)
    return s


def _prepare_norm(c, seed):
    g, dt, rows, d = _gen(seed), DTYPES[c["dtype"]], c["rows"], c["d"]
    s = dict(kind="norm", scale=c["scale"], h=_randn(g, (rows, d), dt, 2.0, 0.1), y=_randn(g, (rows, d), dt, 1.0, -0.1),
             gate=None if c["gate"] == "none" else _randn(g, (d,) if c["gate"] == "channel" else (rows, d), dt, 0.5),
             h_out=torch.empty((rows, d), dtype=dt, device="cuda"), n_out=torch.empty((rows, d), dtype=dt, device="cuda"))
    for name in ("post", "pre"):
        s[name] = None if c[name] == "none" else dict(kind=c[name], gain=_randn(g, (d,), dt, 0.1, 1.0), eps=1e-5,
                                                      bias=_randn(g, (d,), dt, 0.1) if c[name] == "layer" else None)
    if own:
        from paper_2609_27233_amd import lib as sm
        s["norms"] = [None if s[name] is None else sm.norm_params(**s[name]) for name in ("post", "pre")]
    return s


def _prepare_logprobs(c, seed):
    g, dt, rows, V, k = _gen(seed), DTYPES[c["dtype"]], c["rows"], c["V"], min(c["k"], c["V"])
    x = _randn(g, (rows, V), dt, 2.5)
    # a few likely tokens in each row, as a trained model has
    peak = torch.randint(V, (rows, 8), device="cuda", generator=g)
    x.scatter_add_(1, peak, (6.0 + 6.0 * torch.rand((rows, 8), device="cuda", generator=g)).to(dt))
    if c["masked"]:
        # a constrained vocabulary: the first 64 tokens and a random part of the others stay
        off = torch.rand((V,), device="cuda", generator=g) < c["masked"]
        off[:64] = False
        x[:, off] = -math.inf
        tokens = torch.randint(min(V, 64), (rows,), device="cuda", generator=g)
    else:
        tokens = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.5, peak[:, 0],
                             torch.randint(V, (rows,), device="cuda", generator=g))
    f32 = dict(dtype=torch.float32, device="cuda")
    s = dict(kind="logprobs", x=x, tokens=tokens.to(torch.int32), k=k, scale=1.0 / c["temperature"],
             logprob=torch.empty(rows, **f32), entropy=torch.empty(rows, **f32),
             top_ids=torch.empty((rows, k), dtype=torch.int32, device="cuda"), top_logprobs=torch.empty((rows, k), **f32))
    if own:
        from paper_2609_27233_amd import lib as sm
        s["ws"] = torch.zeros(sm.token_logprobs_workspace_bytes(rows, V, k), dtype=torch.uint8, device="cuda")
    return s


_PREPARE = dict(reserve=_prepare_reserve, rotary=_prepare_rotary, write=_prepare_write, norm=_prepare_norm,
                logprobs=_prepare_logprobs)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed)


# --------------------------------------------------------------------------
# the framework's calls

def _run_own(s):
    from paper_2609_27233_amd import lib as sm
    if s["kind"] == "reserve":
        sm.kv_reserve(s["cache"], s["ids"], s["rows"], s["row_offsets"], s["pos"], s["slots"], crop=s["crop"])
        return dict(row_offsets=s["row_offsets"], pos=s["pos"], slots=s["slots"], **s["tables"])
    if s["kind"] == "rotary":
        sm.rotary(s["x"], s["pos"], s["rope"], s["out"], transpose=s["transpose"])
        return s["out"]
    if s["kind"] == "write":
        sm.kv_write_rotary(s["cache"], s["pos"], s["slots"], s["q"], s["k"], s["v"], s["rope"], s["q_out"])
        return dict(q=s["q_out"], k_pool=s["k_pool"], v_pool=s["v_pool"])
    if s["kind"] == "norm":
        post, pre = s["norms"]
        sm.block_norm(s["h"], s["y"], s["h_out"], s["n_out"], post=post, gate=s["gate"], scale=s["scale"], pre=pre)
        return dict(h=s["h_out"], n=s["n_out"])
    sm.token_logprobs(s["x"], s["tokens"], s["logprob"], s["entropy"], s["top_ids"], s["top_logprobs"], s["ws"],
                      scale=s["scale"])
    return {name: s[name] for name in ("logprob", "entropy", "top_ids", "top_logprobs")}


# --------------------------------------------------------------------------
# the plain forms

def _plain_reserve(s):
    t, bs, n, cap = s["tables"], s["bs"], s["ids"].numel(), s["pos"].numel()
    ids, rows, crop = s["ids"].long(), s["rows"].long(), s["crop"].long()
    L = t["lengths"][ids].long()
    keep = L - crop
    had, kept, want = (L + bs - 1) // bs, (keep + bs - 1) // bs, (keep + rows + bs - 1) // bs
    freed, need = had - kept, want - kept
    top, all_freed = t["free_top"].long(), freed.sum()
    j = torch.arange(t["block_table"].shape[1], device="cuda")
    cells = t["block_table"][ids]
    # pushed: the last request's first, the highest logical block first
    gone = (j >= kept[:, None]) & (j < had[:, None])
    place = top + (all_freed - freed.cumsum(0))[:, None] + had[:, None] - 1 - j
    stack = torch.cat([t["free_stack"], t["free_stack"].new_zeros(1)])
    stack[torch.where(gone, place, s["nb"])] = cells
    # popped: the first request's first, the lowest logical block first
    taken = (j >= kept[:, None]) & (j < want[:, None])
    pop = top + all_freed - 1 - ((need.cumsum(0) - need)[:, None] + j - kept[:, None])
    cells = torch.where(taken, stack[torch.where(taken, pop, s["nb"])], torch.where(gone, -1, cells))
    t["free_stack"].copy_(stack[:-1])
    t["block_table"][ids] = cells
    t["lengths"][ids] = (keep + rows).int()
    t["free_top"].copy_(top + all_freed - need.sum())
    ends = rows.cumsum(0)
    s["row_offsets"].copy_(torch.cat([ends.new_zeros(1), ends]))
    r = torch.arange(cap, device="cuda")
    i = torch.searchsorted(ends, r, right=True).clamp_(max=n - 1)
    there = r < ends[-1]
    p = torch.where(there, keep[i] + r - (ends - rows)[i], 0)
    s["pos"].copy_(p)
    s["slots"].copy_(torch.where(there, cells[i, p // bs].long() * bs + p % bs, -1))
    return dict(row_offsets=s["row_offsets"], pos=s["pos"], slots=s["slots"], **t)


def _frequencies(a):
    R, theta = a["rot_dim"], a["theta"]
    j = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    w = theta ** (-2.0 * j / R)
    scaling = a.get("scaling")
    if scaling == "linear":
        w = w / a["factor"]
    elif scaling == "bands":
        u = ((a["context"] * w / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
        w = w * (u + (1 - u) / a["factor"])
    elif scaling == "ramp":
        at = [R * math.log(a["context"] / (2 * math.pi * b)) / (2 * math.log(theta)) for b in (a["high"], a["low"])]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        u = ((j - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        w = w * (1 - u + u / a["factor"])
    return w


def _turned(x, pos, a, transpose=False):
    R, f = a["rot_dim"], a.get("attn_scale", 1.0)
    ang = pos.double()[:, None] * _frequencies(a)
    cos, sin = (f * ang.cos()).float()[:, None], (f * ang.sin()).float()[:, None]
    if transpose:
        sin = -sin
    x32 = x.float()
    out = x32.clone()
    if a["layout"] == "half":
        u, v = x32[..., :R // 2], x32[..., R // 2:R]
        out[..., :R // 2], out[..., R // 2:R] = u * cos - v * sin, u * sin + v * cos
    else:
        u, v = x32[..., 0:R:2], x32[..., 1:R:2]
        out[..., 0:R:2], out[..., 1:R:2] = u * cos - v * sin, u * sin + v * cos
    return out.to(x.dtype)


def _plain_write(s):
    q, k, v, bs = _turned(s["q"], s["pos"], s["args"]), _turned(s["k"], s["pos"], s["args"]), s["v"], s["bs"]
    slots = s["slots"].long()
    # a padded row writes the first row once more
    src = torch.where(slots >= 0, torch.arange(slots.numel(), device="cuda"), 0)
    slots = slots[src]
    s["k_pool"][slots // bs, :, slots % bs] = k[src]
    s["v_pool"][slots // bs, :, :, slots % bs] = v[src]
    s["q_out"].copy_(q)
    return dict(q=s["q_out"], k_pool=s["k_pool"], v_pool=s["v_pool"])


def _normed(x, p):
    if p["kind"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + p["eps"]) * p["gain"].float()
    return x if p["bias"] is None else x + p["bias"].float()


def _plain_norm(s):
    t = s["y"].float()
    if s["post"] is not None:
        t = _normed(t, s["post"])
    if s["gate"] is not None:
        t = t * s["gate"].float()
    h = s["h"].float() + s["scale"] * t
    s["h_out"].copy_(h)
    s["n_out"].copy_(_normed(h, s["pre"]))
    return dict(h=s["h_out"], n=s["n_out"])


def _plain_logprobs(s):
    x, V = s["x"].float(), s["x"].shape[1]
    # values in order, the lower index first among equal ones: one whole number for both
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits >= 0, bits, bits ^ 0x7fffffff).long() * (1 << 32) + (V - 1 - torch.arange(V, device="cuda"))
    ids = V - 1 - (key.topk(s["k"], 1).values & 0xffffffff) if s["k"] else s["top_ids"].long()
    z = x * s["scale"]
    m = z.max(1, keepdim=True).values
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + total.log()
    s["logprob"].copy_(z.gather(1, s["tokens"].long()[:, None])[:, 0] - lse[:, 0])
    s["entropy"].copy_(total.log()[:, 0] - (torch.where(e > 0, (z - m) * e, 0.0).sum(1) / total[:, 0]))
    s["top_ids"].copy_(ids)
    s["top_logprobs"].copy_(z.gather(1, ids) - lse)
    return {name: s[name] for name in ("logprob", "entropy", "top_ids", "top_logprobs")}


def _plain_rotary(s):
    s["out"].copy_(_turned(s["x"], s["pos"], s["args"], s["transpose"]))
    return s["out"]


_PLAIN = dict(reserve=_plain_reserve, rotary=_plain_rotary, write=_plain_write, norm=_plain_norm, logprobs=_plain_logprobs)


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["kind"]](state)


# --------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    c = case
    size = 2 if c.get("dtype", "bf16") == "bf16" else 4
    if c["kind"] == "reserve":
        # ids, counts, lengths (read and written), offsets; the blocks that move (table and stack, both ways); positions and slots
        rows = c["n"] * (c["rlo"] + c["rhi"]) / 2
        return dict(bytes=24 * c["n"] + 16 * rows / c["bs"] + 8 * (rows + c["pad"]), flops=0)
    if c["kind"] == "rotary":
        return dict(bytes=c["rows"] * (2 * c["H"] * c["D"] * size + 4), flops=3 * c["rows"] * c["H"] * c["R"])
    if c["kind"] == "write":
        rows = c["n"] * (c["lo"] + c["hi"]) / 2
        return dict(bytes=rows * ((2 * c["Hq"] + 4 * c["Hkv"]) * c["D"] * size + 8) + c["pad"] * (2 * c["Hq"] * c["D"] * size + 8),
                    flops=3 * rows * (c["Hq"] + c["Hkv"]) * c["R"])
    if c["kind"] == "norm":
        per = 4 + (1 if c["gate"] == "row" else 0)
        return dict(bytes=c["rows"] * c["d"] * per * size, flops=c["rows"] * c["d"] * (6 + (4 if c["post"] != "none" else 0)))
    return dict(bytes=c["rows"] * (c["V"] * size + 12 + 8 * c["k"]), flops=5 * c["rows"] * c["V"])


# --------------------------------------------------------------------------
# the definitions, in 64 bits

def _exact_reserve(c, s):
    """The sequential definition: every push and pop one after another."""
    t = {name: v.cpu().numpy().copy() for name, v in s["tables"].items()}
    ids, rows, crop, bs = s["ids"].cpu().numpy(), s["rows"].cpu().numpy(), s["crop"].cpu().numpy(), s["bs"]
    table, lens, stack, top = t["block_table"], t["lengths"], t["free_stack"], int(t["free_top"][0])
    for i in reversed(range(len(ids))):
        q = ids[i]
        for j in range(-(-int(lens[q]) // bs) - 1, -(-int(lens[q] - crop[i]) // bs) - 1, -1):
            stack[top], table[q, j] = table[q, j], -1
            top += 1
        lens[q] -= crop[i]
    pos, slots = np.zeros(s["pos"].numel(), np.int64), np.full(s["pos"].numel(), -1, np.int64)
    at = 0
    for i, q in enumerate(ids):
        for j in range(-(-int(lens[q]) // bs), -(-int(lens[q] + rows[i]) // bs)):
            top -= 1
            table[q, j] = stack[top]
        p = lens[q] + np.arange(rows[i], dtype=np.int64)
        pos[at:at + rows[i]] = p
        slots[at:at + rows[i]] = table[q, p // bs].astype(np.int64) * bs + p % bs
        at += int(rows[i])
        lens[q] += rows[i]
    t["free_top"][0] = top
    return dict(row_offsets=np.concatenate([[0], np.cumsum(rows)]), pos=pos, slots=slots, **t)


def _exact_turn(x, pos, a, transpose=False):
    """Each pair as a complex number, times attn_scale e^(i angle)."""
    R, j = a["rot_dim"], np.arange(a["rot_dim"] // 2)
    w = np.exp(-2.0 * j / R * np.log(a["theta"]))
    if a.get("scaling") == "linear":
        w /= a["factor"]
    elif a.get("scaling") == "bands":
        turns = a["context"] * w / (2 * np.pi)
        u = np.clip((turns - a["low"]) / (a["high"] - a["low"]), 0, 1)
        w = u * w + (1 - u) * w / a["factor"]
    elif a.get("scaling") == "ramp":
        def at(b):
            return R * np.log(a["context"] / (b * 2 * np.pi)) / (2 * np.log(a["theta"]))
        lo, hi = max(np.floor(at(a["high"])), 0), min(np.ceil(at(a["low"])), R - 1)
        u = 1 - np.clip((j - lo) / max(hi - lo, 0.001), 0, 1)
        w = u * w + (1 - u) * w / a["factor"]
    turn = a.get("attn_scale", 1.0) * torch.exp(1j * pos.double()[:, None] * torch.from_numpy(w).cuda())[:, None]
    turn = turn.conj() if transpose else turn
    out = x.double()
    head = out[..., :R]
    pairs = head.unflatten(-1, (2, R // 2)).transpose(-1, -2) if a["layout"] == "half" else head.unflatten(-1, (R // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.transpose(-1, -2).flatten(-2) if a["layout"] == "half" else z.flatten(-2)
    return torch.cat([z, out[..., R:]], -1)


def _exact_write(c, s):
    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    at = torch.nonzero(s["slots"] >= 0)[:, 0]
    slots = s["slots"][at].long()
    k = _exact_turn(s["k"], s["pos"], s["args"])[at]
    flat = k_pool.transpose(1, 2).flatten(0, 1).index_copy(0, slots, k)
    k_pool = flat.unflatten(0, (-1, s["bs"])).transpose(1, 2)
    flat = v_pool.permute(0, 3, 1, 2).flatten(0, 1).index_copy(0, slots, s["v"].double()[at])
    v_pool = flat.unflatten(0, (-1, s["bs"])).permute(0, 2, 3, 1)
    return dict(q=_exact_turn(s["q"], s["pos"], s["args"]), k_pool=k_pool, v_pool=v_pool)


def _exact_norm(c, s):
    def normed(x, p):
        if p["kind"] == "layer":
            var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            return (x - mean) * torch.rsqrt(var + p["eps"]) * p["gain"].double() + p["bias"].double()
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + p["eps"]) * p["gain"].double()
    t = s["y"].double()
    t = t if s["post"] is None else normed(t, s["post"])
    t = t if s["gate"] is None else s["gate"].double() * t
    h = torch.add(s["h"].double(), t, alpha=s["scale"])
    return dict(h=h, n=normed(h, s["pre"]))


def _exact_logprobs(c, s):
    parts = []
    for x, token in zip(s["x"].split(256), s["tokens"].long().split(256)):
        z = x.double() * s["scale"]
        logp = z - torch.logsumexp(z, 1, keepdim=True)
        p = logp.exp()
        order = x.float().sort(dim=1, descending=True, stable=True).indices[:, :s["k"]]
        parts.append((logp.gather(1, token[:, None])[:, 0], -(p * torch.nan_to_num(logp, neginf=0.0)).sum(1), order,
                      logp.gather(1, order)))
    return dict(zip(("logprob", "entropy", "top_ids", "top_logprobs"), (torch.cat(v) for v in zip(*parts))))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_turn(s["x"], s["pos"], s["args"], s["transpose"])
    return dict(reserve=_exact_reserve, write=_exact_write, norm=_exact_norm, logprobs=_exact_logprobs)[case["kind"]](case, s)
