"""Refusals of the calls over 8-bit pages, behind shared entries and of sampled
tokens, none of which touches a GPU: the C entries' argument checks, and the
binding's."""
import ctypes as C

import pytest
import torch

from paper_2609_27233_amd import lib as sm
from test_abi_cpu import _desc
from test_backbone_calls_cpu import _rope

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    return sm.load()


def _eight(**kw):
    return _desc(**{**dict(dtype=sm.SM_E4M3, k_pool=16, v_pool=32), **kw})


def test_calls_that_take_eight_bit_pages(L):
    """Zero requests or rows: every check of the descriptor, and nothing to do."""
    d, p = _eight(), C.byref(_rope())
    assert L.sm_kv_rollback(C.byref(d), None, None, 0, None) == sm.SM_OK
    assert L.sm_kv_write_rotary(C.byref(d), 1, 1, 0, 1, 4096, 32, 1, 1024, 1, 1024, p, 1, 4096, None) == sm.SM_OK
    assert L.sm_kv_read(C.byref(d), None, None, None, 0, 0, None, 0, None, 0, None) == sm.SM_OK
    assert L.sm_decode_attention(C.byref(d), None, 0, None, 32, 1.0, 16, None, None, 0, None) == sm.SM_OK
    assert L.sm_prefill_attention(C.byref(d), None, 0, None, 0, None, 32, 1.0, 16, None, None) == sm.SM_OK
    # and those that do not
    assert L.sm_kv_append(C.byref(d), 1, 1, 1, 1, 1, 1, None) == sm.SM_EINVAL
    assert L.sm_decode_step(C.byref(d), 1, 1, 1, 1, 1, 8, 1.0, 16, 1, 1, 1 << 30, None) == sm.SM_EINVAL
    assert L.sm_decode_merge_step(C.byref(d), 1, 1, 1, 1, 1, 1, 8, 1.0, 16, 1, 1, 1 << 30, None) == sm.SM_EINVAL
    kp = sm.KVProjParams(256, 16, 16, 500000.0, 1e-5)
    assert L.sm_kv_project(C.byref(d), 1, 1, 16, C.byref(kp), 1, 1, 1, 1 << 30, None) == sm.SM_EINVAL
    assert L.sm_kv_append_projected(C.byref(d), 1, 1, 16, C.byref(kp), 1, 1 << 30, None) == sm.SM_EINVAL
    # 8-bit is a type of pages only
    assert L.sm_rotary(1, 4096, 1, 0, 32, 128, p, 0, sm.SM_E4M3, 1, 4096, None) == sm.SM_EINVAL


@pytest.mark.parametrize("kw", [dict(k_pool=8), dict(v_pool=40), dict(head_dim=96), dict(block_size=24), dict(dtype=3),
                                dict(err=None), dict(num_blocks=1 << 27)], ids=str)
def test_write_and_read_refuse_descriptors(L, kw):
    d = _eight(**kw)
    assert L.sm_kv_write_rotary(C.byref(d), 1, 1, 4, 1, 4096, 32, 1, 1024, 1, 1024, C.byref(_rope(rot_dim=64)), 1, 4096,
                                None) == sm.SM_EINVAL
    assert L.sm_kv_read(C.byref(d), 1, None, 1, 1, 4, 1, 1024, 1, 1024, None) == sm.SM_EINVAL


def test_read_argument_checks(L):
    def call(desc=_eight(), ids=1, start=None, offs=1, n=1, rows=0, k=1, sk=1024, v=1, sv=1024):
        return L.sm_kv_read(C.byref(desc), ids, start, offs, n, rows, k, sk, v, sv, None)
    assert call() == sm.SM_OK and call(k=None, sk=0) == sm.SM_OK
    for kw in (dict(n=-1), dict(n=1025), dict(rows=-1), dict(sk=1023), dict(sv=1023), dict(rows=4, ids=None),
               dict(rows=4, offs=None), dict(rows=4, k=None, v=None), dict(desc=_desc())):   # (pools off 16 bytes)
        assert call(**kw) == sm.SM_EINVAL, kw


def test_shared_argument_checks(L):
    def call(desc=_eight(), ids=1, n=0, prefixes=1, offs=1, groups=1, q=1, hq=32, scale=1.0, longest=16, prefix=16, out=1, ws=1,
             size=1 << 40):
        return L.sm_decode_attention_shared(C.byref(desc), ids, n, prefixes, offs, groups, q, hq, scale, longest, prefix, out, ws,
                                            size, None)
    assert call() == sm.SM_OK and call(desc=_desc()) == sm.SM_OK and call(groups=0) == sm.SM_OK
    need = L.sm_decode_shared_workspace_bytes(4, 32, 128, 16, 16)
    assert need > L.sm_decode_workspace_bytes(4, 32, 128, 16)
    for kw in (dict(n=-1), dict(prefix=-1), dict(groups=-1), dict(groups=65536), dict(scale=NAN), dict(scale=INF),
               dict(desc=_desc(dtype=sm.SM_F32)), dict(n=4, groups=0), dict(n=4, prefixes=None), dict(n=4, offs=None),
               dict(n=4, ids=None), dict(n=4, q=None), dict(n=4, out=None), dict(n=4, ws=None), dict(n=4, size=need - 1),
               dict(n=4, longest=257), dict(n=4, prefix=257), dict(n=4, hq=31), dict(n=4, hq=256), dict(n=65536),
               dict(n=4, desc=_eight(head_dim=96)), dict(n=4, desc=_eight(num_kv_heads=1 << 20), hq=1 << 20)):
        assert call(**kw) == sm.SM_EINVAL, kw
    for bad in ((0, 32, 128, 16, 16), (4, 0, 128, 16, 16), (4, 32, 0, 16, 16), (4, 32, 128, -1, 16), (4, 32, 128, 16, -1)):
        assert L.sm_decode_shared_workspace_bytes(*bad) == 0


def test_sample_argument_checks(L):
    need = L.sm_sample_workspace_bytes(4, 1000)
    assert need > 0 and L.sm_sample_workspace_bytes(0, 1000) == 0 and L.sm_sample_workspace_bytes(4, 0) == 0

    def call(x=1, stride=1000, rows=0, vocab=1000, dt=sm.SM_BF16, u=1, t=None, k=None, p=None, m=None, out=1, lp=None, ws=16,
             size=need):
        return L.sm_sample_tokens(x, stride, rows, vocab, dt, u, t, k, p, m, out, lp, ws, size, None, None)
    assert call() == sm.SM_OK and call(vocab=1 << 19, stride=1 << 19) == sm.SM_OK
    for kw in (dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 19) + 1, stride=1 << 20), dict(stride=999), dict(dt=2),
               dict(rows=4, x=None), dict(rows=4, u=None), dict(rows=4, out=None), dict(rows=4, ws=None), dict(rows=4, ws=8),
               dict(rows=4, size=need - 1)):
        assert call(**kw) == sm.SM_EINVAL, kw


def test_wrappers_refuse_before_anything_is_enqueued(monkeypatch, L):
    monkeypatch.setattr(sm, "_here", lambda stream: (0, -1))      # the host's tensors are "on the device"
    sm_ptr, sm._ptr = sm._ptr, lambda t: t.data_ptr()
    try:
        c = sm.PagedCache(dtype=torch.float8_e4m3fn, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=8, max_seqs=2,
                          max_blocks_per_seq=4, device="cpu")
    finally:
        sm._ptr = sm_ptr
    assert c.row_dtype == torch.bfloat16 and c.desc.dtype == sm.SM_E4M3
    assert c.k_pool.shape == (8, 2, 16, 64) and c.v_pool.shape == (8, 2, 64, 16) and c.k_exp.shape == c.v_exp.shape == (8, 2, 16)
    assert c.k_exp.data_ptr() == c.k_pool.data_ptr() + c.k_pool.numel()            # one pool: values, then exponents
    i32, bf = torch.int32, torch.bfloat16
    ids, offs = torch.zeros(1, dtype=i32), torch.zeros(2, dtype=i32)
    rows = torch.zeros((3, 2, 64), dtype=bf)
    for kw in (dict(K=rows.float()), dict(K=rows[:, :1]), dict(V=rows[:2]), dict(K=rows.transpose(1, 2)), dict(offs=offs[:1]),
               dict(start=ids[:0]), dict(K=None, V=None), dict(ids=ids.long()), dict(offs=offs.long())):
        a = {**dict(ids=ids, offs=offs, K=rows, V=rows, start=None), **kw}
        with pytest.raises(sm.SpanMergeError):
            sm.kv_read(c, a["ids"], a["offs"], a["K"], a["V"], start=a["start"])
    x, u, tok, ws = torch.zeros((4, 100), dtype=bf), torch.zeros(4), torch.zeros(4, dtype=i32), torch.zeros(1 << 20, dtype=torch.uint8)
    for kw in (dict(u=u[:3]), dict(tokens=tok[:3]), dict(tokens=tok.long()), dict(u=u.double()), dict(temperature=u[:3]),
               dict(top_k=u), dict(top_p=tok), dict(min_p=u[:2]), dict(logprob=u[:1]), dict(err=tok[:0]), dict(logits=x[0]),
               dict(logits=x.t()), dict(logits=x.half()), dict(ws=ws[:0])):
        a = {**dict(logits=x, u=u, tokens=tok, ws=ws), **kw}
        with pytest.raises(sm.SpanMergeError):
            sm.sample_tokens(a.pop("logits"), a.pop("u"), a.pop("tokens"), a.pop("ws"), **a)


def test_sizes_that_no_int_holds_are_refused(L):
    b, many = sm._calls(), 1 << 32
    x, one = (torch.zeros((1, 8)),), torch.zeros(64, dtype=torch.int32)
    args = [x, 8, 0, 8, 0, None, None, None, None, None, one, None, one, 256, None, 0, -1]
    assert b.sm_sample_tokens(*args) == sm.SM_OK
    for at in (2, 3):
        bad = list(args)
        bad[at] += many
        with pytest.raises(sm.SpanMergeError, match="argument"):
            b.sm_sample_tokens(*bad)


def test_shared_wrapper_refuses_what_does_not_lie_in_one_piece(monkeypatch, L):
    monkeypatch.setattr(sm, "_here", lambda stream: (0, -1))
    monkeypatch.setattr(sm, "_ptr", lambda t: t.data_ptr())
    c = sm.PagedCache(dtype=torch.float8_e4m3fn, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=8, max_seqs=2,
                      max_blocks_per_seq=4, device="cpu")
    i32, wide = torch.int32, torch.zeros((3, 4, 128), dtype=torch.bfloat16)
    q, two = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=i32)
    ws = torch.zeros(sm.decode_shared_workspace_bytes(3, 4, 64, 64, 64), dtype=torch.uint8)
    good = dict(ids=two[:3], prefixes=two[:1], offs=two[:2], q=q, out=q, ws=ws)
    for kw in (dict(q=wide[..., :64]), dict(out=wide[..., 64:]), dict(q=torch.zeros((3, 8, 64), dtype=q.dtype)[:, :4]),
               dict(q=q.expand(3, 4, 64)[:1].expand(3, 4, 64)), dict(q=q.float()), dict(out=q[:2]), dict(ids=two[::2]),
               dict(offs=torch.zeros(4, dtype=i32)[::2]), dict(prefixes=two[:2]), dict(ws=ws[::2]), dict(ws=ws[:100])):
        a = {**good, **kw}
        with pytest.raises(sm.SpanMergeError):
            sm.decode_attention_shared(c, a["ids"], a["prefixes"], a["offs"], a["q"], a["out"], a["ws"], 64, 64)
