"""Refusals of the calls around a backbone's projections and logits, none of
which touches a GPU: the C entries' argument checks, and the binding's."""
import ctypes as C

import pytest
import torch

from paper_2609_27233_amd import lib as sm
from test_abi_cpu import _desc

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    return sm.load()


def _rope(**kw):
    base = dict(rot_dim=128, layout=0, scaling=0, theta=500000.0, attn_scale=1.0, factor=8.0, low=1.0, high=4.0,
                context=8192.0)
    base.update(kw)
    return sm.RopeParams(*base.values())


BAD_ROPES = [dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=63), dict(rot_dim=130), dict(layout=2), dict(layout=-1),
             dict(scaling=4), dict(scaling=-1), dict(theta=0.0), dict(theta=-1.0), dict(theta=NAN), dict(theta=INF),
             dict(attn_scale=NAN), dict(attn_scale=INF), dict(scaling=1, factor=0.0), dict(scaling=1, factor=NAN),
             dict(scaling=2, factor=INF), dict(scaling=2, low=0.0), dict(scaling=2, high=1.0), dict(scaling=2, high=NAN),
             dict(scaling=2, high=INF), dict(scaling=2, context=0.0), dict(scaling=2, context=INF),
             dict(scaling=3, theta=1.0), dict(scaling=3, low=-1.0)]


def test_reserve_argument_checks(L):
    d = _desc()

    def call(desc=d, ids=1, crop=None, rows=1, n=4, most=64, offs=1, pos=1, slots=1):
        return L.sm_kv_reserve(C.byref(desc), ids, crop, rows, n, most, offs, pos, slots, None)
    for kw in (dict(ids=None), dict(rows=None), dict(offs=None), dict(pos=None), dict(slots=None), dict(n=-1), dict(n=5),
               dict(most=-1)):
        assert call(**kw) == sm.SM_EINVAL, kw
    for kw in (dict(head_dim=96), dict(block_size=24), dict(lengths=None), dict(free_top=None), dict(err=None),
               dict(num_blocks=1 << 27)):                                     # 2^27 blocks of 16: slots would not fit
        assert call(desc=_desc(**kw)) == sm.SM_EINVAL, kw


@pytest.mark.parametrize("kw", BAD_ROPES, ids=str)
def test_rotary_refuses_bad_rotations(L, kw):
    p = _rope(**kw)
    assert L.sm_rotary(1, 4096, 1, 4, 32, 128, C.byref(p), 0, sm.SM_BF16, 1, 4096, None) == sm.SM_EINVAL
    assert L.sm_kv_write_rotary(C.byref(_desc()), 1, 1, 4, 1, 4096, 32, 1, 1024, 1, 1024, C.byref(p), 1, 4096,
                                None) == sm.SM_EINVAL


def test_rotary_argument_checks(L):
    def call(x=1, sx=4096, pos=1, rows=0, heads=32, D=128, p=_rope(), back=0, dt=sm.SM_BF16, out=1, so=4096):
        return L.sm_rotary(x, sx, pos, rows, heads, D, C.byref(p), back, dt, out, so, None)
    assert call() == sm.SM_OK and call(x=None, pos=None, out=None) == sm.SM_OK        # no row: nothing to do
    for kw in (dict(rows=-1), dict(heads=0), dict(heads=1025), dict(D=1), dict(D=258), dict(D=64), dict(sx=4095),
               dict(so=4095), dict(dt=2), dict(back=2), dict(rows=1, x=None), dict(rows=1, pos=None),
               dict(rows=1, out=None), dict(rows=2, so=4104)):                        # (in place with another stride)
        assert call(**kw) == sm.SM_EINVAL, kw
    assert L.sm_rotary(1, 4096, 1, 0, 32, 128, None, 0, sm.SM_BF16, 1, 4096, None) == sm.SM_EINVAL


def test_write_argument_checks(L):
    def call(desc=_desc(), pos=1, slots=1, rows=0, q=1, sq=4096, hq=32, k=1, sk=1024, v=1, sv=1024, p=_rope(), qo=1,
             so=4096):
        return L.sm_kv_write_rotary(C.byref(desc), pos, slots, rows, q, sq, hq, k, sk, v, sv, C.byref(p), qo, so, None)
    assert call() == sm.SM_OK
    assert call(q=None, sq=0, hq=0, qo=None, so=0) == sm.SM_OK                        # K and V alone
    for kw in (dict(rows=-1), dict(hq=-1), dict(hq=1025), dict(sq=4095), dict(so=4095), dict(sk=1023), dict(sv=1023),
               dict(rows=1, pos=None), dict(rows=1, slots=None), dict(rows=1, q=None), dict(rows=1, k=None),
               dict(rows=1, v=None), dict(rows=1, qo=None), dict(rows=2, so=4104), dict(desc=_desc(num_blocks=1 << 27)),
               dict(desc=_desc(k_pool=None)), dict(desc=_desc(head_dim=64))):         # (rot_dim 128 of 64)
        assert call(**kw) == sm.SM_EINVAL, kw


def test_block_norm_argument_checks(L):
    rms = sm.NormParams(0, 1e-5, 1, None)

    def call(h=1, sh=64, y=1, sy=64, rows=0, d=64, post=rms, gate=1, sg=0, scale=1.0, pre=rms, dt=sm.SM_BF16, ho=1, sho=64,
             no=1, sno=64):
        ref = lambda n: None if n is None else C.byref(n)                             # noqa: E731
        return L.sm_block_norm(h, sh, y, sy, rows, d, ref(post), gate, sg, scale, ref(pre), dt, ho, sho, no, sno, None)
    assert call() == sm.SM_OK
    for kw in (dict(rows=-1), dict(d=0), dict(d=16385), dict(dt=2), dict(scale=NAN), dict(scale=INF),
               dict(post=sm.NormParams(2, 1e-5, 1, None)), dict(pre=sm.NormParams(0, -1.0, 1, None)),
               dict(pre=sm.NormParams(0, NAN, 1, None)), dict(post=sm.NormParams(1, INF, 1, None)),
               dict(rows=1, h=None), dict(rows=1, ho=None, no=None), dict(rows=1, pre=None), dict(rows=1, sh=63),
               dict(rows=1, sy=63), dict(rows=1, sg=63), dict(rows=1, sho=63), dict(rows=1, sno=0),
               dict(rows=2, ho=64, no=64),                                            # one place for both outputs
               dict(rows=2, h=64, ho=64, sho=72), dict(rows=2, y=64, no=64, sno=72), dict(rows=2, gate=64, no=64)):
        assert call(**kw) == sm.SM_EINVAL, kw


def test_logprobs_argument_checks(L):
    need = L.sm_token_logprobs_workspace_bytes(4, 1000, 8)
    assert need >= 65536
    for bad in ((-1, 1000, 8), (4, 0, 0), (4, 1000, 65), (4, 5, 6), (4, 1000, -1)):
        assert L.sm_token_logprobs_workspace_bytes(*bad) == 0

    def call(x=1, s=1000, rows=4, V=1000, dt=sm.SM_BF16, scale=1.0, tok=1, lp=1, h=1, k=8, ids=1, tlp=1, ws=16, nbytes=need,
             err=1):
        return L.sm_token_logprobs(x, s, rows, V, dt, scale, tok, lp, h, k, ids, tlp, ws, nbytes, err, None)
    assert call(rows=0) == sm.SM_OK
    for kw in (dict(x=None), dict(s=999), dict(rows=-1), dict(V=0), dict(dt=5), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=NAN), dict(scale=INF), dict(scale=3e38), dict(scale=9e-21), dict(tok=None), dict(k=-1), dict(k=65), dict(V=7, k=8),
               dict(ids=None), dict(ws=None), dict(ws=8), dict(nbytes=need - 1)):
        assert call(**kw) == sm.SM_EINVAL, kw


def test_unknown_names_are_refused():
    for kw in (dict(layout="neox"), dict(scaling="dynamic")):
        with pytest.raises(sm.SpanMergeError):
            sm.rope_params(64, **kw)
    with pytest.raises(sm.SpanMergeError):
        sm.norm_params("batch")


class _Gpu(torch.Tensor):
    """A CPU tensor that says it is on the GPU: for checks that come before any launch."""
    is_cuda = True

    def get_device(self):
        return 0


def _gpu(shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_Gpu)


def test_row_strides_are_looked_at(L):
    f, stride = torch.float32, sm._calls().row_stride
    x = torch.zeros((6, 4, 8))
    assert stride(x, f, "x", 6, 4, 8) == 32
    buf = torch.zeros((6, 80))
    assert stride(buf[:, 8:40].view(6, 4, 8), f, "x", 6, 4, 8) == 80
    assert stride(buf[:1, :32].view(1, 4, 8), f, "x", 1, 4, 8) == 32                    # one row: any stride
    assert stride(torch.zeros(6, 8, 1).transpose(1, 2), f, "x", 6, 1, 8) == 8
    assert stride(torch.zeros((0, 4, 8)), f, "x", 0, 4, 8) == 32
    for bad in (x.transpose(1, 2), x.transpose(0, 1), torch.zeros((6, 4, 16))[..., ::2], torch.zeros((6, 8, 8))[:, ::2],
                x.double(), x[:5], torch.zeros((6, 32))):
        with pytest.raises(sm.SpanMergeError, match="x: expected"):
            stride(bad, f, "x", 6, 4, 8)


def test_wrong_types_and_sizes_are_refused(monkeypatch, L):
    monkeypatch.setattr(sm, "_here", lambda stream: (0, 0))
    i64, i32 = torch.int64, torch.int32
    err = sm.SpanMergeError
    with pytest.raises(err, match="torch.int32"):
        sm.rotary(_gpu((3, 2, 8)), _gpu(3, i64), sm.rope_params(8), _gpu((3, 2, 8)))
    with pytest.raises(err, match="pos"):
        sm.rotary(_gpu((3, 2, 8)), _gpu(2, i32), sm.rope_params(8), _gpu((3, 2, 8)))
    with pytest.raises(err, match="out"):
        sm.rotary(_gpu((3, 2, 8)), _gpu(3, i32), sm.rope_params(8), _gpu((3, 2, 8), torch.bfloat16))
    with pytest.raises(err, match="pre"):
        sm.block_norm(_gpu((3, 8)), None, None, _gpu((3, 8)), pre=sm.norm_params("rms", _gpu(7)))
    with pytest.raises(err, match="gate"):
        sm.block_norm(_gpu((3, 8)), _gpu((3, 8)), _gpu((3, 8)), None, gate=_gpu((2, 8)))
    with pytest.raises(err, match="torch.int32"):
        sm.token_logprobs(_gpu((3, 8)), _gpu(3, i64), _gpu(3), None, None, None, _gpu(65536, torch.uint8))
    with pytest.raises(err, match="torch.float32"):
        sm.token_logprobs(_gpu((3, 8)), _gpu(3, i32), _gpu(3, torch.float64), None, None, None, _gpu(65536, torch.uint8))
    with pytest.raises(err, match="top_ids"):
        sm.token_logprobs(_gpu((3, 8)), None, None, None, _gpu((2, 4), i32), None, _gpu(65536, torch.uint8))
    with pytest.raises(err, match="dtype"):
        sm.token_logprobs(_gpu((3, 8), torch.float16), None, None, None, None, None, _gpu(65536, torch.uint8))
    for bad in (_gpu((6, 8)), _gpu((3, 2, 2, 4)), _gpu(8)):
        with pytest.raises(err, match="x: expected 3 dimensions"):
            sm.rotary(bad, _gpu(3, i32), sm.rope_params(8), _gpu((3, 2, 8)))
    with pytest.raises(err, match="h: expected 2 dimensions"):
        sm.block_norm(_gpu(8), None, None, _gpu(8), pre=sm.norm_params("rms"))
    with pytest.raises(err, match="logits: expected 2 dimensions"):
        sm.token_logprobs(_gpu(8), None, None, _gpu(1), None, None, _gpu(65536, torch.uint8))
    with pytest.raises(err, match="contiguous"):
        sm.rotary(_gpu((3, 2, 8)), _gpu(6, i32)[::2], sm.rope_params(8), _gpu((3, 2, 8)))


@pytest.mark.parametrize("exchange", [True, False], ids=["exchange", "methods"])
def test_what_tensors_are(L, exchange):
    """The same answers by torch's exchange interface, by its methods, and of a class of one's own."""
    b, i32, f32, bf = sm._calls(), torch.int32, torch.float32, torch.bfloat16
    capsule = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    assert capsule is not None                                                          # (this torch has it)
    types = (i32, f32, bf, torch.Tensor, torch.nn.Parameter)
    b.torch_types(*types, capsule if exchange else None)
    try:
        buf = torch.arange(480, dtype=f32).reshape(6, 80)
        for cls in (torch.Tensor, _Gpu):
            dev = 0 if cls is _Gpu else -1

            def t(x):
                return x if cls is torch.Tensor else x.as_subclass(_Gpu)
            assert b.row_stride(t(buf[:, 8:40].view(6, 4, 8)), f32, "x", 6, 4, 8) == 80
            assert b.row_stride(t(buf[:1, :32].view(1, 4, 8).requires_grad_()), f32, "x", 1, 4, 8) == 32
            assert b.row_stride(t(torch.zeros((0, 4, 8), dtype=bf)), bf, "x", 0, 4, 8) == 32
            assert b.row_stride(t(torch.zeros((3, 5), dtype=torch.float16)), torch.float16, "x", 3, 5) == 5
            for bad in (buf.t(), buf.double(), buf.int(), buf[:5], buf[:, ::2], buf.view(6, 8, 10)):
                with pytest.raises(sm.SpanMergeError, match="x: expected"):
                    b.row_stride(t(bad), f32, "x", 6, 80)
            b.need(t(buf), 480, "x")
            b.need(t(torch.zeros(())), 1, "x")
            with pytest.raises(sm.SpanMergeError, match="x: expected 481 values, got 480"):
                b.need(t(buf), 481, "x")
            gain = t(buf[1])
            assert b.parameter(gain, f32, 80, dev, "g") == gain.data_ptr() and b.parameter(None, f32, 80, dev, "g") == 0
            for bad in ((gain, bf, 80, dev), (gain, f32, 79, dev), (gain, f32, 80, 1), (t(buf[:, 0]), f32, 6, dev)):
                with pytest.raises(sm.SpanMergeError):
                    b.parameter(*bad, "g")
        param = torch.nn.Parameter(torch.zeros(7))
        assert b.parameter(param, f32, 7, -1, "g") == param.data_ptr()
    finally:
        b.torch_types(*types, capsule)


def test_a_norm_follows_its_tensors(L):
    gain = _gpu(8)
    n = sm.norm_params("rms", gain)

    def look():
        return sm.NormParams.from_buffer_copy(n.look(sm._calls(), torch.float32, 8, 0, "pre"))
    first = look()
    assert first.gain == gain.data_ptr() and first.bias is None and first.kind == 0
    old, gain.data = gain.data, _gpu(8)
    assert look().gain == gain.data_ptr() != old.data_ptr()
    gain.data = _gpu(16)[::2]
    with pytest.raises(sm.SpanMergeError, match="contiguous"):
        look()
    for other in (_gpu(9), _gpu(8, torch.bfloat16)):
        with pytest.raises(sm.SpanMergeError, match="pre: expected 8 values"):
            sm.norm_params("rms", other).look(sm._calls(), torch.float32, 8, 0, "pre")


def test_other_devices_are_refused(monkeypatch, L):
    x, pos, rope = _gpu((3, 2, 8)), _gpu(3, torch.int32), sm.rope_params(8)
    monkeypatch.setattr(sm, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(sm, "_device", lambda: 1)
    with pytest.raises(sm.SpanMergeError, match="current device 1"):
        sm.rotary(x, pos, rope, _gpu((3, 2, 8)))
    monkeypatch.setattr(sm, "_device", lambda: 0)
    with pytest.raises(sm.SpanMergeError, match="current device 0, got one on -1"):      # a CPU tensor
        sm.rotary(x, torch.zeros(3, dtype=torch.int32), rope, _gpu((3, 2, 8)))
    stream = type("S", (), dict(device_index=1, cuda_stream=0))()
    with pytest.raises(sm.SpanMergeError, match="stream"):
        sm.rotary(x, pos, rope, _gpu((3, 2, 8)), stream=stream)
    with pytest.raises(sm.SpanMergeError, match="post"):
        monkeypatch.setattr(sm, "_device", lambda: 2)
        sm.block_norm(_gpu((3, 8)), _gpu((3, 8)), _gpu((3, 8)), None, post=sm.norm_params("rms", _gpu(8)))


def test_caches_that_share_tables():
    kw = dict(dtype=torch.bfloat16, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=8, max_seqs=2,
              max_blocks_per_seq=4, device="cpu")
    sm_ptr, sm._ptr = sm._ptr, lambda t: t.data_ptr()
    try:
        a = sm.PagedCache(**kw)
        b = sm.PagedCache(**{**kw, "num_kv_heads": 1}, tables=a)                       # heads may differ
        assert b.block_table is a.block_table and b.lengths is a.lengths and b.free_stack is a.free_stack
        assert b.free_top is a.free_top and b.err is a.err and b.k_pool is not a.k_pool
        for other in (dict(block_size=32), dict(num_blocks=9), dict(max_seqs=3), dict(max_blocks_per_seq=5)):
            with pytest.raises(sm.SpanMergeError):
                sm.PagedCache(**{**kw, **other}, tables=a)
        with pytest.raises(sm.SpanMergeError):
            sm.PagedCache(**kw, tables=a, free_order=range(8))
    finally:
        sm._ptr = sm_ptr


def test_a_norm_follows_its_kind_and_epsilon(L):
    def look(n):
        return sm.NormParams.from_buffer_copy(n.look(sm._calls(), torch.float32, 8, 0, "pre"))
    for n in (sm.norm_params("rms"), sm.norm_params("rms", _gpu(8), _gpu(8))):
        first = look(n)
        n.eps = 0.25
        assert look(n).eps == 0.25 and look(n).kind == first.kind == 0 and look(n).gain == first.gain
        n.kind = sm.NORM_KINDS["layer"]
        assert look(n).kind == 1 and look(n).eps == 0.25 and look(n).bias == first.bias


def test_alternatives_of_other_shapes_are_refused(monkeypatch, L):
    monkeypatch.setattr(sm, "_here", lambda stream: (0, 0))
    i32, x, ws = torch.int32, _gpu((4, 100), torch.bfloat16), _gpu(65536, torch.uint8)
    for ids, tlp, name in (((4, 8), (4, 20), "top_logprobs"), ((4, 8), (2, 16), "top_logprobs"), ((4, 8), (32,), "top_logprobs"),
                           ((4,), (4, 2), "top_logprobs"), ((4, 8), (3, 8), "top_logprobs"), ((4, 8), (4, 1, 8), "top_logprobs"),
                           ((4, 2, 4), (4, 2, 4), "top_ids"), ((2, 2, 8), (4, 8), "top_ids"), ((3, 8), (4, 8), "top_ids"),
                           ((), (4,), "top_ids"), ((3,), (4,), "top_ids")):
        with pytest.raises(sm.SpanMergeError, match=name):
            sm.token_logprobs(x, None, None, None, _gpu(ids, i32), _gpu(tlp), ws)
    # as they may be: [rows, k], or [rows] for one alternative, with more rows behind (the argument checks then refuse
    # the call, whose workspace is too small, before anything is enqueued)
    for ids, tlp in (((4, 8), (4, 8)), ((6, 8), (5, 8)), ((4,), (4,)), ((4,), (4, 1)), ((4, 1), (4,)), ((4, 0), (4, 0))):
        with pytest.raises(sm.SpanMergeError, match="sm_token_logprobs"):
            sm.token_logprobs(x, None, None, None, _gpu(ids, i32), _gpu(tlp), ws[:65535])


def test_sizes_that_no_int_holds_are_refused(L):
    """2^32 rows more than none would count as none."""
    b, rope = sm._calls(), sm.rope_params(8)
    x, pos, many = torch.zeros((1, 2, 8)), torch.zeros(2, dtype=torch.int32), 1 << 32
    rows = (x,)
    args = {"sm_rotary": [rows, 16, pos, 0, 2, 8, rope, 0, 0, rows, 16, 0, -1],
            "sm_block_norm": [rows, 16, None, 0, 0, 16, None, None, 0, 1.0, bytes(sm.NormParams(0, 1e-5)), 0, rows, 16,
                              None, 0, 0, -1],
            "sm_token_logprobs": [rows, 16, 0, 16, 0, 1.0, None, None, None, 0, None, None, pos, 8, None, 0, -1]}
    sizes = {"sm_rotary": (3, 4, 5), "sm_block_norm": (4, 5), "sm_token_logprobs": (2, 3, 9)}
    for name, good in args.items():
        entry = getattr(b, name)
        assert entry(*good) == sm.SM_OK, name                                   # no row: nothing to do
        for at in sizes[name]:
            for off in (many, -many, 1 << 31, many << 32):
                bad = list(good)
                bad[at] += off
                with pytest.raises(sm.SpanMergeError, match="argument"):
                    entry(*bad)
