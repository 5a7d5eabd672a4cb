"""What the binding of the 8-bit decoder layer makes of its tensors: layouts, types and devices that the C calls cannot see are refused, the others
arrive as they are.  Nothing is called: the four entry points are replaced by one that keeps its arguments."""
import pytest
import torch

bf, f32, i8, i32 = torch.bfloat16, torch.float32, torch.int8, torch.int32


@pytest.fixture()
def E(monkeypatch):
    from paper_2511_00603_b200 import build
    build.build()
    from paper_2511_00603_b200 import epara
    seen = []

    def keep(*args):
        seen.append(args)
        return 0

    for name in ("_norm_i8", "_gemm_i8", "_kv8_append", "_kv8_attention"):
        monkeypatch.setattr(epara, name, keep)
    monkeypatch.setattr(epara, "seen", seen, raising=False)
    return epara


def _norm(E, **k):
    a = dict(x=torch.zeros((4, 64)), gain=torch.zeros(64, dtype=bf), q=torch.zeros((4, 64), dtype=i8), scales=torch.zeros(4), resid=torch.zeros((4, 64)),
             resid_out=torch.zeros((4, 64)))
    a.update(k)
    E.epara_rms_norm_i8(a["x"], a["gain"], a["q"], a["scales"], 0, resid=a["resid"], resid_out=a["resid_out"])
    return E.seen[-1]


def _gemm(E, **k):
    a = dict(A=torch.zeros((4, 64), dtype=i8), W=torch.zeros((32, 64), dtype=i8), a_scale=torch.zeros(4), w_scale=torch.zeros(32), C=torch.zeros((4, 32), dtype=bf),
             bias=torch.zeros(32, dtype=bf), M=4, N=32, K=64, epilogue=1)
    status = k.pop("status", torch.zeros(1, dtype=i32))
    a.update(k)
    E.epara_gemm_i8(a, 0, status)
    return E.seen[-1]


def _tables(k):
    a = dict(layer=torch.zeros((9, 2, 2, 16, 64), dtype=torch.float8_e4m3fn), scales=torch.zeros((9, 2, 2)), lens=torch.ones(3, dtype=i32), tables=torch.zeros((3, 4), dtype=i32),
             status=torch.zeros(1, dtype=i32), q_rows=torch.arange(4, dtype=i32), kv_pages=0)
    a.update(k)
    return a


def _append(E, **k):
    a = _tables(dict(k=torch.zeros((3, 2, 64), dtype=bf), v=torch.zeros((3, 2, 64), dtype=bf)))
    a.update(k)
    E.epara_kv8_append(a["k"], a["v"], a["layer"], a["scales"], a["lens"], a["tables"], 64, a["status"], 0, q_rows=a["q_rows"], kv_pages=a["kv_pages"])
    return E.seen[-1]


def _attend(E, **k):
    a = _tables(dict(q=torch.zeros((3, 256), dtype=bf), out=torch.zeros((3, 256), dtype=bf), scratch=None))
    a.update(k)
    E.epara_kv8_attention(a["q"], a["layer"], a["scales"], a["lens"], a["tables"], a["out"], 4, 2, 64, 64, a["scratch"], a["status"], 0, q_rows=a["q_rows"], kv_pages=a["kv_pages"])
    return E.seen[-1]


def _refused(E, call, error, **bad):
    n = len(E.seen)
    with pytest.raises(error):
        call(E, **bad)
    assert len(E.seen) == n


def _wide(rows, cols, dtype):
    """Every second element of a row."""
    return torch.zeros((rows, 2 * cols), dtype=dtype)[:, ::2]


class _Elsewhere(torch.Tensor):
    """A tensor that says it lies on another device than the others."""

    def get_device(self):
        return 3


@pytest.mark.parametrize("name,tensor", [("q", _wide(4, 64, i8)), ("resid", _wide(4, 64, f32)), ("resid_out", _wide(4, 64, f32)), ("x", _wide(4, 64, f32)), ("gain", torch.zeros(128, dtype=bf)[::2]),
                                         ("scales", torch.zeros(8)[::2]), ("scales", torch.zeros(3)), ("gain", torch.zeros(63, dtype=bf)), ("resid", torch.zeros((3, 64))),
                                         ("resid_out", torch.zeros((4, 63))), ("q", torch.zeros((3, 64), dtype=i8)), ("resid", torch.zeros((64, 4)).t())])
def test_norm_refuses_layouts(E, name, tensor):
    _refused(E, _norm, ValueError, **{name: tensor})


@pytest.mark.parametrize("name,tensor", [("q", torch.zeros((4, 64), dtype=torch.uint8)), ("resid", torch.zeros((4, 64), dtype=bf)), ("resid_out", torch.zeros((4, 64), dtype=bf)),
                                         ("gain", torch.zeros(64)), ("scales", torch.zeros(4, dtype=torch.float64)), ("x", torch.zeros((4, 64), dtype=torch.float16))])
def test_norm_refuses_types(E, name, tensor):
    _refused(E, _norm, TypeError, **{name: tensor})


@pytest.mark.parametrize("name,tensor", [("A", _wide(4, 64, i8)), ("W", _wide(32, 64, i8)), ("C", _wide(4, 32, bf)), ("a_scale", torch.zeros(8)[::2]), ("w_scale", torch.zeros(64)[::2]),
                                         ("bias", torch.zeros(64, dtype=bf)[::2]), ("A", torch.zeros((3, 64), dtype=i8)), ("A", torch.zeros((4, 48), dtype=i8)), ("W", torch.zeros((31, 64), dtype=i8)),
                                         ("C", torch.zeros((4, 31), dtype=bf)), ("C", torch.zeros((3, 32), dtype=bf)), ("a_scale", torch.zeros(3)), ("w_scale", torch.zeros(31))])
def test_product_refuses_layouts(E, name, tensor):
    _refused(E, _gemm, ValueError, **{name: tensor})


@pytest.mark.parametrize("name,tensor", [("A", torch.zeros((4, 64), dtype=torch.uint8)), ("W", torch.zeros((32, 64))), ("C", torch.zeros((4, 32))), ("a_scale", torch.zeros(4, dtype=bf)),
                                         ("w_scale", torch.zeros(32, dtype=bf)), ("bias", torch.zeros(32)), ("status", torch.zeros(1, dtype=torch.int64))])
def test_product_refuses_types(E, name, tensor):
    _refused(E, _gemm, TypeError, **{name: tensor})


def test_product_wants_an_fp32_stream_and_half_the_columns_of_a_gated_one(E):
    _gemm(E, epilogue=8, C=torch.zeros((4, 32)))
    _refused(E, _gemm, TypeError, epilogue=8)
    _gemm(E, epilogue=4, C=torch.zeros((4, 16), dtype=bf))
    _refused(E, _gemm, ValueError, epilogue=4, C=torch.zeros((4, 15), dtype=bf))


POOL = torch.zeros((9, 3, 2, 2, 16, 64), dtype=torch.float8_e4m3fn)
CACHE_LAYOUTS = [("layer", POOL[:, 1]), ("scales", torch.zeros((9, 3, 2, 2))[:, 1]), ("scales", torch.zeros((8, 2, 2))), ("lens", torch.ones(6, dtype=i32)[::2]),
                 ("tables", _wide(3, 4, i32)), ("tables", torch.zeros((2, 4), dtype=i32)), ("q_rows", torch.zeros(3, dtype=i32)),
                 ("q_rows", torch.zeros(8, dtype=i32)[::2]), ("kv_pages", 10)]
CACHE_TYPES = [("layer", POOL[:, 1].to(torch.float16).contiguous()), ("scales", torch.zeros((9, 2, 2), dtype=bf)), ("lens", torch.ones(3, dtype=torch.int64)),
               ("tables", torch.zeros((3, 4), dtype=torch.int64)), ("q_rows", torch.arange(4)), ("status", torch.zeros(1, dtype=torch.int64))]


@pytest.mark.parametrize("name,value", CACHE_LAYOUTS + [("k", torch.zeros((3, 2, 128), dtype=bf)[:, :, ::2]), ("v", torch.zeros((3, 2, 128), dtype=bf)[:, :, ::2]), ("v", torch.zeros((2, 2, 64), dtype=bf)),
                                                        ("v", torch.zeros((2, 3, 64), dtype=bf).transpose(0, 1)), ("layer", torch.zeros((9, 2, 2, 8, 64), dtype=torch.float8_e4m3fn))])
def test_append_refuses_layouts(E, name, value):
    _refused(E, _append, ValueError, **{name: value})


@pytest.mark.parametrize("name,value", CACHE_TYPES + [("k", torch.zeros((3, 2, 64))), ("v", torch.zeros((3, 2, 64), dtype=torch.float16))])
def test_append_refuses_types(E, name, value):
    _refused(E, _append, TypeError, **{name: value})


@pytest.mark.parametrize("name,value", CACHE_LAYOUTS + [("q", _wide(3, 256, bf)), ("q", torch.zeros((3, 255), dtype=bf)), ("out", _wide(3, 256, bf)), ("out", torch.zeros((3, 255), dtype=bf)),
                                                        ("out", torch.zeros((3, 264), dtype=bf)[:, :256]), ("layer", torch.zeros((9, 2, 1, 16, 64), dtype=torch.float8_e4m3fn))])
def test_attention_refuses_layouts(E, name, value):
    _refused(E, _attend, ValueError, **{name: value})


@pytest.mark.parametrize("name,value", CACHE_TYPES + [("q", torch.zeros((3, 256))), ("out", torch.zeros((3, 256)))])
def test_attention_refuses_types(E, name, value):
    _refused(E, _attend, TypeError, **{name: value})


DEFAULTS = dict(gain=torch.zeros(64, dtype=bf), q=torch.zeros((4, 64), dtype=i8), scales=torch.zeros(4), resid=torch.zeros((4, 64)), resid_out=torch.zeros((4, 64)),
                W=torch.zeros((32, 64), dtype=i8), a_scale=torch.zeros(4), w_scale=torch.zeros(32), C=torch.zeros((4, 32), dtype=bf), bias=torch.zeros(32, dtype=bf),
                status=torch.zeros(1, dtype=i32))


@pytest.mark.parametrize("call,names", [(_norm, ("gain", "q", "scales", "resid", "resid_out")), (_gemm, ("W", "a_scale", "w_scale", "C", "bias", "status")),
                                        (_append, ("v", "layer", "scales", "lens", "tables", "q_rows", "status")),
                                        (_attend, ("out", "scratch", "layer", "scales", "lens", "tables", "q_rows", "status"))])
def test_tensors_of_another_device_are_refused(E, call, names):
    """What is passed on is an address: a kernel would read it on its own device."""
    cache = call in (_append, _attend)
    ours = _tables(dict(v=torch.zeros((3, 2, 64), dtype=bf), out=torch.zeros((3, 256), dtype=bf), scratch=torch.zeros(16, dtype=torch.uint8))) if cache else DEFAULTS
    call(E)
    for name in names:
        _refused(E, call, ValueError, **{name: ours[name].as_subclass(_Elsewhere)})


def test_what_arrives(E):
    """Row distances; of a single row they are not the tensor's, which may have any."""
    x = torch.zeros((4, 80))[:, 8:72]
    a = _norm(E, x=x, resid=torch.zeros((4, 100))[:, :64])
    assert a[2] == x.data_ptr() and a[4] == 80 and a[6] == 100 and a[8] == 64 and a[12] == 64
    one = torch.zeros((64, 1)).t()                          # [1, 64] with a row distance of 1
    a = _norm(E, x=one, q=torch.zeros((1, 64), dtype=i8), scales=torch.zeros(1), resid=torch.zeros((1, 64)), resid_out=torch.zeros((1, 64)))
    assert a[4] >= 64 and a[14] == 1
    a = _gemm(E, A=torch.zeros((6, 96), dtype=i8)[1:5, :64], C=torch.zeros((4, 40), dtype=bf)[:, :32], a_scale=torch.zeros((4, 1)), w_scale=torch.zeros((1, 32)))
    assert a[11] == 96 and a[12] == 64 and a[13] == 40
    a = _gemm(E, A=torch.zeros((1, 60), dtype=i8), a_scale=torch.zeros(1), C=torch.zeros((1, 32), dtype=bf), M=1, K=60)      # one row: of any length
    assert a[11] == 64 and a[13] >= 32
    qkv = torch.zeros((3, 8, 64), dtype=bf)
    a = _append(E, k=qkv[:, 4:6], v=qkv[:, 6:])
    assert a[2] == qkv[:, 4:6].data_ptr() and a[3] == a[5] == 512 and a[8] == 9 and a[12] == 4
    head_first = torch.zeros((2, 1, 64), dtype=bf).transpose(0, 1)                # [1, 2, 64] with a row distance of 64
    a = _append(E, k=head_first, v=head_first, lens=torch.ones(1, dtype=i32), tables=torch.zeros((1, 4), dtype=i32), q_rows=None, kv_pages=5)
    assert a[3] == a[5] == 128 and a[8] == 5 and a[9] is None and a[12] == 4
    a = _attend(E, q=qkv.view(3, 512)[:, :256], tables=torch.zeros((3, 7), dtype=i32)[:, :4], scratch=torch.zeros(80, dtype=torch.uint8))
    assert a[3] == 512 and a[10] == 7 and a[20] == 80
    buffers = dict(q_rows=torch.zeros(9, dtype=i32), tables=torch.zeros((8, 4), dtype=i32), out=torch.zeros((8, 256), dtype=bf))           # larger than the call needs
    assert _attend(E, **buffers)[12] == 3
    assert _norm(E, q=torch.zeros((9, 72), dtype=i8), scales=torch.zeros(9), resid=torch.zeros((5, 64)))[12] == 72
    assert _attend(E, q=qkv[:, :4])[3] == 512 and _attend(E, out=torch.zeros((3, 4, 64), dtype=bf))
    assert _attend(E, layer=torch.zeros((9, 2, 2, 16, 64), dtype=torch.uint8))


@pytest.mark.parametrize("max_q", [1, 64])
@pytest.mark.parametrize("max_len", [(1 << 30) + 1, (1 << 31) - 1])
def test_no_scratch_for_lengths_that_no_call_takes(max_q, max_len):
    from paper_2511_00603_b200 import epara
    assert epara.epara_kv8_attention_scratch_bytes(1, max_q, 8, 2, 128, max_q, max_len) == 0
    assert epara.epara_kv8_attention_scratch_bytes(1, max_q, 8, 2, 128, max_q, 1 << 30) < 1 << 40
