"""The entry points of the 8-bit decoder layer refuse what they cannot take before anything reaches a GPU."""
import pytest


@pytest.fixture(scope="module")
def E():
    from paper_2511_00603_b200 import build
    build.build()
    from paper_2511_00603_b200 import epara
    return epara


P = 1 << 20    # an address that is never read: every call below is refused on the host


def _norm(E, **k):
    a = dict(x=P, x_type=0, x_stride=64, resid=P, resid_stride=64, resid_out=P, resid_out_stride=64, gain=P, eps=1e-5, q=P, q_stride=64, scales=P, rows=2, d=64)
    a.update(k)
    return E.lib.epara_rms_norm_i8(0, None, *a.values())


@pytest.mark.parametrize("bad", [dict(x=None), dict(q=None), dict(scales=None), dict(rows=-1), dict(d=0), dict(x_type=2), dict(x_stride=63), dict(q_stride=63),
                                 dict(resid_stride=63), dict(resid_out_stride=1), dict(resid=None), dict(x=P + 1), dict(x_type=1, x=P + 2), dict(scales=P + 2),
                                 dict(resid=P + 2), dict(gain=P + 1), dict(eps=-1.0), dict(eps=float("nan"))])
def test_norm_refuses(E, bad):
    assert _norm(E, **bad) == E.E_INVALID


def test_empty_calls_are_fine(E):
    assert _norm(E, rows=0) == E.OK
    assert _gemm(E, M=0) == E.OK
    assert _append(E, B=0, T=0) == E.OK and _append(E, T=0, q_rows=P) == E.OK
    assert _attn(E, B=0, T=0) == E.OK
    # tensors without elements have no address
    assert _norm(E, rows=0, x=None, q=None, scales=None) == E.OK and _gemm(E, M=0, A=None, C=None, a_scale=None) == E.OK
    assert _append(E, B=0, T=0, k=None, v=None, lens=None, tables=None) == E.OK and _attn(E, B=0, T=0, q=None, out=None, lens=None, tables=None) == E.OK


def test_norm_takes_no_other_type_for_bf16(E):
    import torch
    x = torch.zeros((1, 8), dtype=torch.float16)
    with pytest.raises(TypeError):
        E.epara_rms_norm_i8(x, None, torch.zeros((1, 8), dtype=torch.int8), torch.zeros(1), 0, device=0)


def test_layouts_that_the_calls_cannot_see(E):
    import torch
    one, st = torch.zeros(1), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        E.epara_rms_norm_i8(torch.zeros((8, 4)).t(), None, torch.zeros((4, 8), dtype=torch.int8), torch.zeros(4), 0, device=0)
    with pytest.raises(ValueError):
        E.epara_rms_norm_i8(torch.zeros((4, 8)), None, torch.zeros((4, 16), dtype=torch.int8)[:, ::2], torch.zeros(4), 0, device=0)
    layer, x = torch.zeros((3, 2, 4, 16, 64), dtype=torch.float8_e4m3fn), torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    for bad in (x[:, ::2], x, x[:, :4, :32]):
        with pytest.raises(ValueError):
            E.epara_kv8_append(bad, x[:, 4:], layer, one, st, st[None], 16, st, 0, device=0)
    with pytest.raises(ValueError):
        E.epara_kv8_append(x[:, :4], x[:, 4:], layer.view(6, 2, 4, 8, 64), one, st, st[None], 16, st, 0, device=0)
    with pytest.raises(ValueError):
        E.epara_kv8_attention(x.view(2, 512), layer, one, st, st[None], torch.zeros((2, 1024), dtype=torch.bfloat16)[:, :512], 8, 4, 64, 16, None, st, 0, device=0)


def _gemm(E, status=P, **k):
    a = dict(A=P, W=P, a_scale=P, w_scale=P, C=P, bias=P, M=3, N=32, K=48, lda=48, ldw=48, ldc=32, epilogue=0)
    a.update(k)
    return E.lib.epara_gemm_i8(0, None, E.GemmI8Problem(*a.values()), status)


@pytest.mark.parametrize("bad", [dict(A=None), dict(W=None), dict(C=None), dict(a_scale=None), dict(w_scale=None), dict(M=-1), dict(N=0), dict(K=0), dict(lda=40, K=40),
                                 dict(ldw=56), dict(lda=32), dict(A=P + 8), dict(W=P + 4), dict(C=P + 2), dict(a_scale=P + 4), dict(w_scale=P + 4),
                                 dict(epilogue=1, bias=None), dict(epilogue=1, bias=P + 2), dict(epilogue=16), dict(epilogue=12), dict(epilogue=4, N=33), dict(ldc=31),
                                 dict(epilogue=4, ldc=15), dict(status=None), dict(status=P + 2)])
def test_gemm_refuses(E, bad):
    assert _gemm(E, **bad) == E.E_INVALID


def test_sizes_beyond_what_is_counted_in_32_bits(E):
    assert _gemm(E, K=E.GEMM_I8_MAX_K + 1, lda=1 << 18, ldw=1 << 18) == E.E_UNSUPPORTED          # sums past 31 bits
    assert _gemm(E, M=(1 << 31) - 1, N=1 << 20, ldc=1 << 20) == E.E_UNSUPPORTED
    assert _gemm(E, N=(1 << 30) + 1, ldc=(1 << 31) - 1) == E.E_UNSUPPORTED and _gemm(E, M=(1 << 30) + 1) == E.E_UNSUPPORTED
    big = (1 << 30) + 8
    assert _norm(E, d=big, x_stride=big, resid_stride=big, resid_out_stride=big, q_stride=big) == E.E_UNSUPPORTED
    for call in (_append, _attn):
        assert call(E, max_len=big, table_stride=1 << 27) == E.E_UNSUPPORTED
    for B, T, Hq, Hkv, q in ((1, 1 << 25, 1 << 15, 1, 1 << 25), (1 << 30, 1 << 30, 8, 2, 1 << 30), (1 << 20, 1 << 20, 1 << 14, 1 << 14, 1), (2, 2, 1 << 30, 1 << 30, 1)):
        assert E.epara_kv8_attention_scratch_bytes(B, T, Hq, Hkv, 64, q, 4096) == 0
        assert _attn(E, B=B, T=T, Hq=Hq, Hkv=Hkv, hd=64, max_q=q, max_len=4096, table_stride=256, q_rows=P, q_stride=(1 << 31) - 8) == E.E_UNSUPPORTED


def _append(E, **k):
    a = dict(k=P, k_stride=256, v=P, v_stride=256, kv8=P, scales=P, pages=10, q_rows=None, lens=P, tables=P, table_stride=4, B=2, T=2, Hkv=2, hd=128, max_q=1,
             max_len=64, status=P)
    a.update(k)
    return E.lib.epara_kv8_append(0, None, *a.values())


def _attn(E, **k):
    a = dict(q=P, q_stride=1024, kv8=P, scales=P, pages=10, q_rows=None, lens=P, tables=P, table_stride=4, out=P, B=2, T=2, Hq=8, Hkv=2, hd=128, max_q=1, max_len=64,
             scratch=P, scratch_bytes=1 << 30, status=P)
    a.update(k)
    return E.lib.epara_kv8_attention(0, None, *a.values())


CACHE = [dict(kv8=None), dict(scales=None), dict(lens=None), dict(tables=None), dict(status=None), dict(pages=0), dict(B=-1), dict(T=-1), dict(Hkv=0), dict(hd=0),
         dict(max_q=0), dict(max_len=0), dict(kv8=P + 8), dict(scales=P + 2), dict(q_rows=P + 2), dict(lens=P + 2), dict(tables=P + 1), dict(status=P + 2),
         dict(table_stride=3), dict(max_q=2), dict(T=3)]


@pytest.mark.parametrize("bad", CACHE + [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(k_stride=257), dict(v_stride=252), dict(k_stride=248)])
def test_append_refuses(E, bad):
    assert _append(E, **bad) == E.E_INVALID


@pytest.mark.parametrize("bad", CACHE + [dict(q=None), dict(out=None), dict(Hq=0), dict(Hq=7), dict(q=P + 8), dict(q_stride=1025), dict(q_stride=1016), dict(out=P + 1)])
def test_attention_refuses(E, bad):
    assert _attn(E, **bad) == E.E_INVALID


def test_cache_calls_refuse_other_head_sizes(E):
    assert _append(E, hd=96) == E.E_UNSUPPORTED and _attn(E, hd=32) == E.E_UNSUPPORTED


def test_attention_asks_for_its_scratch(E):
    need = E.epara_kv8_attention_scratch_bytes(2, 2, 8, 2, 128, 1, 131072)
    assert need > 0
    big = dict(max_len=131072, table_stride=8192)
    assert _attn(E, scratch_bytes=need - 1, **big) == E.E_RESOURCE
    assert _attn(E, scratch=None, scratch_bytes=need, **big) == E.E_INVALID
    assert _attn(E, scratch=P + 4, scratch_bytes=need, **big) == E.E_INVALID
    assert E.epara_kv8_attention_scratch_bytes(2, 2, 8, 2, 128, 1, 64) == 0       # a single chunk needs none
    assert E.epara_kv8_attention_scratch_bytes(2, 2, 7, 2, 128, 1, 64) == 0


def test_calls_without_ctypes_take_what_ctypes_takes(E):
    """The compiled forms of the four calls: the same answers for the same arguments, and Python errors for wrong ones."""
    fast = pytest.importorskip("paper_2511_00603_b200._fastcall")
    assert E._norm_i8.__name__ == "epara_rms_norm_i8" and not hasattr(E._gemm_i8, "argtypes") and fast
    norm = [0, None, P, 0, 64, P, 64, P, 64, P, 1e-5, P, 64, P, 0, 64]
    gemm = [0, None, P, P, P, P, P, None, 0, 32, 48, 48, 48, 32, 0, P]
    append = [0, None, P, 256, P, 256, P, P, 10, None, P, P, 4, 0, 0, 2, 128, 1, 64, P]
    attn = [0, None, P, 1024, P, P, 10, None, P, P, 4, P, 0, 0, 8, 2, 128, 1, 64, None, 0, P]
    general = [E.lib.epara_rms_norm_i8, E._gemm_i8_ctypes, E.lib.epara_kv8_append, E.lib.epara_kv8_attention]
    for call, plain, args in zip((E._norm_i8, E._gemm_i8, E._kv8_append, E._kv8_attention), general, (norm, gemm, append, attn)):
        assert call(*args) == plain(*args) == E.OK
        for i in range(2, len(args)):
            pointer = args[i] is None or args[i] == P
            for other in ((None, P + 1) if pointer else (0.5,) if call is E._norm_i8 and i == 10 else (-7, 1 << 30)):
                a = args[:i] + [other] + args[i + 1:]
                if (call is E._norm_i8 and i == 14 or call is E._gemm_i8 and i == 8) and other > 0:
                    continue                               # (rows to work on: such a call would go on to the GPU)
                assert call(*a) == plain(*a), (call, i, other)
        with pytest.raises(TypeError):
            call(*args[:-1])
        with pytest.raises(TypeError):
            call(*args[:2], "7", *args[3:])
        with pytest.raises(OverflowError):
            call(1 << 40, *args[1:])
