"""The operators of the 8-bit decoder layer on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F64 = torch.float64
HALF_BF16, HALF_F16, HALF_F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24     # half a step, relative


@pytest.fixture(scope="module")
def E():
    from paper_2511_00603_b200 import build
    build.build()
    from paper_2511_00603_b200 import epara
    return epara


def _st():
    return torch.cuda.current_stream().cuda_stream


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _within(got, want, tol, what=""):
    """Element by element; where the definition gives NaN the output has to be NaN."""
    got = got.to(F64)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    over = ((got - want).abs() - tol)[~nan]
    assert over.numel() == 0 or over.max().item() <= 0, f"{what}: {over.max().item():.3g} over its tolerance"


# ------------------------------------------------------------------------------------------------ norm
def _check_norm(x, r, gain, q, s, r_out, eps=1e-5):
    d = x.shape[1]
    h = x.to(F64)
    if r is not None:
        h32 = x.float() + r
        if r_out is not None:
            assert torch.equal(r_out, h32)                 # one addition, rounded once
        h = h32.to(F64)                                    # (what the norm is defined on: the stored sum)
    y = h * gain.to(F64) / torch.sqrt(h.square().mean(1, keepdim=True) + eps) if gain is not None else h
    want = torch.clamp(y.abs().amax(1) / 127, min=2.0 ** -126)
    # sum of squares in fp32: at most 128 additions on the way of a value (a thread's, the block's), halved by the root; the products
    # and the division around it add a few roundings
    rel = 80 * HALF_F32
    _within(s, want, rel * want, "scale")
    # a code is the nearest to y / s, where y and s are off by as much
    assert ((q.to(F64) - y / want[:, None]).abs() <= 0.5 + 127 * 2 * rel).all()


@pytest.mark.parametrize("rows", [1, 5, 300])
@pytest.mark.parametrize("d", [1, 7, 64, 100, 200, 1000, 1111, 1112, 2048, 4092, 4096, 4097, 8200, 8205, 16384, 16400, 20001])
@pytest.mark.parametrize("x_type,resid", [("bf16", True), ("bf16", False), ("f32", True)])
def test_norm(E, rows, d, x_type, resid):
    g = _gen(rows * 31 + d)
    x = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16 if x_type == "bf16" else torch.float32)
    r = 2 * torch.randn((rows, d), generator=g, device="cuda") if resid else None
    gain = (1 + 0.3 * torch.randn((d,), generator=g, device="cuda")).to(torch.bfloat16)
    q = torch.full((rows, d), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(rows, device="cuda")
    r_out = torch.empty_like(r) if resid else None
    for gn in (gain, None):
        E.epara_rms_norm_i8(x, gn, q, s, _st(), resid=r, resid_out=r_out)
        _check_norm(x, r, gn, q, s, r_out)
    if resid:                                              # in place, and without writing the sum back
        keep = r.clone()
        E.epara_rms_norm_i8(x, gain, q, s, _st(), resid=r)
        assert torch.equal(r, keep)
        _check_norm(x, keep, gain, q, s, None)
        E.epara_rms_norm_i8(x, gain, q, s, _st(), resid=r, resid_out=r)
        _check_norm(x, keep, gain, q, s, r)


@pytest.mark.parametrize("d", [1023, 4095, 4097, 90])
def test_norm_does_not_see_what_stands_behind_the_gain(E, d):
    rows, room = 300, torch.full((d + 8,), math.nan, dtype=torch.bfloat16, device="cuda")
    room[:d] = (1 + 0.3 * torch.randn((d,), generator=_gen(d), device="cuda")).to(torch.bfloat16)
    x = torch.randn((rows, d), generator=_gen(d + 1), device="cuda")
    q, s = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    E.epara_rms_norm_i8(x, room[:d], q, s, _st())
    _check_norm(x, None, room[:d], q, s, None)


@pytest.mark.parametrize("d", [64, 4096, 1001])
def test_norm_strides_and_what_stands_beside(E, d):
    rows, g = 37, _gen(d)
    wide = torch.randn((rows, d + 24), generator=g, device="cuda").to(torch.bfloat16)
    r = torch.randn((rows, 2 * d), generator=g, device="cuda")
    q = torch.full((rows + 1, d + 40), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 1,), -5.0, device="cuda")
    for off in (0, 8, 3):
        x = wide[:, off:off + d]
        E.epara_rms_norm_i8(x, None, q[:rows, off:off + d], s[:rows], _st(), resid=r[:, d:])
        _check_norm(x, r[:, d:], None, q[:rows, off:off + d], s[:rows], None)
        assert (q[:rows, :off] == 77).all() and (q[:rows, off + d:] == 77).all() and (q[rows] == 77).all() and s[rows] == -5
        q.fill_(77)


@pytest.mark.parametrize("d", [64, 4096, 999, 20000])
def test_norm_of_zeros_and_of_what_is_not_finite(E, d):
    x = torch.randn((6, d), device="cuda").float()
    x[1] = 0
    x[2, d // 2] = float("nan")
    x[3, 0] = float("inf")
    x[4] = 1e30                                            # squares overflow fp32
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    q, s = torch.full((6, d), 5, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    E.epara_rms_norm_i8(x, gain, q, s, _st())
    assert torch.isnan(s).tolist() == [False, False, True, True, True, False]
    assert (q[1:5] == 0).all() and q[0].abs().max() == 127 and q[5].abs().max() == 127 and s[1] == 2.0 ** -126
    E.epara_rms_norm_i8(x, None, q, s, _st())
    assert torch.isnan(s).tolist() == [False, False, True, True, False, False] and (q[1:4] == 0).all() and (q[4] == 127).all()
    x = torch.full((1, d), 1e-41, device="cuda")           # subnormal: the scale does not vanish
    E.epara_rms_norm_i8(x, None, q[:1], s[:1], _st())
    assert s[0] == 2.0 ** -126 and (q[0] == 0).all()
    x.fill_(2e-39)                                         # 316 times that, the norm's 1 / sqrt(eps), over the smallest scale: 54
    E.epara_rms_norm_i8(x, gain, q[:1], s[:1], _st())
    assert s[0] == 2.0 ** -126 and (q[0] == round(2e-39 * 1e-5 ** -0.5 * 2.0 ** 126)).all()


# ------------------------------------------------------------------------------------------------ product
def _gemm_case(M, N, K, epi, seed, pad=0, dev="cuda"):
    g = _gen(seed)
    ld = (K + 15) // 16 * 16 + pad

    def int8(rows):
        return torch.randint(-128, 128, (rows, ld), generator=g, device=dev, dtype=torch.int8)     # (the pad behind K too)

    p = dict(A=int8(max(M, 1)), W=int8(N), M=M, N=N, K=K, epilogue=epi)
    p["a_scale"] = (0.5 + torch.rand((max(M, 1),), generator=g, device=dev)) / 64
    p["w_scale"] = (0.5 + torch.rand((N,), generator=g, device=dev)) / (64 * math.sqrt(K))
    p["bias"] = torch.randn((N,), generator=g, device=dev).to(torch.bfloat16) if epi & 1 else None
    cols = N // 2 if epi & 4 else N
    p["C"] = torch.randn((max(M, 1), cols), generator=g, device=dev) if epi & 8 else torch.full((max(M, 1), cols), 7.0, dtype=torch.bfloat16, device=dev)
    return p


def _check_gemm(p, before):
    M, K, epi = p["M"], p["K"], p["epilogue"]
    acc = p["A"][:M, :K].to(F64) @ p["W"][:, :K].to(F64).t()
    v = acc * p["a_scale"][:M, None].to(F64) * p["w_scale"].to(F64)
    tol = 4 * HALF_F32 * v.abs()                           # the sum to fp32, two factors, the bias's addition
    if epi & 1:
        v = v + p["bias"].to(F64)
        tol = tol + HALF_F32 * v.abs()
    if epi & 2:
        # the device's GELU: its formula within 2.6e-5 of the erf form, the hardware tanh within 2^-11 of tanh
        tol = 1.2 * tol + 2.6e-5 + 0.5 * v.abs() * 2.0 ** -11 + 4 * HALF_F32 * v.abs()
        v = 0.5 * v * torch.special.erfc(-v / math.sqrt(2))
    if epi & 4:
        gate, up = v[:, 0::2], v[:, 1::2]
        tg, tu = tol[:, 0::2], tol[:, 1::2]
        sg = torch.sigmoid(gate)
        # |d silu| <= 1.1; exp with a relative error of (2 + |x|) 2^-22 and a division of 2 ulp
        tol = 1.1 * tg * up.abs() + gate.abs() * sg * tu + (gate * sg * up).abs() * (6 + gate.abs()) * 2.0 ** -22 + 2.0 ** -126
        v = gate * sg * up
    if epi & 8:
        v = before.to(F64) + v
        tol = tol + HALF_F32 * v.abs()
    else:
        tol = tol + HALF_BF16 * (v.abs() + tol)
    _within(p["C"][:M], v, tol, f"M={M} N={p['N']} K={K} epi={epi}")


SHAPES = [
    (0, 64, 64), (1, 1, 1), (1, 16, 16), (1, 4096, 4096), (3, 10, 511), (8, 1000, 776), (9, 257, 4099), (16, 2048, 8200), (16, 17, 33),
    (17, 128, 128), (17, 40, 16), (31, 1000, 777), (33, 4097, 513), (64, 512, 8192), (96, 6144, 4096), (128, 2048, 14336), (129, 130, 260), (200, 1000, 100),
    (257, 512, 1025), (394, 1000, 776), (512, 2048, 2048), (513, 1000, 777), (1000, 130, 4096), (1024, 4096, 128), (2000, 2050, 513), (4100, 260, 260),
    (1030, 2050, 260), (600, 5000, 2000), (2100, 1500, 130),         # pairs, 160, 224 and 192 columns
    (8200, 2048, 300), (3000, 5000, 140),                            # ... with several tiles each
    (192, 2048, 14336), (250, 900, 4096), (100, 30000, 300),         # swapped operands: wide tiles in four ranges; two CTAs to an SM in several rounds
    (45, 13213, 456), (75, 16232, 1614), (40, 29951, 267), (258, 11962, 3762), (516, 6171, 1000),       # ... one range; one and two CTAs to an SM
    (37, 5011, 1486), (71, 7143, 1945), (262, 3135, 6150), (33, 2388, 1014), (33, 19368, 2342),         # ... two
    (683, 129, 1870), (793, 271, 2828), (935, 531, 6041), (21, 9653, 10547), (33, 1173, 7516), (652, 146, 10982),       # ... four and eight
]


@pytest.mark.parametrize("epi", [0, 1, 2, 3, 4, 5, 8, 9, 11])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm(E, M, N, K, epi):
    if epi & 4 and N % 2:
        N += 1
    p, st = _gemm_case(M, N, K, epi, M * 7 + N + K + epi), _status()
    before = p["C"].clone()
    E.epara_gemm_i8(p, _st(), st)
    _check_gemm(p, before)
    assert st.item() == 0
    if M == 0:
        assert torch.equal(p["C"], before)


@pytest.mark.parametrize("epi", [0, 4, 8, 3])
@pytest.mark.parametrize("M", [5, 16, 40, 150, 700])
def test_gemm_strides_and_what_stands_beside(E, M, epi):
    """C inside a larger tensor whose rows start at any element; pads of A and W hold anything."""
    N, K = 200, 300
    for ldc_pad in (1, 2, 8, 13):
        p, st = _gemm_case(M, N, K, epi, M + epi, pad=32), _status()
        cols = p["C"].shape[1]
        big = torch.full((M + 2, cols + ldc_pad), 3.0, dtype=p["C"].dtype, device="cuda")
        big[:M, :cols] = p["C"]
        before = big[:M, :cols].clone()
        p["C"] = big[:, :cols]
        E.epara_gemm_i8(p, _st(), st)
        _check_gemm(p, before)
        assert (big[:M, cols:] == 3).all() and (big[M:] == 3).all() and st.item() == 0


@pytest.mark.parametrize("M", [4, 60, 600])
def test_gemm_sums_at_the_largest_k_and_values(E, M):
    """All codes -128: the sum is 2^14 K, just under 2^31 at the largest K."""
    N, K = 24, E.GEMM_I8_MAX_K
    p, st = _gemm_case(M, N, K, 8, 1), _status()
    p["A"].fill_(-128), p["W"].fill_(-128)
    p["C"].zero_()
    p["a_scale"].fill_(1.0), p["w_scale"].fill_(1.0)
    E.epara_gemm_i8(p, _st(), st)
    assert (p["C"][:M] == float(16384 * K)).all() and st.item() == 0


@pytest.mark.parametrize("M", [4, 60, 600])
def test_gemm_rows_of_nan_scale_stay_apart(E, M):
    p, st = _gemm_case(M, 128, 256, 0, 5), _status()
    p["a_scale"][M // 2] = float("nan")
    E.epara_gemm_i8(p, _st(), st)
    _check_gemm(p, None)


def test_gemm_sums_are_exact_whatever_the_kernel(E):
    """A row has the same bits in every batch: int32 sums know no order, the epilogue is the same arithmetic."""
    p, st = _gemm_case(700, 512, 1000, 1, 9), _status()
    E.epara_gemm_i8(p, _st(), st)
    for M in (1, 12, 50, 300):
        out = torch.empty((M, 512), dtype=torch.bfloat16, device="cuda")
        E.epara_gemm_i8(dict(p, M=M, C=out), _st(), st)
        assert torch.equal(out, p["C"][:M]), M


# ------------------------------------------------------------------------------------------------ cache
class Cache:
    """max_len: what the calls are told, which decides about kernels and chunks; used: tokens that there are pages for (the tables name
    none behind them)."""

    def __init__(self, B, max_len, Hkv, hd, seed, spare=3, fill="random", used=None):
        g = _gen(seed)
        self.B, self.max_len, self.Hkv, self.hd = B, max_len, Hkv, hd
        self.width = (max_len + 15) // 16
        used = (min(used or max_len, max_len) + 15) // 16
        self.pages = B * used + spare
        self.tables = torch.full((B, self.width), -1, dtype=torch.int32, device="cuda")
        self.tables[:, :used] = torch.randperm(self.pages, generator=g, device="cuda")[:B * used].to(torch.int32).view(B, used)
        shape = (self.pages, 2, Hkv, 16, hd)
        if fill == "random":
            self.codes = (torch.randn(shape, generator=g, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
        else:
            self.codes = torch.full(shape, fill, device="cuda").to(torch.float8_e4m3fn)
        self.scales = torch.exp2(torch.randint(-9, -4, shape[:3], generator=g, device="cuda").float())

    def values(self, b, n):
        """K, V [Hkv, n, hd] in 64 bits"""
        page = self.tables[b, : (n + 15) // 16].long()
        kv = self.codes.view(torch.uint8)[page].view(torch.float8_e4m3fn).to(F64) * self.scales[page].to(F64)[..., None, None]
        return kv.permute(1, 2, 0, 3, 4).reshape(2, self.Hkv, -1, self.hd)[:, :, :n]


class Part:
    """One request of a cache."""

    def __init__(self, c, b):
        self.Hkv, self.hd, self.values = c.Hkv, c.hd, lambda _, n: c.values(b, n)


def _rows(ns):
    r = [0]
    for n in ns:
        r.append(r[-1] + n)
    return torch.tensor(r, dtype=torch.int32, device="cuda"), r


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _attend(E, c, q, lens, ns, G, out=None, q_rows="prefix", max_q=None, max_len=None, st=None, stream=None):
    Hq = c.Hkv * G
    st = _status() if st is None else st
    out = torch.full((q.shape[0], Hq * c.hd), 55.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    rows = _rows(ns)[0] if isinstance(q_rows, str) else q_rows
    max_q, max_len = max_q or max(max(ns), 1), max_len or c.max_len
    need = E.epara_kv8_attention_scratch_bytes(c.B, q.shape[0], Hq, c.Hkv, c.hd, max_q, max_len)
    scratch = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")       # (NaN: nothing of it may count)
    E.epara_kv8_attention(q, c.codes, c.scales, _int(lens), c.tables, out, Hq, c.Hkv, c.hd, max_len, scratch, st, stream or _st(), q_rows=rows, max_q=max_q)
    return out, st


def _check_attention(c, q, lens, ns, G, out, what="", row0=0):
    hd, start = c.hd, row0
    for b, (n, L) in enumerate(zip(ns, lens)):
        rows = slice(start, start + n)
        start += n
        if n == 0:
            continue
        K, V = c.values(b, max(L, 1))
        qb = q[rows, : c.Hkv * G * hd].to(F64).view(n, c.Hkv, G, hd)
        t = torch.einsum("thgd,hld->thgl", qb, K) / math.sqrt(hd)
        mag = torch.einsum("thgd,hld->thgl", qb.abs(), K.nan_to_num(0).abs()) / math.sqrt(hd)
        hide = (torch.arange(max(L, 1), device="cuda")[None] >= (L - n + 1 + torch.arange(n, device="cuda"))[:, None])[:, None, None]
        none = hide.all(-1).squeeze()
        t, mag = t.masked_fill(hide, -math.inf), mag.masked_fill(hide, 0)
        p = torch.softmax(t, -1)
        Vx = V.nan_to_num(0)
        o = torch.einsum("thgl,hld->thgd", p, Vx)
        bad = torch.einsum("thgl,hld->thgd", (~hide).to(F64).expand_as(p), torch.isnan(V).to(F64)) > 0
        o = torch.where(bad, math.nan, o)
        # a probability: fp16 (half a step; below 2^-14 of the largest V scale's, 2^-25 of it), and the error of its exponent:
        # the products' sums in fp32 with a truncating adder, the factor, the subtraction of the maximum, exp2 of 2 ulp
        e_p = (mag.amax(-1) * 2.0 ** -21 + 2.0 ** -20)[..., None]
        pv = torch.einsum("thgl,hld->thgd", p, Vx.abs())
        m = torch.where(hide, 0, 1).sum(-1)[..., None]
        low = 2.0 ** -25 * Vx.abs().amax() * 2 * m.clamp(max=2.0 ** 15) * torch.exp(t.amax(-1) - torch.logsumexp(t, -1))[..., None]
        tol = (HALF_F16 + 3 * e_p) * pv + low + HALF_BF16 * (o.abs().nan_to_num(0) + 2 * HALF_F16 * pv)
        got = out[rows].to(F64).view(n, c.Hkv, G, hd)
        seen = ~none.reshape(n) if n > 1 else ~none.reshape(1)
        if (~seen).any():
            assert (out[rows][~seen] == 55).all(), what           # a row with nothing to attend to is left as it was
        _within(got[seen], o[seen], tol.expand_as(o)[seen], f"{what} b={b} n={n} L={L}")


LENS = [0, 1, 2, 15, 16, 17, 31, 63, 64, 65, 100, 129, 255, 256, 257, 1000, 1023]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hkv,G", [(1, 1), (2, 4), (8, 4), (3, 3), (2, 8), (1, 16), (1, 17), (2, 32)])
def test_attention_one_token(E, hd, Hkv, G):
    c = Cache(len(LENS), 1100, Hkv, hd, Hkv + G)
    q = torch.randn((len(LENS), Hkv * G * hd), generator=_gen(G), device="cuda").to(torch.bfloat16)
    ns = [1] * len(LENS)
    out, st = _attend(E, c, q, LENS, ns, G)
    assert st.item() == 0
    _check_attention(c, q, LENS, ns, G, out)
    out2, _ = _attend(E, c, q, LENS, ns, G, q_rows=None)   # the same without prefix sums, and again: the same bits
    assert torch.equal(out, out2)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hkv,G", [(2, 4), (1, 3), (2, 1), (1, 8)])
@pytest.mark.parametrize("ns,lens", [
    ([1, 2, 3, 0, 4], [1, 2, 3, 9, 500]), ([5, 16, 17, 1], [5, 16, 400, 77]), ([33, 0, 64, 100], [33, 1, 1000, 129]), ([130, 7, 257], [130, 900, 700]),
    ([600, 31], [1090, 600]), ([40, 4], [17, 2]),          # (fewer tokens than new rows: the first rows see none)
])
@pytest.mark.parametrize("max_len", [1100, 4000, 1 << 20])     # the last one: the kernel for many rows wherever there are more than 48
def test_attention_several_tokens(E, hd, Hkv, G, ns, lens, max_len):
    c = Cache(len(ns), max_len, Hkv, hd, sum(ns) + G, used=1100)
    T = sum(ns)
    q = torch.randn((T + 3, Hkv * G * hd), generator=_gen(T), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, ns, G)
    assert st.item() == 0
    _check_attention(c, q, lens, ns, G, out)
    assert (out[T:] == 55).all()                           # rows of no request


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_long_context(E, hd):
    c = Cache(2, 40000, 2, hd, 3)
    for ns, lens in (([1, 1], [40000, 33333]), ([20, 3], [39999, 20]), ([70, 40], [40000, 31000])):
        q = (2 * torch.randn((sum(ns), 8 * hd), generator=_gen(4), device="cuda")).to(torch.bfloat16)
        out, _ = _attend(E, c, q, lens, ns, 4)
        _check_attention(c, q, lens, ns, 4, out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hkv,G", [(2, 4), (3, 3)])
def test_attention_many_rows_in_several_chunks(E, hd, Hkv, G):
    """Rows that end in each of the chunks, so many of them that a warp merges a row."""
    c = Cache(2, 4000, Hkv, hd, 5)
    for ns, lens in (([600, 500], [3900, 1500]), ([300, 1], [300, 4000])):
        q = torch.randn((sum(ns), Hkv * G * hd), generator=_gen(6), device="cuda").to(torch.bfloat16)
        out, st = _attend(E, c, q, lens, ns, G)
        assert st.item() == 0
        _check_attention(c, q, lens, ns, G, out)
        again, _ = _attend(E, c, q, lens, ns, G)
        assert torch.equal(out, again)


MIXED = [([1] * 9 + [300] + [1] * 7, 16), ([700, 0, 1, 2, 3, 4, 5, 6, 16, 17, 33, 0], 5), ([0, 64, 1, 0, 130], 2), ([90] + [1, 0] * 260, 3), ([1] * 30 + [50, 60], 31)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hkv,G", [(2, 4), (1, 1), (3, 3), (1, 8), (2, 16), (1, 17), (1, 33)])
@pytest.mark.parametrize("ns,seed", MIXED)
@pytest.mark.parametrize("max_len", [3000, 40000])
def test_attention_of_short_and_long_requests_in_one_call(E, hd, Hkv, G, ns, seed, max_len):
    """Single tokens beside prompt chunks: each goes to its kernel, with chunks of its own; requests without rows and rows without requests."""
    c = Cache(len(ns), max_len, Hkv, hd, seed, used=2500 if len(ns) < 40 else 700)
    lens = [n + (181 * i + 7 * seed) % (2500 - 700 if len(ns) < 40 else 600) if n else 5 * i % 40 for i, n in enumerate(ns)]
    T = sum(ns)
    q = torch.randn((T + 5, Hkv * G * hd), generator=_gen(seed), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, ns, G)
    assert st.item() == 0
    if len(ns) > 40:
        pick = [0, 1, 2, 3, 101, 399, 519, 520]
        _, starts = _rows(ns)
        for b in pick:
            _check_attention(Part(c, b), q, [lens[b]], [ns[b]], G, out, f"request {b}", row0=starts[b])
    else:
        _check_attention(c, q, lens, ns, G, out)
    assert (out[T:] == 55).all()
    again, _ = _attend(E, c, q, lens, ns, G)
    assert torch.equal(out, again)
    # rows before the first request, and what max_q cuts off
    rows = _int([3 + r for r in _rows(ns)[1]])
    moved, st = _attend(E, c, torch.cat([q[:3], q[:T]]), lens, ns, G, q_rows=rows)
    assert st.item() == 0 and (moved[:3] == 55).all()
    if len(ns) < 40:
        _check_attention(c, torch.cat([q[:3], q[:T]]), lens, ns, G, moved, "moved", row0=3)


@pytest.mark.parametrize("hd", [64, 128])
def test_captured_call_follows_the_rows_on_the_device(E, hd):
    """One graph, replayed with other requests long and short, other lengths, and fewer rows than it was captured for: the eager calls' bits."""
    B, T, G, max_q = 6, 420, 4, 300
    c = Cache(B, 20000, 2, hd, 9, used=3000)
    q = torch.randn((T, 8 * hd), generator=_gen(9), device="cuda").to(torch.bfloat16)
    k = torch.randn((T, 4, hd), generator=_gen(10), device="cuda").to(torch.bfloat16)
    rows, lens, st, out = _int([0] * (B + 1)), _int([1] * B), _status(), torch.empty((T, 8 * hd), dtype=torch.bfloat16, device="cuda")
    need = E.epara_kv8_attention_scratch_bytes(B, T, 8, 2, hd, max_q, 20000)
    scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def calls():
        E.epara_kv8_append(k[:, :2], k[:, 2:], c.codes, c.scales, lens, c.tables, 20000, st, _st(), q_rows=rows, max_q=max_q)
        E.epara_kv8_attention(q, c.codes, c.scales, lens, c.tables, out, 8, 2, hd, 20000, scratch, st, _st(), q_rows=rows, max_q=max_q)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for ns, now in (([1, 300, 1, 1, 1, 116], [900, 2900, 17, 1, 300, 700]), ([300, 0, 4, 5, 100, 0], [300, 50, 2500, 2500, 1000, 9]), ([1] * 6, [10, 20, 3000, 1, 2, 16])):
        rows.copy_(_rows(ns)[0])
        lens.copy_(_int(now))
        codes, scales = c.codes.clone(), c.scales.clone()
        out.fill_(55)
        calls()
        want, want_codes = out.clone(), c.codes.clone()
        c.codes.copy_(codes), c.scales.copy_(scales)
        out.fill_(55)
        g.replay()
        assert st.item() == 0 and torch.equal(out, want) and torch.equal(c.codes.view(torch.uint8), want_codes.view(torch.uint8))
        _check_attention(c, q, now, ns, G, out)
        assert (out[sum(ns):] == 55).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_long_requests_cut_off_beside_short_ones(E, hd):
    ns, lens = [1, 80, 2, 50], [700, 900, 30, 1000]
    c = Cache(4, 3000, 2, hd, 3, used=1000)
    q = torch.randn((133, 8 * hd), generator=_gen(3), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, ns, 4, max_q=60)
    assert st.item() == E.ERR_ROWS and (out[61:81] == 55).all()
    for b, row, n, L in ((0, 0, 1, 700), (1, 1, 60, 880), (2, 81, 2, 30), (3, 83, 50, 1000)):
        _check_attention(Part(c, b), q, [L], [n], 4, out, row0=row)


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_many_requests_in_several_chunks(E, hd):
    B, Hkv, G = 300, 3, 3
    c = Cache(B, 8192, Hkv, hd, 7, used=2200)
    lens = [(37 * b) % 90 + 1 for b in range(B)]
    lens[3], lens[150], lens[298], lens[299] = 2200, 2049, 2048, 0
    q = torch.randn((B, Hkv * G * hd), generator=_gen(8), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, [1] * B, G)
    assert st.item() == 0
    _check_attention(c, q, lens, [1] * B, G, out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ns", [[1, 1, 1], [5, 1, 40], [70, 200, 33]])
@pytest.mark.parametrize("max_len", [320, 1 << 20])
def test_attention_does_not_see_what_stands_behind(E, hd, ns, max_len):
    """Slots behind the length, tokens behind a row's own, pages of nobody: NaN in all of them; and large and small scales side by side."""
    lens = [77, 300, 223]
    c = Cache(3, max_len, 2, hd, 8, used=320)
    codes = c.codes.view(torch.uint8)
    used = torch.zeros((c.pages, 16), dtype=torch.bool, device="cuda")
    for b, L in enumerate(lens):
        for t in range(L):
            used[c.tables[b, t // 16].long(), t % 16] = True
    codes.masked_fill_(~used[:, None, None, :, None].expand_as(codes), 0x7f)
    c.scales[c.tables[1, 3].long()] *= 2.0 ** 20
    c.scales[c.tables[1, 5].long()] = 0
    q = torch.randn((sum(ns), 8 * hd), generator=_gen(5), device="cuda").to(torch.bfloat16)
    q[0] = 0
    out, _ = _attend(E, c, q, lens, ns, 4)
    assert torch.isfinite(out.float()).all()
    _check_attention(c, q, lens, ns, 4, out)
    # NaN in K and V of visible tokens, some of them visible to a request's last rows only
    for b, L in enumerate(lens):
        for back, kv, h, d in ((1, 1, 0, 5), (3, 1, 1, hd - 1), (min(ns[b], 30), 0, 1, 7)):
            t = L - back
            codes[c.tables[b, t // 16].long(), kv, h, t % 16, d] = 0xff if back == 1 else 0x7f
    out, _ = _attend(E, c, q, lens, ns, 4)
    _check_attention(c, q, lens, ns, 4, out, "NaN tokens")


@pytest.mark.parametrize("many", [0, 30])                  # rows before the last one of each request: 30 reach the kernel for many rows
def test_attention_extreme_queries(E, many):
    c = Cache(4, 1 << 20 if many else 200, 1, 64, 6, used=200)
    lens, ns = [200, 150, 33, 90], [1 + many] * 4
    q = torch.randn((4, 1 + many, 4 * 64), generator=_gen(1), device="cuda")
    q[0, -1] *= 2.0 ** 60
    q[1, -1] *= 2.0 ** -60
    q[2, -1] *= 300
    q[3, -1, 3] = float("inf")
    q = q.to(torch.bfloat16).view(4 * (1 + many), 4 * 64)
    out, _ = _attend(E, c, q, lens, ns, 4)
    last = torch.arange(4, device="cuda") * (1 + many) + many
    q, out = q[last], out[last]
    K, V = c.values(0, 200)
    t = torch.einsum("gd,hld->gl", q[0].to(F64).view(4, 64), K)
    hit = V[0][t.argmax(1)]                                # scores of 2^60: the largest takes all
    assert ((out[0].to(F64).view(4, 64) - hit).abs() <= HALF_BF16 * hit.abs() + 1e-30).all()
    mean = c.values(1, 150)[1][0].mean(0)                  # scores of 2^-60: all alike
    spread = c.values(1, 150)[1][0].abs().mean(0)
    assert ((out[1].to(F64).view(4, 64) - mean).abs() <= 2 * HALF_F16 * spread + HALF_BF16 * mean.abs()).all()
    assert torch.isnan(out[3, :64].float()).all() and torch.isfinite(out[3, 64:].float()).all()


@pytest.mark.parametrize("max_len", [600, 1 << 20])
def test_attention_strides_and_alignment(E, max_len):
    c, lens, ns = Cache(3, max_len, 2, 128, 9, used=600), [600, 17, 345], [1, 30, 2]
    wide = torch.randn((33, 8 * 128 + 512), generator=_gen(3), device="cuda").to(torch.bfloat16)      # q inside a QKV row
    flat = torch.full((33 * 1024 + 5,), 55.0, dtype=torch.bfloat16, device="cuda")
    for off in (0, 1, 2, 5):
        out = flat[off:off + 33 * 1024].view(33, 1024)
        _attend(E, c, wide[:, 256:256 + 1024], lens, ns, 4, out=out)
        _check_attention(c, wide[:, 256:256 + 1024], lens, ns, 4, out)
        flat.fill_(55.0)


def test_bad_pages_rows_and_lengths_are_reported_and_skipped(E):
    """Page ids outside the pool are read as absent, tokens beyond max_q and max_len left out: nothing is read or written for them."""
    c = Cache(3, 200, 2, 64, 2)
    lens, ns = [100, 60, 200], [1, 1, 1]
    q = torch.randn((3, 8 * 64), generator=_gen(2), device="cuda").to(torch.bfloat16)
    good, st = _attend(E, c, q, lens, ns, 4)
    keep = c.tables.clone()
    c.tables[1, 2] = c.pages
    c.tables[2, 0] = -1
    out, st = _attend(E, c, q, lens, ns, 4)
    assert st.item() == E.ERR_PAGE_ATTEND and torch.equal(out[0], good[0])
    c.tables.copy_(keep)
    out, st = _attend(E, c, q, [100, -7, 10 ** 6], ns, 4)  # clamped: no token, max_len
    assert st.item() == 0 and torch.equal(out[0], good[0]) and (out[1] == 55).all() and torch.equal(out[2], good[2])
    # more rows than max_q: the first max_q of them are right, the rest stays
    q = torch.randn((9, 8 * 64), generator=_gen(2), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, [1, 7, 1], 4, max_q=3)
    full, _ = _attend(E, c, q, lens, [1, 7, 1], 4)
    assert st.item() == E.ERR_ROWS and (out[4:8] == 55).all() and torch.equal(out[8], full[8])
    _check_attention(c, q[:1], lens[:1], [1], 4, out[:1])
    _check_attention(Part(c, 1), q[1:4], [lens[1] - 4], [3], 4, out[1:4])
    # prefix sums that leave the tensor are clamped to it
    out, st = _attend(E, c, q, lens, [1], 4, q_rows=_int([-5, 1, 4, 10 ** 9]), max_q=9)
    assert (out.float() != 55).any(1).all()


def _append_reference(codes, scales, k, v, tables, lens, ns):
    """From the definition, a page at a time, in 64 bits."""
    codes, scales, start = codes.to(F64), scales.to(F64), 0
    for b, (n, L) in enumerate(zip(ns, lens)):
        done = 0
        while done < n:
            pos = L - n + done
            page, slot = int(tables[b, pos // 16]), pos % 16
            take = min(16 - slot, n - done)
            for i, x in enumerate((k, v)):
                x = x[start + done:start + done + take].to(F64).permute(1, 0, 2)         # [Hkv, take, hd]
                fin = torch.where(torch.isfinite(x), x.abs(), 0).amax((1, 2))
                need = torch.exp2(torch.ceil(torch.log2((fin / 448).clamp(min=2.0 ** -126)) - 1e-9))
                if slot:
                    new = torch.maximum(need, scales[page, i])
                    f = (scales[page, i] / new)[:, None, None]
                    codes[page, i, :, :slot] = torch.where(f == 1, codes[page, i, :, :slot], _e4m3(codes[page, i, :, :slot] * f))
                    need = new
                codes[page, i, :, slot:slot + take] = _e4m3(torch.where(torch.isfinite(x), x, math.nan) / need[:, None, None])
                scales[page, i] = need
            done += take
        start += n
    return codes, scales


def _e4m3(x):
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(0), b.nan_to_num(0))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hkv", [1, 3, 8])
@pytest.mark.parametrize("ns,lens", [([1, 1, 1, 1], [1, 16, 17, 40]), ([3, 0, 16, 50], [3, 5, 40, 64]), ([16, 17, 31, 33], [16, 64, 64, 50]), ([64, 1], [64, 8])])
def test_append(E, hd, Hkv, ns, lens):
    c, T = Cache(len(ns), 64, Hkv, hd, sum(ns)), sum(ns)
    g = _gen(T + hd)
    qkv = torch.randn((T, 2 * Hkv + 4, hd), generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (T, 2 * Hkv + 4, 1), generator=g, device="cuda").float())
    qkv = qkv.to(torch.bfloat16)
    qkv[0, 4, 3], qkv[0, 4 + Hkv, 5] = float("inf"), float("nan")
    k, v = qkv[:, 4:4 + Hkv], qkv[:, 4 + Hkv:4 + 2 * Hkv]
    c.scales[c.tables[0, 0].long(), 0] = 0.013             # a scale of somebody else's, no power of two
    st = _status()
    want = _append_reference(c.codes, c.scales, k, v, c.tables, lens, ns)
    E.epara_kv8_append(k, v, c.codes, c.scales, _int(lens), c.tables, 64, st, _st(), q_rows=_rows(ns)[0], max_q=max(ns))
    assert st.item() == 0 and torch.equal(c.scales.to(F64), want[1].to(torch.float32).to(F64))
    if lens[0] - ns[0] == 0:                               # (with the foreign scale still in use a quotient is not exact)
        assert _same(c.codes.to(F64), want[0])


@pytest.mark.parametrize("hd", [64, 128])
def test_append_single_tokens_beside_a_prompt(E, hd):
    """Few of the requests have as many tokens as the longest: the same cache as by a call for each."""
    ns = [1] * 30 + [0, 257, 0, 16, 1, 17] + [1] * 30
    lens = [n + (7 * i) % 50 if n else 9 for i, n in enumerate(ns)]
    g = _gen(4)
    x = torch.randn((sum(ns) + 4, 6, hd), generator=g, device="cuda").to(torch.bfloat16)
    one, each = Cache(len(ns), 400, 3, hd, 4), Cache(len(ns), 400, 3, hd, 4)
    st = _status()
    rows = [r + 2 for r in _rows(ns)[1]]                       # (two rows of nobody at both ends)
    E.epara_kv8_append(x[:, :3], x[:, 3:], one.codes, one.scales, _int(lens), one.tables, 400, st, _st(), q_rows=_int(rows), max_q=257)
    assert st.item() == 0
    for b, n in enumerate(ns):
        if n:
            y = x[rows[b]:rows[b] + n]
            E.epara_kv8_append(y[:, :3], y[:, 3:], each.codes, each.scales, _int([lens[b]]), each.tables[b:b + 1], 400, st, _st(), q_rows=_int([0, n]), max_q=n)
    assert st.item() == 0
    assert torch.equal(one.codes.view(torch.uint8), each.codes.view(torch.uint8)) and torch.equal(one.scales, each.scales)
    lens[31], st = 200, _status()                              # fewer tokens than new ones: reported, the others as before
    E.epara_kv8_append(x[:, :3], x[:, 3:], one.codes, one.scales, _int(lens), one.tables, 400, st, _st(), q_rows=_int(rows), max_q=257)
    assert st.item() == E.ERR_PAGE_APPEND
    st = _status()
    E.epara_kv8_append(x[:, :3], x[:, 3:], one.codes, one.scales, _int(lens), one.tables, 400, st, _st(), q_rows=_int(rows), max_q=100)
    assert st.item() in (E.ERR_ROWS, E.ERR_PAGE_APPEND)


def test_append_largest_smallest_and_zero_values(E):
    c, st = Cache(5, 16, 1, 64, 1, fill=0.0), _status()
    x = torch.zeros((5, 1, 64), device="cuda")
    x[0, 0, 0], x[1, 0, 1], x[2, 0, 2], x[3, 0, 3] = 3.3e38, 448.0, 449.0 * 1.01, 1e-40
    x = x.to(torch.bfloat16)
    E.epara_kv8_append(x, -x, c.codes, c.scales, _int([1] * 5), c.tables, 16, st, _st())
    want = _append_reference(c.codes, c.scales, x, -x, c.tables, [1] * 5, [1] * 5)
    assert _same(c.codes.to(F64), want[0]) and torch.equal(c.scales.to(F64), want[1])
    at = c.tables[:, 0].long()
    assert c.scales[at[1], 0, 0] == 1 and c.scales[at[2], 0, 0] == 2 and c.scales[at[4], 0, 0] == 2.0 ** -126 and torch.isfinite(c.scales[at]).all()


def test_append_token_by_token_and_at_once(E):
    """Powers of two: a page filled a token at a time ends with the same codes as one filled at once, but for values that a larger
    scale has made subnormal."""
    n, Hkv, hd = 50, 2, 128
    x = torch.randn((n, 2 * Hkv, hd), generator=_gen(1), device="cuda")
    x = (x * (1 + torch.arange(n, device="cuda").view(n, 1, 1) / 5)).to(torch.bfloat16)
    a, b = Cache(1, 64, Hkv, hd, 2, fill=0.0), Cache(1, 64, Hkv, hd, 2, fill=0.0)
    st = _status()
    E.epara_kv8_append(x[:, :Hkv], x[:, Hkv:], a.codes, a.scales, _int([n]), a.tables, 64, st, _st(), q_rows=_int([0, n]), max_q=n)
    for t in range(n):
        E.epara_kv8_append(x[t:t + 1, :Hkv], x[t:t + 1, Hkv:], b.codes, b.scales, _int([t + 1]), b.tables, 64, st, _st())
    used = a.tables[0, :4].long()
    assert torch.equal(a.scales[used], b.scales[used])
    ka, kb = a.values(0, n), b.values(0, n)
    big = ka.abs() >= a.scales[used].to(F64).amax() * 2.0 ** -6
    assert torch.equal(ka[big], kb[big])
    assert ((ka - kb).abs() <= a.scales[used].to(F64).amax() * 2.0 ** -9).all()          # one subnormal step


def test_append_skips_what_it_must_not_touch(E):
    c, st = Cache(4, 64, 2, 64, 3), _status()
    x = torch.randn((9, 4, 64), generator=_gen(3), device="cuda").to(torch.bfloat16)
    ns, lens = [2, 3, 2, 2], [1, 40, 65, 20]               # fewer than n tokens; fine; past max_len; a bad page
    c.tables[3, 1] = c.pages + 5
    before = c.codes.clone(), c.scales.clone()
    want = _append_reference(c.codes, c.scales, x[2:5, :2], x[2:5, 2:], c.tables[1:2], [40], [3])
    E.epara_kv8_append(x[:, :2], x[:, 2:], c.codes, c.scales, _int(lens), c.tables, 64, st, _st(), q_rows=_rows(ns)[0], max_q=3)
    assert st.item() == E.ERR_PAGE_APPEND and _same(c.codes.to(F64), want[0]) and torch.equal(c.scales.to(F64), want[1])
    c.codes.copy_(before[0]), c.scales.copy_(before[1]), st.zero_()
    want = _append_reference(c.codes, c.scales, x[:2, :2], x[:2, 2:], c.tables[:1], [39], [2])     # max_q 2 of 3: the first two rows, at their places
    E.epara_kv8_append(x[:3, :2], x[:3, 2:], c.codes, c.scales, _int([40]), c.tables[:1], 64, st, _st(), q_rows=_int([0, 3]), max_q=2)
    assert st.item() == E.ERR_ROWS and _same(c.codes.to(F64), want[0])


def test_cache_past_32_bit_offsets(E):
    """A pool of more than 4 GiB: append to and attend over its last pages."""
    pages, Hkv, hd = (1 << 32) // (2 * 8 * 16 * 128) + 40, 8, 128
    codes = torch.zeros((pages, 2, Hkv, 16, hd), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.ones((pages, 2, Hkv), device="cuda")
    tables = torch.arange(pages - 1, pages - 9, -1, dtype=torch.int32, device="cuda").view(2, 4)
    g, st = _gen(1), _status()
    x = torch.randn((80, 2 * Hkv, hd), generator=g, device="cuda").to(torch.bfloat16)
    c = Cache(2, 64, Hkv, hd, 1)
    c.codes, c.scales, c.tables, c.pages = codes, scales, tables, pages
    E.epara_kv8_append(x[:, :Hkv], x[:, Hkv:], codes, scales, _int([64, 16]), tables, 64, st, _st(), q_rows=_int([0, 64, 80]), max_q=64)
    for b, (L, lo) in enumerate(((64, 0), (16, 64))):
        K, V = c.values(b, L)
        for got, want in ((K, x[lo:lo + L, :Hkv]), (V, x[lo:lo + L, Hkv:])):
            want = want.to(F64).permute(1, 0, 2)
            assert ((got - want).abs() <= want.abs() * 2.0 ** -4 + want.abs().amax() / 224 * 2.0 ** -10).all()
    assert not codes[: pages - 8].view(torch.uint8).any().item()
    q = torch.randn((2, 32 * hd), generator=g, device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, [64, 16], [1, 1], 4)
    _check_attention(c, q, [64, 16], [1, 1], 4, out)
    assert st.item() == 0


# ------------------------------------------------------------------------------------------------ together
def _layer_buffers(B, max_len, seed):
    d, Hkv, G, hd, ffn = 256, 2, 2, 64, 320
    g = _gen(seed)

    def weight(n, k):
        return torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8), (0.5 + torch.rand((n,), generator=g, device="cuda")) / (70 * math.sqrt(k))

    s = dict(d=d, Hkv=Hkv, G=G, hd=hd, ffn=ffn, B=B)
    s["Wqkv"], s["Wo"], s["Wgu"], s["Wd"] = weight((G + 2) * Hkv * hd, d), weight(d, G * Hkv * hd), weight(2 * ffn, d), weight(d, ffn)
    s["g1"], s["g2"] = ((1 + 0.2 * torch.randn((d,), generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    s["cache"] = Cache(B, max_len, Hkv, hd, seed)
    return s


def _layer(E, s, resid, lens, q_rows, max_q, st, keep=None):
    """One decoder layer over the rows of `resid` (fp32 [T, d], updated), in 8 bits."""
    T, d, Hkv, G, hd, ffn, c = resid.shape[0], s["d"], s["Hkv"], s["G"], s["hd"], s["ffn"], s["cache"]
    Hq, bf, dev = Hkv * G, torch.bfloat16, "cuda"
    b = keep if keep is not None else {}
    if not b:
        b.update(x8=torch.empty((T, d), dtype=torch.int8, device=dev), xs=torch.empty(T, device=dev), qkv=torch.empty((T, (G + 2) * Hkv * hd), dtype=bf, device=dev),
                 att=torch.empty((T, Hq * hd), dtype=bf, device=dev), a8=torch.empty((T, Hq * hd), dtype=torch.int8, device=dev), as_=torch.empty(T, device=dev),
                 y8=torch.empty((T, d), dtype=torch.int8, device=dev), ys=torch.empty(T, device=dev), h=torch.empty((T, ffn), dtype=bf, device=dev),
                 h8=torch.empty((T, ffn), dtype=torch.int8, device=dev), hs=torch.empty(T, device=dev),
                 scratch=torch.empty(max(16, E.epara_kv8_attention_scratch_bytes(c.B, T, Hq, Hkv, hd, max_q, c.max_len)), dtype=torch.uint8, device=dev))
    stream = _st()

    def mm(a, a_s, w, out, epi=0):
        E.epara_gemm_i8(dict(A=a, W=w[0], a_scale=a_s, w_scale=w[1], C=out, M=T, N=w[0].shape[0], K=w[0].shape[1], epilogue=epi), stream, st)

    E.epara_rms_norm_i8(resid, s["g1"], b["x8"], b["xs"], stream)
    mm(b["x8"], b["xs"], s["Wqkv"], b["qkv"])
    heads = b["qkv"].view(T, (G + 2) * Hkv, hd)
    E.epara_kv8_append(heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:], c.codes, c.scales, lens, c.tables, c.max_len, st, stream, q_rows=q_rows, max_q=max_q)
    E.epara_kv8_attention(b["qkv"], c.codes, c.scales, lens, c.tables, b["att"], Hq, Hkv, hd, c.max_len, b["scratch"], st, stream, q_rows=q_rows, max_q=max_q)
    E.epara_rms_norm_i8(b["att"], None, b["a8"], b["as_"], stream)
    mm(b["a8"], b["as_"], s["Wo"], resid, E.EPI_RESID_F32)
    E.epara_rms_norm_i8(resid, s["g2"], b["y8"], b["ys"], stream)
    mm(b["y8"], b["ys"], s["Wgu"], b["h"], E.EPI_SWIGLU)
    E.epara_rms_norm_i8(b["h"], None, b["h8"], b["hs"], stream)
    mm(b["h8"], b["hs"], s["Wd"], resid, E.EPI_RESID_F32)
    return b


def _check_layer(s, before, b, resid, codes, scales, lens, ns):
    """Stage by stage, each fed the device's own input of it."""
    T, d, Hkv, G, hd, ffn, c = before.shape[0], s["d"], s["Hkv"], s["G"], s["hd"], s["ffn"], s["cache"]
    Hq = Hkv * G
    _check_norm(before, None, s["g1"], b["x8"], b["xs"], None)
    _check_gemm(dict(A=b["x8"], W=s["Wqkv"][0], a_scale=b["xs"], w_scale=s["Wqkv"][1], C=b["qkv"], M=T, K=d, N=(G + 2) * Hkv * hd, epilogue=0), None)
    heads = b["qkv"].view(T, (G + 2) * Hkv, hd)
    want = _append_reference(codes, scales, heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:], c.tables, lens, ns)
    assert _same(c.codes.to(F64), want[0]) and torch.equal(c.scales.to(F64), want[1])
    _check_attention(c, b["qkv"], lens, ns, G, b["att"])
    _check_norm(b["att"], None, None, b["a8"], b["as_"], None)
    mid = before.to(F64) + (b["a8"].to(F64) @ s["Wo"][0].to(F64).t()) * b["as_"].to(F64)[:, None] * s["Wo"][1].to(F64)
    _check_gemm(dict(A=b["y8"], W=s["Wgu"][0], a_scale=b["ys"], w_scale=s["Wgu"][1], C=b["h"], M=T, K=d, N=2 * ffn, epilogue=4), None)
    _check_norm(b["h"], None, None, b["h8"], b["hs"], None)
    add = (b["h8"].to(F64) @ s["Wd"][0].to(F64).t()) * b["hs"].to(F64)[:, None] * s["Wd"][1].to(F64)
    assert ((resid.to(F64) - mid - add).abs() <= 8 * HALF_F32 * (before.abs() + mid.abs() + add.abs() + (mid - before).abs())).all()


@pytest.mark.parametrize("ns,lens", [([1, 1, 1], [1, 40, 200]), ([20, 1, 5], [20, 300, 77]), ([300, 1, 250], [310, 9, 250])])
def test_a_decoder_layer_in_8_bits(E, ns, lens):
    s, T = _layer_buffers(3, 320, sum(ns)), sum(ns)
    resid = torch.randn((T, s["d"]), generator=_gen(T), device="cuda")
    before, codes, scales, st = resid.clone(), s["cache"].codes.clone(), s["cache"].scales.clone(), _status()
    b = _layer(E, s, resid, _int(lens), _rows(ns)[0], max(ns), st)
    assert st.item() == 0
    _check_layer(s, before, b, resid, codes, scales, lens, ns)


def test_a_layer_on_another_stream_and_captured(E):
    """A decode layer in a CUDA graph, replayed while the sequences grow, gives the bits of the calls made one by one; two graphs with
    workspaces of their own, replayed on two streams at once, too."""
    sets = []
    for seed in (1, 2):
        s = _layer_buffers(2, 128, seed)
        lens, resid, st, rows = _int([30, 77]), torch.empty((2, s["d"]), device="cuda"), _status(), _rows([1, 1])[0]
        x0 = torch.randn((6, 2, s["d"]), generator=_gen(seed), device="cuda")
        codes, scales = s["cache"].codes.clone(), s["cache"].scales.clone()
        eager = []
        for i in range(6):
            resid.copy_(x0[i])
            _layer(E, s, resid, lens, rows, 1, st)
            eager.append(resid.clone())
            lens += 1
        want_codes = s["cache"].codes.clone()
        s["cache"].codes.copy_(codes), s["cache"].scales.copy_(scales)
        lens.copy_(_int([30, 77]))
        keep, side = {}, torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _layer(E, s, resid, lens, rows, 1, st, keep)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        s["cache"].codes.copy_(codes), s["cache"].scales.copy_(scales)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _layer(E, s, resid, lens, rows, 1, st, keep)
            lens += 1
        lens.copy_(_int([30, 77]))
        keep["rows"] = rows                                # (the graph reads it)
        sets.append((s, lens, resid, st, x0, eager, want_codes, g, side, keep))
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(6):
        for n, (s, lens, resid, st, x0, eager, want_codes, g, side, keep) in enumerate(sets):
            with torch.cuda.stream(side):
                resid.copy_(x0[i])
                g.replay()
                got[n].append(resid.clone())
    torch.cuda.synchronize()
    for n, (s, lens, resid, st, x0, eager, want_codes, g, side, keep) in enumerate(sets):
        assert all(torch.equal(a, b) for a, b in zip(got[n], eager)) and st.item() == 0
        assert torch.equal(s["cache"].codes.view(torch.uint8), want_codes.view(torch.uint8))


def test_an_8_bit_cache_beside_the_bf16_one(E):
    """The same sequence in both caches: the difference is what e4m3 loses, at most half of its step in K and V each."""
    from paper_2511_00603_b200 import synth
    L, Hkv, G, hd = 300, 2, 4, 64
    g = _gen(1)
    x = torch.randn((L, 2 * Hkv, hd), generator=g, device="cuda").to(torch.bfloat16)
    c, st = Cache(1, 304, Hkv, hd, 1, fill=0.0), _status()
    E.epara_kv8_append(x[:, :Hkv], x[:, Hkv:], c.codes, c.scales, _int([L]), c.tables, 304, st, _st(), q_rows=_int([0, L]), max_q=L)
    pool = torch.zeros((c.pages, 2, Hkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    for t in range(L):
        pool[c.tables[0, t // 16].long(), :, :, t % 16] = x[t].view(2, Hkv, hd)
    q = torch.randn((1, Hkv * G * hd), generator=g, device="cuda").to(torch.bfloat16)
    ref = torch.empty_like(q)
    scratch = torch.empty(E.lib.epara_decode_attention_scratch_bytes(1, Hkv * G, hd, L), dtype=torch.uint8, device="cuda")
    E.epara_decode_attention(q, pool, _int([L]), c.tables, ref, Hkv * G, Hkv, hd, L, scratch, _st())
    out, _ = _attend(E, c, q, [L], [1], G)
    _check_attention(c, q, [L], [1], G, out)
    # V off by 2^-4 of itself at most; K by as much: a score by at most 2^-4 sum |q k| / sqrt(hd), in practice its root
    rel = ((out.to(F64) - ref.to(F64)).norm() / ref.to(F64).norm()).item()
    assert rel < 2.0 ** -4 * 3, rel


@pytest.mark.parametrize("hd", [64, 128])
def test_many_rows_bad_pages_and_rows_beyond_max_q(E, hd):
    """The kernel for many rows: a page outside the pool is reported and not read, the other requests are as they were; rows beyond max_q stay."""
    c = Cache(3, 1 << 20, 2, hd, 2, used=300)
    lens, ns = [300, 150, 220], [40, 90, 25]
    q = torch.randn((155, 8 * hd), generator=_gen(2), device="cuda").to(torch.bfloat16)
    good, st = _attend(E, c, q, lens, ns, 4)
    _check_attention(c, q, lens, ns, 4, good)
    keep = c.tables.clone()
    c.tables[1, 2], c.tables[1, 5] = c.pages, -3
    out, bad = _attend(E, c, q, lens, ns, 4)
    assert st.item() == 0 and bad.item() == E.ERR_PAGE_ATTEND and torch.equal(out[:40], good[:40]) and torch.equal(out[130:], good[130:])
    c.tables.copy_(keep)
    out, st = _attend(E, c, q, lens, ns, 4, max_q=41)
    assert st.item() == E.ERR_ROWS and torch.equal(out[:40], good[:40]) and (out[81:130] == 55).all() and torch.equal(out[130:], good[130:])
    _check_attention(Part(c, 1), q[40:81], [lens[1] - 49], [41], 4, out[40:81])


@pytest.mark.parametrize("M", [3, 100, 700])
def test_a_call_reads_what_the_call_before_wrote(E, M):
    """Weights quantised on the stream right before the product that reads them, in the same buffers again and again; the result quantised in turn."""
    N, K, st = 640, 1024, _status()
    A = torch.randint(-127, 128, (M, K), generator=_gen(1), device="cuda", dtype=torch.int8)
    sa = torch.rand(M, generator=_gen(2), device="cuda")
    W8, ws, C = torch.empty((N, K), dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    C8, cs = torch.empty((M, N), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    Ws = [torch.randn((N, K), generator=_gen(9 + i), device="cuda").to(torch.bfloat16) for i in range(8)]

    def run(W, wait):
        for call in (lambda: E.epara_rms_norm_i8(W, None, W8, ws, _st()),
                     lambda: E.epara_gemm_i8(dict(A=A, W=W8, a_scale=sa, w_scale=ws, C=C, M=M, N=N, K=K), _st(), st),
                     lambda: E.epara_rms_norm_i8(C, None, C8, cs, _st())):
            call()
            if wait:
                torch.cuda.synchronize()
        return C.clone(), C8.clone(), cs.clone()

    want = [run(W, True) for W in Ws]
    for _ in range(3):
        got = [run(W, False) for W in Ws]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    assert st.item() == 0


def test_empty_tensors(E):
    st, none = _status(), _int([])
    f, b, i8 = (torch.empty((0, 64), dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16, torch.int8))
    E.epara_rms_norm_i8(b, torch.ones(64, dtype=torch.bfloat16, device="cuda"), i8, f[:, 0], _st(), resid=f, resid_out=f)
    p = _gemm_case(0, 64, 64, 0, 1)
    E.epara_gemm_i8(dict(p, A=i8, a_scale=f[:, 0], C=b), _st(), st)
    c = Cache(2, 64, 1, 64, 1)
    before = c.codes.clone()
    E.epara_kv8_append(b.view(0, 1, 64), b.view(0, 1, 64), c.codes, c.scales, none, c.tables[:0], 64, st, _st(), q_rows=_int([0]))
    E.epara_kv8_append(b.view(0, 1, 64), b.view(0, 1, 64), c.codes, c.scales, _int([5, 9]), c.tables, 64, st, _st(), q_rows=_int([0, 0, 0]))
    E.epara_kv8_attention(b, c.codes, c.scales, _int([5, 9]), c.tables, b, 1, 1, 64, 64, None, st, _st(), q_rows=_int([0, 0, 0]))
    assert st.item() == 0 and torch.equal(before.view(torch.uint8), c.codes.view(torch.uint8))


def test_calls_leave_the_current_device(E):
    assert torch.cuda.current_device() == 0
    x, q, s = torch.randn((2, 64), device="cuda"), torch.empty((2, 64), dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    E.epara_rms_norm_i8(x, None, q, s, _st(), device=0)
    with pytest.raises(E.EparaError) as e:                 # a device that is not there
        E.epara_rms_norm_i8(x, None, q, s, _st(), device=63)
    assert e.value.status == E.E_CUDA and torch.cuda.current_device() == 0
    E.epara_rms_norm_i8(x, None, q, s, _st())
    _check_norm(x, None, None, q, s, None)
