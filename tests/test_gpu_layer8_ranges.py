"""The 8-bit decoder layer at the ends of its ranges: V scales far apart, scales that are no powers of two, GELU's tail, very long rows."""
import math

import pytest
import torch

from .test_gpu_layer8 import (F64, HALF_BF16, HALF_F16, HALF_F32, Cache, Part, _append_reference, _attend, _check_attention, _check_norm, _gen, _int, _rows, _st,
                              _status, _within)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from paper_2511_00603_b200 import build
    build.build()
    from paper_2511_00603_b200 import epara
    return epara


# ------------------------------------------------------------------------------------------------ attention
def _check_by_weight(c, q, lens, ns, G, out, what=""):
    """Against the definition in 64 bits, with a tolerance from what each row itself sums up: neither a token that the row does not see nor
    one that it gives no weight makes it wider."""
    hd, start = c.hd, 0
    for b, (n, L) in enumerate(zip(ns, lens)):
        rows = slice(start, start + n)
        start += n
        K, V = c.values(b, L)
        page = c.tables[b, : (L + 15) // 16].long()
        sv = c.scales[page, 1].to(F64).t().repeat_interleave(16, 1)[:, :L]              # [Hkv, L]: the scale of each token's V
        qb = q[rows].to(F64).view(n, c.Hkv, G, hd)
        t = torch.einsum("thgd,hld->thgl", qb, K) / math.sqrt(hd)
        mag = torch.einsum("thgd,hld->thgl", qb.abs(), K.abs()) / math.sqrt(hd)
        hide = (torch.arange(L, device="cuda")[None] >= (L - n + 1 + torch.arange(n, device="cuda"))[:, None])[:, None, None]
        t, mag = t.masked_fill(hide, -math.inf), mag.masked_fill(hide, 0)
        p = torch.softmax(t, -1)
        o = torch.einsum("thgl,hld->thgd", p, V)
        pv = torch.einsum("thgl,hld->thgd", p, V.abs())
        # A probability's error: its exponent's (sums in fp32 with a truncating adder, the factor, the maximum's subtraction, exp2 of 2 ulp).  In
        # fp16 stands probability x V scale, the largest so far in (2^6, 2^15]: half a step of it, or of the subnormals 2^-25, which is 2^-31 of the
        # largest weight a code (up to 448, twice that with the scale's mantissa) is multiplied by.  One more half step for
        # a V code times a mantissa that is no power of two.
        e_p = (mag.amax(-1) * 2.0 ** -21 + 2.0 ** -20)[..., None]
        low = 2.0 ** -31 * 896 * (p * sv[None, :, None]).amax(-1, keepdim=True) * (~hide).to(F64).sum(-1)[..., None]
        tol = (2 * HALF_F16 + 3 * e_p) * pv + low + HALF_BF16 * (o.abs() + 3 * HALF_F16 * pv)
        _within(out[rows].view(n, c.Hkv, G, hd), o, tol, f"{what} b={b} n={n} L={L}")


# Short contexts; long ones, whose chunks hold many pages for each warp; so long ones that the kernel for many rows takes all beyond 16
MAX_LENS = [320, 40000, 1 << 20]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ns", [[1, 1, 1], [5, 2, 40], [70, 200, 33]])
@pytest.mark.parametrize("max_len", MAX_LENS)
def test_v_scales_far_apart(E, hd, ns, max_len):
    """Every (page, head) with a V scale of its own between 2^-40 and 2^40: what a row sees, and with what weight, decides what counts."""
    lens = [77, 300, 223]
    c = Cache(3, max_len, 2, hd, 11, used=320)
    c.scales[:, 1] = torch.exp2(torch.randint(-40, 41, c.scales[:, 1].shape, generator=_gen(3), device="cuda").float())
    q = torch.randn((sum(ns), 8 * hd), generator=_gen(12), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, ns, 4)
    assert st.item() == 0
    _check_by_weight(c, q, lens, ns, 4, out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [2, 30, 120])
@pytest.mark.parametrize("max_len", MAX_LENS)
def test_an_outlier_in_v_that_a_row_does_not_see(E, hd, n, max_len):
    """The last page's V is 2^30 times the others': only the rows that see a token of it may notice."""
    L = 257
    c = Cache(1, max_len, 2, hd, 13, used=320)
    c.scales[c.tables[0, 16].long(), 1] *= 2.0 ** 30       # token 256, which the last row alone sees
    q = torch.randn((n, 8 * hd), generator=_gen(14), device="cuda").to(torch.bfloat16)
    out, _ = _attend(E, c, q, [L], [n], 4)
    _check_by_weight(c, q, [L], [n], 4, out)
    plain, _ = _attend(E, c, q[:n - 1], [L - 1], [n - 1], 4, max_q=n)          # ... and they are what they would be without it
    _check_by_weight(c, q[:n - 1], [L - 1], [n - 1], 4, plain)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("far", [8.0, 40.0])
@pytest.mark.parametrize("max_len", MAX_LENS)
def test_an_outlier_in_v_that_gets_next_to_no_weight(E, hd, n, far, max_len):
    """A page whose keys stand against the queries: its V, 2^40 times the others', counts by probability times value, whichever is larger."""
    L, G = 290, 4
    c = Cache(1, max_len, 2, hd, 15, used=320)
    base = torch.sign(torch.randn(hd, generator=_gen(16), device="cuda"))
    q = (base * (1 + 0.2 * torch.rand((n, 8, hd), generator=_gen(17), device="cuda"))).to(torch.bfloat16).view(n, 8 * hd)
    at = c.tables[0, 5].long()
    c.codes[at, 0] = (-base * 64).to(torch.float8_e4m3fn)
    c.scales[at, 0] = far / (64 * math.sqrt(hd))           # scores of about -far
    c.scales[at, 1] *= 2.0 ** 40
    out, _ = _attend(E, c, q, [L], [n], G)
    _check_by_weight(c, q, [L], [n], G, out, f"far={far}")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ns", [[1, 1], [3, 1], [200, 90]])
def test_v_scales_far_apart_in_long_contexts(E, hd, ns):
    """Several chunks, whose results meet; pages far behind the first ones read."""
    lens = [9000, 5111]
    c = Cache(2, 9000, 2, hd, 18)
    c.scales[:, 1] = torch.exp2(torch.randint(-30, 31, c.scales[:, 1].shape, generator=_gen(19), device="cuda").float())
    q = torch.randn((sum(ns), 8 * hd), generator=_gen(20), device="cuda").to(torch.bfloat16)
    out, _ = _attend(E, c, q, lens, ns, 4)
    _check_by_weight(c, q, lens, ns, 4, out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lo,hi", [(-126, -100), (80, 100)])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("max_len", MAX_LENS)
def test_v_scales_at_the_ends(E, hd, lo, hi, n, max_len):
    c = Cache(1, max_len, 1, hd, 21, used=320)
    c.scales[:, 1] = torch.exp2(torch.randint(lo, hi, c.scales[:, 1].shape, generator=_gen(22), device="cuda").float())
    q = torch.randn((n, 4 * hd), generator=_gen(23), device="cuda").to(torch.bfloat16)
    out, _ = _attend(E, c, q, [300], [n], 4)
    _check_by_weight(c, q, [300], [n], 4, out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ns", [[1, 1, 1], [5, 2, 40], [70, 200, 33]])
@pytest.mark.parametrize("max_len", MAX_LENS)
def test_scales_that_are_no_powers_of_two(E, hd, ns, max_len):
    """A cache that another program has written: any finite scale that is not negative, zero among them."""
    lens = [77, 300, 223]
    c = Cache(3, max_len, 2, hd, 24, used=320)
    c.scales *= 1 + torch.rand(c.scales.shape, generator=_gen(25), device="cuda")
    c.scales[c.tables[1, 2].long(), 1] = 0
    c.scales[c.tables[2, 4].long(), 0] = 0
    q = torch.randn((sum(ns), 8 * hd), generator=_gen(26), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, ns, 4)
    assert st.item() == 0
    _check_by_weight(c, q, lens, ns, 4, out)


@pytest.mark.parametrize("many", [0, 30])
def test_large_queries_against_the_definition(E, many):
    """Scores of some hundreds: the weights are those of few tokens."""
    c = Cache(1, 1 << 20 if many else 200, 1, 64, 6, used=200)
    q = (300 * torch.randn((1 + many, 4 * 64), generator=_gen(1), device="cuda")).to(torch.bfloat16)
    out, _ = _attend(E, c, q, [33], [1 + many], 4)
    _check_by_weight(c, q, [33], [1 + many], 4, out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("power", [8, 20, 24, 26, 30, 60])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("max_len", MAX_LENS)
def test_equal_scores_have_equal_weights(E, hd, power, n, max_len):
    """All keys alike: however large the scores, an output is the mean of V, and pages of other V scales do not change that."""
    L = 290
    c = Cache(1, max_len, 1, hd, 27, used=320)
    key = (40 * torch.randn(hd, generator=_gen(28), device="cuda")).to(torch.float8_e4m3fn)
    c.codes[:, 0] = key
    c.scales[:, 0] = 2.0 ** -6
    c.scales[:, 1] = torch.exp2(torch.randint(-9, 4, c.scales[:, 1].shape, generator=_gen(29), device="cuda").float())
    q = (2.0 ** power * torch.randn((n, 4 * hd), generator=_gen(30), device="cuda")).to(torch.bfloat16)
    out, _ = _attend(E, c, q, [L], [n], 4)
    V = c.values(0, L)[1][0]
    for i in range(n):
        sees = L - n + 1 + i
        mean, spread = V[:sees].mean(0), V[:sees].abs().mean(0)
        # (a weight is exact but for its rounding to fp16 and the sum's roundings)
        tol = (HALF_F16 + 2.0 ** -16) * spread + HALF_BF16 * (mean.abs() + HALF_F16 * spread)
        assert ((out[i].to(F64).view(4, hd) - mean).abs() <= tol).all(), i


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B", [48, 49, 700, 4096, 4200])
def test_many_requests_with_several_tokens_each(E, hd, B):
    """Some hundreds or thousands of requests for the kernel for many rows, many of one length, some without rows: each row is computed, and once."""
    G, Hkv = 8, 1
    ns = [(5 + 7 * i) % 41 if i % 3 else 0 for i in range(B)]
    ns[B // 2], ns[B - 1] = 200, 33
    lens = [n + (13 * i) % 50 if i % 4 else 150 + n // 2 for i, n in enumerate(ns)]
    c = Cache(B, 1 << 20, Hkv, hd, B, used=max(lens))
    T = sum(ns)
    q = torch.randn((T + 2, G * hd), generator=_gen(B), device="cuda").to(torch.bfloat16)
    out, st = _attend(E, c, q, lens, ns, G)
    assert st.item() == 0 and (out[T:] == 55).all()
    starts = _rows(ns)[1]
    for b in sorted({0, 1, 2, 4, B // 2, B - 2, B - 1, *range(5, B, max(1, B // 40))}):
        if ns[b]:
            _check_attention(Part(c, b), q, [lens[b]], [ns[b]], G, out, f"request {b}", row0=starts[b])
    one, _ = _attend(E, c, q, lens, ns, G, max_len=max(lens))           # (fewer tokens at most: other kernels, other chunks)
    assert torch.equal(torch.isfinite(one.float()), torch.isfinite(out.float())) and ((one.float() - out.float()).abs() <= 0.05 * out.float().abs().amax(1, keepdim=True)).all()


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ns,lens", [([1, 3, 20], [8, 40, 45]), ([2, 1, 9], [16, 18, 25])])
def test_append_to_pages_with_scales_that_are_no_powers_of_two(E, hd, ns, lens):
    """Tokens behind others whose scale another program has chosen: larger than the new ones need, it stays and the new codes are quotients by it;
    smaller, the older codes are rescaled by a factor that is no power of two."""
    Hkv = 4
    c, g = Cache(3, 64, Hkv, hd, 31, fill=0.0), _gen(32)
    c.codes.copy_((torch.randn(c.codes.shape, generator=g, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn))
    c.scales.copy_(torch.rand(c.scales.shape, generator=g, device="cuda") * 0.05)      # about half of them larger than 3 / 448 to the next power
    c.scales[:, :, 0] *= 0.01                              # heads that certainly grow, and one that certainly does not
    c.scales[:, :, 1] += 0.1
    x = torch.randn((sum(ns), 2 * Hkv, hd), generator=g, device="cuda").to(torch.bfloat16)
    codes, scales, st = c.codes.to(F64), c.scales.clone(), _status()
    _, want = _append_reference(c.codes, c.scales, x[:, :Hkv], x[:, Hkv:], c.tables, lens, ns)
    E.epara_kv8_append(x[:, :Hkv], x[:, Hkv:], c.codes, c.scales, _int(lens), c.tables, 64, st, _st(), q_rows=_rows(ns)[0], max_q=max(ns))
    assert st.item() == 0 and torch.equal(c.scales.to(F64), want)
    got, start, kept, grown = c.codes.to(F64), 0, 0, 0
    for b, (n, L) in enumerate(zip(ns, lens)):
        for pos in range((L - n) // 16 * 16, L):
            page, slot, t = int(c.tables[b, pos // 16]), pos % 16, pos - (L - n)
            now = want[page]                               # [2, Hkv]
            if t >= 0:
                exact = x[start + t].to(F64).view(2, Hkv, hd) / now[..., None]
            else:
                f = scales[page].to(F64) / now
                kept, grown = kept + int((f == 1).sum()), grown + int((f < 1).sum())
                exact = codes[page][:, :, slot] * f[..., None]
            # the nearest code, but for a product or quotient whose own rounding in fp32 has put it on the other side of a border
            step = torch.exp2(torch.floor(torch.log2(exact.abs().clamp(min=2.0 ** -6))) - 3)
            assert ((got[page][:, :, slot] - exact).abs() <= 0.5 * step + HALF_F32 * exact.abs()).all()
        start += n
    assert kept > 0 and grown > 0                          # both were there


# ------------------------------------------------------------------------------------------------ product
@pytest.mark.parametrize("M", [3, 127, 700])
@pytest.mark.parametrize("epi", [2, 3])
def test_gelu_to_the_end_of_its_tail(E, M, epi):
    """x from -9 to 9: relative to the result, GELU is as good as the bf16 that it is stored in."""
    N, K = 255, 16
    A, W = torch.zeros((M, 16), dtype=torch.int8, device="cuda"), torch.zeros((N, 16), dtype=torch.int8, device="cuda")
    A[:, 0] = torch.linspace(127, 1, M, device="cuda").to(torch.int8)
    W[:, 0] = torch.arange(-127, 128, device="cuda").to(torch.int8)
    p = dict(A=A, W=W, M=M, N=N, K=K, epilogue=epi, a_scale=torch.full((M,), 9 / 127, device="cuda"), w_scale=torch.full((N,), 1 / 127, device="cuda"),
             bias=torch.full((N,), -0.25, device="cuda").to(torch.bfloat16), C=torch.empty((M, N), dtype=torch.bfloat16, device="cuda"))
    st = _status()
    E.epara_gemm_i8(p, _st(), st)
    x = A[:, :1].to(F64) * W[:, 0].to(F64) * p["a_scale"][:, None].to(F64) * p["w_scale"].to(F64) - (0.25 if epi & 1 else 0)
    want = 0.5 * x * torch.special.erfc(-x / math.sqrt(2))
    # x has three roundings in fp32, an error of at most 2^-22 x 10, by which the tail changes by up to 10 times its own value; the function itself
    # within 2^-13
    tol = (HALF_BF16 * (1 + 2.0 ** -11) + 2.0 ** -13 + 100 * 2.0 ** -22) * want.abs()
    _within(p["C"], want, tol, f"M={M} epi={epi}")


def test_gelu_of_what_is_not_finite(E):
    M, N, K = 5, 32, 16
    for rows in (M, 700):
        A, W = torch.ones((rows, 16), dtype=torch.int8, device="cuda"), torch.ones((N, 16), dtype=torch.int8, device="cuda")
        W[1::2] = -1
        a = torch.ones(rows, device="cuda")
        a[0], a[1], a[2] = math.inf, math.nan, 1e30
        p = dict(A=A, W=W, M=rows, N=N, K=K, epilogue=2, a_scale=a, w_scale=torch.ones(N, device="cuda"), C=torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"))
        E.epara_gemm_i8(p, _st(), _status())
        out = p["C"].float()
        assert (out[0, 0::2] == math.inf).all() and torch.isnan(out[0, 1::2]).all() and torch.isnan(out[1]).all()
        assert ((out[2, 0::2] / 1.6e31 - 1).abs() < 2.0 ** -8).all() and (out[2, 1::2] == 0).all()


@pytest.mark.parametrize("epi", [0, 1, 2, 3, 4, 5, 8, 9, 11])
def test_a_row_has_the_same_bits_in_every_batch(E, epi):
    """Whichever kernel a batch runs on, each epilogue; the fp32 stream has subnormal values among the others."""
    M, N, K, g = 1100, 512, 1000, _gen(33)
    ld = (K + 15) // 16 * 16
    A, W = (torch.randint(-128, 128, (n, ld), generator=g, device="cuda", dtype=torch.int8) for n in (M, N))
    a, w = (0.5 + torch.rand((M,), generator=g, device="cuda")) / 64, (0.5 + torch.rand((N,), generator=g, device="cuda")) / 2000
    a[::7] = 2.0 ** -120                                   # ... and products that are subnormal
    bias = torch.randn((N,), generator=g, device="cuda").to(torch.bfloat16)
    bias[::3] = 0
    cols = N // 2 if epi & 4 else N
    C0 = torch.randn((M, cols), generator=g, device="cuda") if epi & 8 else torch.zeros((M, cols), dtype=torch.bfloat16, device="cuda")
    if epi & 8:
        C0[::7, ::2] = 1e-40 * torch.randn(C0[::7, ::2].shape, generator=g, device="cuda")
    outs, st = [], _status()
    for m in (1100, 300, 50, 12, 1):
        C = C0[:m].clone()
        E.epara_gemm_i8(dict(A=A, W=W, a_scale=a, w_scale=w, bias=bias, C=C, M=m, N=N, K=K, epilogue=epi), _st(), st)
        outs.append(C)
    for C in outs[1:]:
        assert torch.equal(C.view(torch.int32 if epi & 8 else torch.int16), outs[0][:len(C)].view(torch.int32 if epi & 8 else torch.int16)), len(C)
    if epi == 8:                                           # and the sum is rounded once, subnormal or not
        acc = (A[:, :K].to(F64) @ W[:, :K].to(F64).t()).float()
        assert torch.equal(outs[0], C0 + acc * a[:, None] * w)


# ------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("rows", [1, 5, 300])
@pytest.mark.parametrize("d", [1, 64, 1111, 4095, 4096, 8200, 20001])
def test_norm_of_the_fp32_stream_alone(E, rows, d):
    """x in fp32 with gains and without a residual: the call a layer makes."""
    g = _gen(rows + d)
    x = torch.randn((rows, d), generator=g, device="cuda")
    gain = (1 + 0.3 * torch.randn((d,), generator=g, device="cuda")).to(torch.bfloat16)
    q, s = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    E.epara_rms_norm_i8(x, gain, q, s, _st())
    _check_norm(x, None, gain, q, s, None)


@pytest.mark.parametrize("x_type,resid", [("bf16", False), ("f32", True)])
def test_norm_of_very_long_rows(E, x_type, resid):
    """Rows of some millions of like values, where a running fp32 sum loses a little with every addition."""
    d = (1 << 23) + 5
    x = torch.full((2, d), 1.1, device="cuda").to(torch.bfloat16 if x_type == "bf16" else torch.float32)
    x[1] += 0.01 * torch.randn((d,), generator=_gen(34), device="cuda").to(x.dtype)
    r = torch.full((2, d), 0.3, device="cuda") if resid else None
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty((2, d), dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    r_out = torch.empty_like(r) if resid else None
    E.epara_rms_norm_i8(x, gain, q, s, _st(), resid=r, resid_out=r_out)
    _check_norm(x, r, gain, q, s, r_out)
