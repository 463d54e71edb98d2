"""Tables in 4 bits (ember_quantize_rows_q4, ember_rows_q4, ember_logits_q4), through the C ABI.

A code times its bf16 scale has at most 11 significant bits, so a row read back is
that product, exact in fp32 and rounded once to bf16: the same bits as torch's.
Rounding to 4 bits is fp32 and correctly rounded, and so is torch's: the same codes.
A logit is a sum of n_g terms (an exact integer to fp32, times a scale, added: two
roundings a term if they are not fused), times the token's scale, plus the bias:
|Y - E| <= u (2 n_g + 3) sum_g |term| xs + u |Y| with u = 2^-24, and 2^-8 |E| more in bf16."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def em():
    from paper_2607_01455_amd import ember
    return ember


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def mat(rows, cols, dtype, extra=1, fill=None):
    """rows x cols, rows on 16-byte boundaries, the padding NaN (or for codes 0x5A)."""
    q = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = ((cols + q - 1) // q + extra) * q
    if fill is None:
        fill = float("nan") if dtype.is_floating_point else 0x5A
    return torch.full((rows, ld), fill, dtype=dtype, device=DEV)[:, :cols]


def where(D):
    """Byte and half of each column's code."""
    k = torch.arange(D, device=DEV)
    return k // 128 * 64 + k % 16 // 4 * 16 + k % 128 // 32 * 4 + k % 4, k % 32 // 16


def pack(codes, extra=1, garbage=0):
    """Codes (rows x D, -8..7) as the library packs them; the codes past D are `garbage`."""
    rows, D = codes.shape
    full = torch.full((rows, (D + 127) // 128 * 128), garbage, dtype=torch.int64, device=DEV)
    full[:, :D] = codes
    at, half = where(full.shape[1])
    Q = mat(rows, full.shape[1] // 2, torch.uint8, extra)
    lo, hi = full[:, half == 0] & 15, full[:, half == 1] & 15
    Q[:, at[half == 0]] = lo.to(torch.uint8)
    Q[:, at[half == 1]] |= (hi << 4).to(torch.uint8)
    return Q


def unpack(Q, D):
    at, half = where(D)
    n = (Q[:, at].to(torch.int64) >> (4 * half)) & 15
    return torch.where(n > 7, n - 16, n)


def table(V, D, group, seed, extra=1, lo=-8):
    g = gen(seed)
    codes = torch.randint(lo, 8, (V, D), generator=g, device=DEV)
    n = (D + group - 1) // group
    scale = mat(V, n, BF, extra)
    scale.copy_(torch.rand(V, n, generator=g, device=DEV) * 0.01 + 1e-3)
    return codes, pack(codes, extra, garbage=-3), scale


def values(codes, scale, group):
    return codes.double() * scale.double().repeat_interleave(group, dim=1)[:, :codes.shape[1]]


def tokens(T, D, seed, extra=1):
    g = gen(seed)
    X = mat(T, D, torch.int8, extra)
    X.copy_(torch.randint(-128, 128, (T, D), generator=g, device=DEV, dtype=torch.int8))
    return X, torch.rand(T, generator=g, device=DEV) + 0.1


# ---------------------------------------------------------------------------
# rounding and reading back
# ---------------------------------------------------------------------------

def rounded(X, group):
    """Codes and scales as the header has them, in torch's fp32."""
    rows, D = X.shape
    x = torch.nn.functional.pad(X.float(), (0, -D % group)).view(rows, -1, group)
    a = x.abs().amax(dim=2)
    s = (a * (1 / 7)).to(BF)                   # the fp32 nearest 1/7, a product rounded to fp32, then to bf16
    c = torch.round(x / s.float()[:, :, None])
    c = torch.where((a >= 1e-36)[:, :, None], c, 0.0)
    return c.view(rows, -1)[:, :D].long(), torch.where(a >= 1e-36, s, 0.0)


@pytest.mark.parametrize("V,D", [(1, 1), (3, 31), (5, 32), (7, 33), (2, 127), (4, 128), (9, 129), (100, 1000), (64, 4096),
                                 (33, 896), (1000, 64), (5, 32768), (3, 8193), (2049, 200), (70000, 16)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F])
def test_rows_to_4_bits_and_back(em, V, D, group, dtype):
    print(f"q4 rows V={V} D={D} group={group} {dtype}", flush=True)
    X = mat(V, D, dtype)
    X.copy_(torch.randn(V, D, generator=gen(V + D), device=DEV) * torch.rand(D, generator=gen(D), device=DEV))
    X[0] = 0                                   # groups of zeros
    X[-1] *= 1e-30                             # small, but not zeros
    n, nbytes = (D + group - 1) // group, (D + 127) // 128 * 64
    Q, s = mat(V, nbytes, torch.uint8), mat(V, n, BF)
    em.ember_quantize_rows_q4(X, Q, s, group)
    want, scale = rounded(X, group)
    assert torch.equal(s, scale)
    assert torch.equal(unpack(Q, D), want)
    assert (unpack(Q, nbytes * 2)[:, D:] == 0).all()
    assert (Q._base[:, nbytes:] == 0x5A).all() and torch.isnan(s._base[:, n:].float()).all()   # padding is left alone
    step = s.double().repeat_interleave(group, dim=1)[:, :D]
    assert ((X.double() - want.double() * step).abs() <= step / 2 * (1 + 2.0 ** -20)).all()
    for out in (BF, F):
        Y = mat(V, D, out)
        em.ember_rows_q4(Q, s, Y, group)
        assert torch.equal(Y, values(want, s, group).to(out))
        assert torch.isnan(Y._base[:, D:].float()).all()


@pytest.mark.parametrize("group", [32, 64, 128])
def test_groups_that_are_not_finite(em, group):
    D = 300
    X = torch.randn(6, 304, generator=gen(1), device=DEV)[:, :D]
    X[1, 5], X[2, 200], X[3, 299] = float("nan"), float("inf"), -float("inf")
    X[4, :32] = 3.0e38
    X[5] = 1e-37
    head = em.HeadQ4.from_table(X, group)
    n = (D + group - 1) // group
    bad = torch.zeros(6, n, dtype=torch.bool, device=DEV)
    for r, k in ((1, 5), (2, 200), (3, 299)):
        bad[r, k // group] = True
    assert torch.equal(torch.isnan(head.wscale), bad)
    assert torch.isfinite(head.wscale[4]).all() and (head.wscale[5] == 0).all()
    codes = unpack(head.Wq, D)
    assert (codes[bad.repeat_interleave(group, dim=1)[:, :D]] == 0).all()
    fine = X.clone()
    fine[1, 5] = fine[2, 200] = fine[3, 299] = 0
    other = em.HeadQ4.from_table(fine, group)
    assert torch.equal(head.wscale[~bad], other.wscale[~bad])
    # a channel with such a group has NaN logits, the others none
    for T in (3, 200):
        Xq, xs = tokens(T, D, T)
        Y = mat(T, 6, F)
        head.logits(Xq, xs, Y)
        assert torch.equal(torch.isnan(Y), bad.any(dim=1).expand(T, 6))


@pytest.mark.parametrize("V,D,group", [(50, 100, 32), (1000, 1000, 64), (300, 4096, 128), (7, 33, 128)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_rows_of_tokens(em, V, D, group, dtype):
    print(f"q4 gather V={V} D={D} group={group} {dtype}", flush=True)
    codes, Q, s = table(V, D, group, 3)
    want = values(codes, s, group).to(dtype)
    for n in (1, 2, 63, 500):
        tok = torch.randint(0, V, (n,), generator=gen(n), device=DEV)
        tok[-1] = V - 1
        tok[n // 2] = tok[0]
        if n > 2:
            tok[1], tok[2] = -1, V             # tokens outside the table
            if n > 100:
                tok[50], tok[51] = 2 ** 62, -2 ** 63
        Y = mat(n, D, dtype)
        em.ember_rows_q4(Q, s, Y, group, tok)
        inside = (tok >= 0) & (tok < V)
        assert torch.equal(Y[inside], want[tok[inside]])
        assert torch.isnan(Y[~inside].float()).all()
        assert torch.isnan(Y._base[:, D:].float()).all()
    # the first rows of the table, and none
    Y = mat(V // 2, D, dtype)
    em.ember_rows_q4(Q, s, Y, group)
    assert torch.equal(Y, want[:V // 2])
    em.ember_rows_q4(Q, s, Y[:0], group, torch.empty(0, dtype=torch.int64, device=DEV))
    em.ember_quantize_rows_q4(Y[:0].float(), Q[:0], s[:0], group)


# ---------------------------------------------------------------------------
# logits
# ---------------------------------------------------------------------------

def check(em, T, V, D, group, dtype, bias, seed=0, extra=1):
    codes, Q, s = table(V, D, group, seed + 1, extra)
    Xq, xs = tokens(T, D, seed + 2, extra)
    b = torch.randn(V, generator=gen(5), device=DEV) if bias else None
    Y = mat(T, V, dtype, extra)
    em.HeadQ4(Q, s, D, group, b).logits(Xq, xs, Y)
    near(Y, codes, s, group, Xq, xs, b)
    assert torch.isnan(Y._base[:, V:].float()).all()


def near(Y, codes, s, group, Xq, xs, b):
    T, D = Xq.shape
    n = s.shape[1]
    E = torch.zeros(T, len(codes), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(E)
    for g in range(n):
        k = slice(g * group, min(D, (g + 1) * group))
        term = Xq[:, k].double() @ codes[:, k].double().t().contiguous() * s[:, g].double() * xs.double()[:, None]
        E += term
        size += term.abs()
    if b is not None:
        E += b.double()
    bar = U * (2 * n + 3) * size + U * E.abs() * 2
    if Y.dtype == BF:
        bar = bar + 2.0 ** -8 * E.abs()
    assert ((Y.double() - E).abs() <= bar + 1e-37).all()


SHAPES = [(1, 1, 1), (1, 5, 16), (1, 300, 64), (2, 1000, 200), (3, 64, 4096), (5, 257, 1023), (15, 2000, 130),
          (16, 513, 512), (17, 600, 96), (31, 100, 77), (32, 1024, 64), (33, 1025, 640), (64, 256, 128), (65, 700, 1000),
          (100, 4097, 48), (129, 515, 333), (255, 256, 256), (256, 1000, 896), (300, 3001, 520), (513, 770, 100),
          (1, 40000, 256), (1, 70001, 384), (2, 37, 32768), (4, 129, 17), (16, 130, 8192), (16, 33, 32768), (40, 300, 8200),
          (700, 2500, 72), (17, 90, 4097), (9, 5000, 1040), (12, 3000, 768), (32, 4097, 1024), (64, 3000, 2048),
          (64, 2000, 2300), (500, 2001, 1100), (1025, 300, 1000), (128, 3333, 999), (1, 3, 15), (1, 16385, 2047)]


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_logits(em, T, V, D, group):
    dtype, bias = (BF, F)[(T + V + group // 32) % 2], (V + D) % 3 == 0
    print(f"q4 logits T={T} V={V} D={D} group={group} {dtype} bias={bias}", flush=True)
    check(em, T, V, D, group, dtype, bias, extra=(T + D) % 2)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_logits_of_few_and_odd_steps(em, group):
    """Tiles of many tokens with 1 to 9 blocks of columns, the last one whole or not."""
    for T in (70, 700):
        for D in (1, 128, 129, 250, 256, 300, 384, 500, 513, 640, 768, 800, 1000, 1040):
            print(f"q4 steps T={T} D={D} group={group}", flush=True)
            check(em, T, 150, D, group, F, True, seed=D)


@pytest.mark.parametrize("T,V,D", [(700, 20001, 1000), (130, 70001, 700), (1000, 33000, 200), (70, 66000, 900)])
@pytest.mark.parametrize("group,dtype", [(32, BF), (64, F), (128, BF)])
def test_more_tiles_than_blocks(em, T, V, D, group, dtype):
    """Blocks that go on to other tiles, and of few steps one a tile."""
    print(f"q4 tiles T={T} V={V} D={D} group={group} {dtype}", flush=True)
    check(em, T, V, D, group, dtype, True)


@pytest.mark.parametrize("T", [1, 20, 50, 70, 300])
def test_logits_of_one_scale_are_exact_integers(em, T):
    """Scales that are powers of two: every partial sum is an integer below 2^24."""
    V, D = 777, 1000
    codes, Q, _ = table(V, D, 64, 9)
    s = torch.full((V, 16), 2.0 ** -4, dtype=BF, device=DEV)
    Xq, _ = tokens(T, D, 3)
    Y = mat(T, V, F)
    em.ember_logits_q4(Xq, torch.ones(T, device=DEV), Q, s, Y, 64)
    assert torch.equal(Y.double(), Xq.double() @ codes.double().t().contiguous() / 16)


def test_largest_group_sums(em):
    """Codes of -8 and states of -128 in groups of 128: sums of 2^17 a group, 2^21 as the operands have them."""
    D = 32768
    Q = pack(torch.full((40, D), -8, device=DEV))
    s = torch.ones(40, D // 128, dtype=BF, device=DEV)
    for T in (1, 20, 130):
        Xq = torch.full((T, D), -128, dtype=torch.int8, device=DEV)
        Y = mat(T, 40, F)
        em.ember_logits_q4(Xq, torch.ones(T, device=DEV), Q, s, Y, 128)
        assert (Y == 1024.0 * D).all()


def test_scales_that_are_not_finite(em):
    for T in (5, 40, 130):
        codes, Q, s = table(333, 200, 32, 4)
        Xq, xs = tokens(T, 200, 3)
        xs[2] = float("nan")
        s[7, 6] = float("inf")
        Y = mat(T, 333, F)
        em.ember_logits_q4(Xq, xs, Q, s, Y, 32)
        assert torch.isnan(Y[2]).all()
        rest = torch.arange(T, device=DEV) != 2
        cols = torch.arange(333, device=DEV) != 7
        near(Y[rest][:, cols], codes[cols], s[cols], 32, Xq[rest], xs[rest], None)


def test_offsets_past_32_bits(em):
    """2.3 GB of codes and their scales: the last rows are where the offsets say."""
    V, D = 140000, 32768
    print("q4 table of 2.3 GB", flush=True)
    Q = torch.zeros(V, D // 2, dtype=torch.uint8, device=DEV)
    s = torch.ones(V, D // 128, dtype=BF, device=DEV)
    codes, Qt, st = table(200, D, 128, 8, 0)
    Q[V - 200:], s[V - 200:] = Qt, st
    for T in (3, 40):
        Xq, xs = tokens(T, D, 9, 0)
        Y = mat(T, V, F, 0)
        em.ember_logits_q4(Xq, xs, Q, s, Y, 128)
        near(Y[:, V - 200:], codes, st, 128, Xq, xs, None)
        assert (Y[:, :V - 200] == 0).all()
    tok = torch.tensor([V - 1, 0, V - 200], device=DEV)
    Y = mat(3, D, F, 0)
    em.ember_rows_q4(Q, s, Y, 128, tok)
    want = values(codes, st, 128).float()
    assert torch.equal(Y[0], want[-1]) and torch.equal(Y[2], want[0]) and (Y[1] == 0).all()
    X = torch.zeros(V, D, dtype=BF, device=DEV)
    X[V - 200:] = want.to(BF)
    Q.zero_()
    s.zero_()
    print("q4 rounding a table of 9.2 GB", flush=True)
    em.ember_quantize_rows_q4(X, Q, s, 128)
    c, sc = rounded(X[V - 200:], 128)
    assert torch.equal(unpack(Q[V - 200:], D), c) and torch.equal(s[V - 200:], sc) and (Q[:V - 200] == 0).all()


def test_wide_strides(em):
    """Rows at the largest strides: what counts is the row's own offset."""
    ld = (1 << 22) - 16
    n = 600
    buf = torch.zeros(n * ld, dtype=torch.uint8, device=DEV)
    codes, Qt, s = table(n, 48, 32, 1, 0)
    Q = buf.as_strided((n, 64), (ld, 1))
    Q.copy_(Qt)
    for T in (1, 20, 70, 300):
        print(f"q4 wide strides T={T}", flush=True)
        Xq, xs = tokens(T, 48, T)
        Y = mat(T, n, F, 0)
        em.ember_logits_q4(Xq, xs, Q, s, Y, 32)
        near(Y, codes, s, 32, Xq, xs, None)
    Y = mat(n, 48, F)
    em.ember_rows_q4(Q, s, Y, 32)
    assert torch.equal(Y, values(codes, s, 32).float())
    del buf, Q
    far = torch.zeros(n * ld, dtype=torch.int8, device=DEV).as_strided((n, 48), (ld, 1))
    for V in (40, 300):
        Xq, xs = tokens(n, 48, V)
        far.copy_(Xq)
        Y = mat(n, V, F, 0)
        em.ember_logits_q4(far, xs, Qt[:V], s[:V], Y, 32)
        near(Y, codes[:V], s[:V], 32, Xq, xs, None)


def test_wide_scale_strides(em):
    """Scales at the largest strides, the rows between them NaN."""
    ld, n = (1 << 22) - 8, 300
    codes, Q, st = table(n, 1000, 32, 1, 0)
    s = torch.full((n * ld,), float("nan"), dtype=BF, device=DEV).as_strided((n, 32), (ld, 1))
    s.copy_(st)
    for T in (1, 20, 70, 300, 1000):
        print(f"q4 wide scale strides T={T}", flush=True)
        Xq, xs = tokens(T, 1000, T)
        Y = mat(T, n, F, 0)
        em.ember_logits_q4(Xq, xs, Q, s, Y, 32)
        near(Y, codes, st, 32, Xq, xs, None)
    Y = mat(n, 1000, F)
    em.ember_rows_q4(Q, s, Y, 32)
    assert torch.equal(Y, values(codes, st, 32).float())


def test_more_rows_than_a_launch(em):
    """2^20 blocks of 64 rows and some more: the rows behind them are where those before are."""
    V, D = (1 << 26) + 3000, 8
    print("q4 rows V=2^26 + 3000", flush=True)
    X = torch.randn(V, D, generator=gen(3), device=DEV).to(BF)
    Q = torch.full((V, 64), 0x5A, dtype=torch.uint8, device=DEV)
    s = torch.full((V, 8), 7.0, dtype=BF, device=DEV)
    em.ember_quantize_rows_q4(X, Q, s[:, :1], 32)
    Y = torch.full((V, D), float("nan"), dtype=BF, device=DEV)
    em.ember_rows_q4(Q, s[:, :1], Y, 32)
    for a, b in ((0, 5000), (V - 5000, V)):
        c, sc = rounded(X[a:b], 32)
        assert torch.equal(unpack(Q[a:b], D), c) and torch.equal(s[a:b, :1], sc)
        assert torch.equal(Y[a:b], values(c, sc, 32).to(BF))
    # a code is off by half a step at most, the scale by 2^-8: 7 * 2^-8 of a step more
    err = (X.float() - Y.float()).abs().amax(dim=1)
    assert (err <= s[:, 0].float() * (0.5 + 7 * 2.0 ** -8) * (1 + 2.0 ** -7)).all()


def test_a_part_of_a_table(em):
    """Channels of a larger table: what lies behind them is not read into them."""
    codes, Q, s = table(500, 300, 64, 2)
    for T in (1, 33, 200):
        Xq, xs = tokens(T, 300, T)
        for a, b in ((0, 1), (3, 20), (17, 400), (499, 500)):
            Y = mat(T, b - a, F)
            em.ember_logits_q4(Xq, xs, Q[a:b], s[a:b], Y, 64)
            near(Y, codes[a:b], s[a:b], 64, Xq, xs, None)


def test_same_bits_for_a_token_alone_and_among_others(em):
    """Within the streaming form a token's logits do not depend on the other tokens."""
    codes, Q, s = table(3000, 1000, 128, 2)
    Xq, xs = tokens(60, 1000, 7)
    whole = mat(60, 3000, F)
    em.ember_logits_q4(Xq, xs, Q, s, whole, 128)
    for n in (1, 16, 17, 40):
        Y = mat(n, 3000, F)
        em.ember_logits_q4(Xq[:n], xs[:n], Q, s, Y, 128)
        assert torch.equal(Y, whole[:n])


def test_on_another_stream_and_in_a_graph(em):
    for T in (2, 40, 150):
        codes, Q, s = table(777, 300, 32, 4)
        Xq, xs = tokens(T, 300, 3)
        Y, R = mat(T, 777, BF), mat(T, 300, BF)
        tok = torch.randint(0, 777, (T,), generator=gen(1), device=DEV)

        def call():
            em.ember_logits_q4(Xq, xs, Q, s, Y, 32)
            em.ember_rows_q4(Q, s, R, 32, tok)

        call()
        want = Y.clone(), R.clone()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            Y.zero_()
            R.zero_()
            call()
        side.synchronize()
        assert torch.equal(Y, want[0]) and torch.equal(R, want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for k in range(3):
            xs.copy_(torch.rand(T, device=DEV))
            tok.copy_(torch.randint(0, 777, (T,), device=DEV))
            call()
            want = Y.clone(), R.clone()
            Y.zero_()
            R.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(Y, want[0]) and torch.equal(R, want[1]), (T, k)


def test_no_tokens(em):
    _, Q, s = table(10, 40, 32, 1)
    em.ember_logits_q4(torch.empty(0, 48, dtype=torch.int8, device=DEV)[:, :40], torch.empty(0, device=DEV), Q, s,
                       torch.empty(0, 10, device=DEV), 32)


# Shapes by the form that answers them: the streaming form in tiles of 32 tokens (waves that share strips up to 32736
# channels, several strips a wave from there), in two such tiles, in tiles of 16 for 17 to 32 tokens of more columns than
# the LDS holds of 32 (groups of 128: tiles), and in windows of the columns where it does not hold 16 or fewer either,
# a strip a wave.
STREAMED = [(17, 16385, 1000), (18, 16384, 512), (25, 20000, 96), (31, 20001, 4097), (32, 33000, 2047), (24, 40003, 640),
            (32, 32737, 4600), (17, 131073, 200),
            (33, 65665, 1000), (64, 70001, 2047), (63, 65537, 130), (48, 131072, 512), (40, 99999, 33),
            (20, 40001, 8192), (17, 32769, 4700), (32, 33001, 12000),
            (16, 40001, 12000), (5, 33001, 32768), (13, 32737, 15000)]


@pytest.mark.parametrize("T,V,D", STREAMED)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F])
def test_logits_of_few_tokens_and_many_channels(em, T, V, D, group, dtype):
    print(f"q4 streamed T={T} V={V} D={D} group={group} {dtype}", flush=True)
    check(em, T, V, D, group, dtype, (T + V + group // 32) % 2 == 0, extra=(V + D) % 2)


@pytest.mark.parametrize("V,D,counts", [(16384, 1000, (1, 16, 17, 31)), (33000, 4500, (2, 16, 17, 32)),
                                        (70000, 1000, (1, 15, 16, 17, 32, 33, 63)), (66000, 2048, (1, 16, 32, 48))])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_same_bits_in_every_streaming_form(em, V, D, counts, group):
    """Tiles of 16, of 32 and of twice 32 tokens add a logit's groups in one order."""
    print(f"q4 streamed bits V={V} D={D} group={group}", flush=True)
    codes, Q, s = table(V, D, group, 2)
    del codes
    most = max(counts) + 1 if max(counts) % 32 else max(counts)
    Xq, xs = tokens(most, D, 7)
    whole = mat(most, V, F)
    em.ember_logits_q4(Xq, xs, Q, s, whole, group)
    for n in counts:
        Y = mat(n, V, F)
        em.ember_logits_q4(Xq[most - n:], xs[most - n:], Q, s, Y, group)
        assert torch.equal(Y, whole[most - n:]), n


def test_scales_that_are_not_finite_of_many_channels(em):
    """What stands behind a row's scales, or in another row's, does not reach a channel (widest tiles and windows)."""
    for T, V, D in ((20, 16400, 200), (50, 66000, 200), (12, 33000, 13000), (30, 33000, 5000)):
        print(f"q4 streamed scales T={T} V={V} D={D}", flush=True)
        codes, Q, s = table(V, D, 32, 4)                  # the scales' padding is NaN
        Xq, xs = tokens(T, D, 3)
        xs[2] = float("nan")
        s[7, 6], s[V - 1, 0] = float("inf"), float("nan")
        Y = mat(T, V, F)
        em.ember_logits_q4(Xq, xs, Q, s, Y, 32)
        assert torch.isnan(Y[2]).all() and torch.isnan(Y[:, V - 1]).all()
        rest = torch.arange(T, device=DEV) != 2
        cols = (torch.arange(V, device=DEV) != 7) & (torch.arange(V, device=DEV) != V - 1)
        near(Y[rest][:, cols], codes[cols], s[cols], 32, Xq[rest], xs[rest], None)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F])
def test_scales_against_a_seventh_of_the_largest(em, group, dtype):
    """s = a / 7 (1 + d1) (1 + d2) (1 + d3): the constant and the product within 2^-24 each, bf16 to the nearest of
    what that gives: |s - a / 7| <= half a step of bf16 + a / 7 (2^-23 + 2^-47), below 2^-22 a / 7 more than half a step."""
    V, D = 4000, 8 * group
    X = torch.randn(V, D, generator=gen(group), device=DEV) * torch.rand(V, 1, generator=gen(1), device=DEV) * 10
    if dtype == F:
        # ties of a / 7 between two scales, and the fp32 next to them
        k = torch.arange(128, 256, device=DEV, dtype=torch.float64)
        tie = (7 * (2 * k + 1)).float()
        X[:128] *= 1e-3
        X[:128, 0], X[:128, group] = tie, torch.nextafter(tie, torch.zeros_like(tie))
        X[:128, 2 * group] = torch.nextafter(tie, tie * 2)
    X = X.to(dtype)
    head = em.HeadQ4.from_table(X, group)
    a = X.double().view(V, 8, group).abs().amax(dim=2)
    s = head.wscale.double()
    half = torch.exp2(torch.floor(torch.log2(a / 7)) - 8)
    assert ((s - a / 7).abs() <= half + a / 7 * 2.0 ** -22).all()


@pytest.mark.parametrize("D,group", [(4096, 128), (1000, 64), (1001, 32), (8191, 128)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_rows_on_both_sides_of_the_store_limit(em, D, group, dtype):
    """About 96 MiB of rows, where stores past the caches begin: each row is its token's, the padding is left alone,
    and a reader next on the stream has them."""
    V = 700
    codes, Q, s = table(V, D, group, 6)
    want = values(codes, s, group).to(dtype)
    limit = -(-(96 << 20) // (D * (4 if dtype == F else 2)))
    for n in (limit - 1, limit, limit + 1):
        print(f"q4 rows D={D} n={n} {dtype}", flush=True)
        tok = torch.randint(0, V, (n,), generator=gen(n), device=DEV)
        tok[n // 3] = V
        Y = mat(n, D, dtype)
        em.ember_rows_q4(Q, s, Y, group, tok)
        same = Y == want[tok.clamp(max=V - 1)]
        same[n // 3] = torch.isnan(Y[n // 3].float())
        assert same.all()
        assert torch.isnan(Y._base[:, D:].float()).all()


@pytest.mark.parametrize("T", [1, 20, 70, 300])
def test_sums_near_the_end_of_fp32(em, T):
    """Sums of up to 2^124 before the token's scale (held times 16, below 2^128), exact: one group, powers of two."""
    V, D = 600, 128
    codes, Q, s = table(V, D, 128, 3)
    Xq, _ = tokens(T, D, 5)
    sums = Xq.double() @ codes.double().t().contiguous()
    top = 123 - int(sums.abs().max().log2().floor())
    s.fill_(2.0 ** top)
    Y = mat(T, V, F)
    em.ember_logits_q4(Xq, torch.full((T,), 2.0 ** -100, device=DEV), Q, s, Y, 128)
    assert torch.equal(Y.double(), sums * 2.0 ** (top - 100))
