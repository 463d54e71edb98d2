"""8-bit logits (ember_logits_q8), through the C ABI.

The sum over D is an integer and exact, so with scales that are powers of two and
no bias the result is the integer, rounded to fp32 and then to Y's type: the same
bits as torch's chain.  With other scales and a bias: acc to fp32, the scales'
product, its product with acc (and the sum with the bias, fused or not) are a
rounding each, |Y - E| <= 4 u (|acc xs ws| + |bias|), u = 2^-24, plus the rounding
to bf16 (2^-8 |E|)."""
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


def codes(rows, D, seed, extra=1, lo=-127):
    """int8 codes in rows on 16-byte boundaries; the padding holds other codes."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld = ((D + 15) // 16 + extra) * 16
    return torch.randint(lo, 128, (rows, ld), generator=g, device=DEV, dtype=torch.int8)[:, :D]


def out(T, V, dtype, extra=1):
    q = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = ((V + q - 1) // q + extra) * q
    return torch.full((T, ld), float("nan"), dtype=dtype, device=DEV)[:, :V]


def sums(Xq, Wq):
    """Exact integer products: float64 holds every sum below 2^53."""
    return Xq.double() @ Wq.double().t().contiguous()


SHAPES = [(1, 1, 1), (1, 5, 16), (1, 300, 64), (2, 1000, 200), (3, 64, 4096), (5, 257, 1023), (15, 2000, 130),
          (16, 513, 512), (17, 600, 96), (31, 100, 77), (32, 1024, 64), (33, 1025, 640), (64, 256, 128),
          (65, 700, 1000), (100, 4097, 48), (129, 515, 333), (255, 256, 256), (256, 1000, 896), (300, 3001, 520),
          (513, 770, 100), (1, 40000, 256), (700, 2500, 72), (2, 37, 32768), (1, 3, 15), (4, 129, 17),
          (16, 130, 8192), (3, 500, 5000), (32, 200, 4096), (30, 333, 3001), (9, 5000, 1040), (16, 9000, 2047),
          (31, 9000, 2048), (2, 70000, 40), (40, 300, 8200), (17, 90, 4097),
          # each tiling, with whole and with ragged 16-column chunks
          (300, 30000, 512), (300, 30001, 500), (257, 40000, 130), (1000, 6000, 256), (600, 9003, 333),
          (333, 8200, 1024), (333, 8191, 1000), (64, 40000, 512), (60, 40003, 300), (64, 30000, 128),
          (129, 9001, 300), (12, 3000, 768), (32, 4097, 1024), (20, 5000, 1001), (64, 3000, 2048), (50, 2001, 1100),
          (257, 40000, 128), (400, 30003, 144), (900, 12345, 64),
          # blocks that go on to other tiles
          (262, 43046, 500), (261, 42975, 512), (386, 56313, 500), (391, 55480, 512), (520, 100003, 500),
          # groups of wavefronts that share the steps
          (500, 2000, 1008), (500, 2000, 1001), (64, 12000, 2064), (60, 12001, 2050), (64, 1500, 4096), (28, 3743, 6096),
          (40, 1000, 8175)]


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F])
def test_exact_sums(em, T, V, D, dtype):
    print(f"logits exact T={T} V={V} D={D} {dtype}", flush=True)
    Xq, Wq = codes(T, D, T + D, 1, -128), codes(V, D, V + D, 2, -128)
    Y = out(T, V, dtype)
    xs = torch.full((T,), 2.0 ** -6, device=DEV)
    xs[::2] = 2.0 ** -9
    ws = torch.full((V,), 0.5, device=DEV)
    ws[::3] = 4.0
    em.ember_logits_q8(Xq, xs, Wq, ws, Y)
    want = (sums(Xq, Wq).float() * xs[:, None] * ws).to(dtype)
    assert torch.equal(Y, want)
    assert torch.isnan(Y._base[:, V:].float()).all()


@pytest.mark.parametrize("T,V,D", [(1, 1000, 100), (7, 2049, 4096), (40, 300, 1023), (200, 1111, 256), (600, 515, 333)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_scales_and_bias(em, T, V, D, dtype):
    print(f"logits scaled T={T} V={V} D={D} {dtype}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(V)
    Xq, Wq = codes(T, D, 1), codes(V, D, 2)
    xs, ws = torch.rand(T, generator=g, device=DEV), torch.rand(V, generator=g, device=DEV) * 1e-2
    bias = torch.randn(V, generator=g, device=DEV)
    if T > 1:
        xs[0] = 0.0
    for b in (None, bias):
        Y = out(T, V, dtype, 0)
        em.HeadQ8(Wq, ws, b).logits(Xq, xs, Y)
        p = sums(Xq, Wq) * xs.double()[:, None] * ws.double()
        E = p if b is None else p + b.double()
        bar = 4 * U * (p.abs() + (0 if b is None else b.double().abs())) + (2.0 ** -8 * E.abs() if dtype == BF else 0)
        assert ((Y.double() - E).abs() <= bar + 1e-37).all()


@pytest.mark.parametrize("V,D,dtype", [(300, 1100, BF), (77, 1024, F), (500, 65, F), (40, 1023, BF)])
def test_head_of_a_table(em, V, D, dtype):
    """from_table: the codes of ember_quantize_rows, wide rows on 128-byte boundaries."""
    g = torch.Generator(device=DEV).manual_seed(V)
    W = out(V, D, dtype, 0).copy_(torch.randn(V, D, generator=g, device=DEV))
    head = em.HeadQ8.from_table(W)
    q, scale = codes(V, D, 1), torch.empty(V, device=DEV)
    em.ember_quantize_rows(W, q, scale)
    assert torch.equal(head.Wq, q) and torch.equal(head.wscale, scale)
    assert head.Wq.stride(0) % (128 if D >= 1024 else 16) == 0 and head.Wq.data_ptr() % 16 == 0
    Xq, Y = codes(9, D, 2), out(9, V, F, 0)
    head.logits(Xq, torch.ones(9, device=DEV), Y)
    want = sums(Xq, head.Wq) * scale.double()
    assert ((Y.double() - want).abs() <= 4 * U * want.abs() + 1e-37).all()


def test_largest_sums_do_not_overflow(em):
    D = 32768
    Xq = torch.full((20, D), -128, dtype=torch.int8, device=DEV)
    Wq = torch.full((70, D), -128, dtype=torch.int8, device=DEV)
    Wq[1] = 127
    for T in (1, 20):
        Y = out(T, 70, F, 0)
        em.ember_logits_q8(Xq[:T], torch.ones(T, device=DEV), Wq, torch.ones(70, device=DEV), Y)
        assert (Y[:, 0] == 2.0 ** 14 * D).all() and (Y[:, 1] == -128.0 * 127 * D).all()


def test_scales_that_are_not_finite(em):
    """A token whose scale is NaN (its hidden state was not finite) has NaN logits, the others none."""
    for T in (5, 130):
        Xq, Wq = codes(T, 200, 3), codes(333, 200, 4)
        xs, ws = torch.ones(T, device=DEV), torch.ones(333, device=DEV)
        xs[2] = float("nan")
        ws[7] = float("inf")
        Y = out(T, 333, F, 0)
        em.ember_logits_q8(Xq, xs, Wq, ws, Y)
        assert torch.isnan(Y[2]).all()
        rest = [t for t in range(T) if t != 2]
        cols = [v for v in range(333) if v != 7]
        assert torch.equal(Y[rest][:, cols], sums(Xq, Wq).float()[rest][:, cols])
        assert not torch.isfinite(Y[rest][:, 7]).any()


def test_offsets_past_32_bits(em):
    """A table of 2.3 GB of codes, and logits past 2^31 bytes: the last rows are where the offsets say."""
    V, D = 70000, 32768
    print("logits of a 2.3 GB table", flush=True)
    Wq = torch.zeros(V, D, dtype=torch.int8, device=DEV)
    Wq[V - 200:] = codes(200, D, 8, 0)
    for T in (3, 40):
        Xq = codes(T, D, 9, 0)
        Y = out(T, V, F, 0)
        em.ember_logits_q8(Xq, torch.ones(T, device=DEV), Wq, torch.ones(V, device=DEV), Y)
        assert torch.equal(Y[:, V - 200:], sums(Xq, Wq[V - 200:]).float()) and (Y[:, :V - 200] == 0).all()
    del Wq, Y
    T, V, D = 9000, 70000, 32
    print("logits of 2.5 GB", flush=True)
    Xq, Wq = codes(T, D, 5), codes(V, D, 6)
    Y = out(T, V, F, 0)
    em.ember_logits_q8(Xq, torch.ones(T, device=DEV), Wq, torch.ones(V, device=DEV), Y)
    for at in (slice(0, 10), slice(T - 300, T)):
        assert torch.equal(Y[at], sums(Xq[at], Wq).float())


def test_wide_strides(em):
    """Rows of a few codes at the largest stride: what counts is the row's own offset."""
    ld = (1 << 22) - 16
    n = 600      # 2.5 GB from the first row to the last
    buf = torch.zeros(n * ld, dtype=torch.int8, device=DEV)
    Wq = buf.as_strided((n, 48), (ld, 1))
    Wq.copy_(codes(n, 48, 1))
    for T in (1, 20, 70, 300):
        print(f"logits wide strides T={T}", flush=True)
        Xq = codes(T, 48, T)
        Y = out(T, n, F, 0)
        em.ember_logits_q8(Xq, torch.ones(T, device=DEV), Wq, torch.ones(n, device=DEV), Y)
        assert torch.equal(Y, sums(Xq, Wq).float()), T
        # and the other way round: the tokens far apart
        Z = out(n, T, F, 0)
        em.ember_logits_q8(Wq, torch.ones(n, device=DEV), Xq, torch.ones(T, device=DEV), Z)
        assert torch.equal(Z, sums(Wq, Xq).float()), T


def test_no_tokens(em):
    Wq = codes(10, 32, 1, 0)
    em.ember_logits_q8(Wq[:0], torch.empty(0, device=DEV), Wq, torch.ones(10, device=DEV), torch.empty(0, 10, device=DEV))


def test_on_another_stream_and_in_a_graph(em):
    for T in (2, 90):
        Xq, Wq = codes(T, 300, 3), codes(777, 300, 4)
        xs, ws = torch.rand(T, device=DEV), torch.rand(777, device=DEV)
        Y = out(T, 777, BF, 0)
        em.ember_logits_q8(Xq, xs, Wq, ws, Y)
        want = Y.clone()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            Y.zero_()
            em.ember_logits_q8(Xq, xs, Wq, ws, Y)
        side.synchronize()
        assert torch.equal(Y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            em.ember_logits_q8(Xq, xs, Wq, ws, Y)
        for k in range(3):
            xs.copy_(torch.rand(T, device=DEV))
            em.ember_logits_q8(Xq, xs, Wq, ws, Y)
            want = Y.clone()
            Y.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(Y, want), (T, k)


@pytest.mark.parametrize("V", [1, 2, 5, 15, 16, 17])
@pytest.mark.parametrize("T,D", [(1, 2500), (16, 4096), (17, 2064), (32, 4000), (33, 1100), (64, 2048), (3, 100)])
def test_tables_shorter_than_a_strip(em, T, V, D):
    """Fewer channels than a streaming round takes, with rounds past the table: columns in
    two parts, of which the second one's loads end with the table too."""
    print(f"logits T={T} V={V} D={D}", flush=True)
    Xq, Wq = codes(T, D, T + D, 0, -128), codes(V, D, V + D, 0, -128)
    Y = out(T, V, F)
    em.ember_logits_q8(Xq, torch.ones(T, device=DEV), Wq, torch.ones(V, device=DEV), Y)
    assert torch.equal(Y, sums(Xq, Wq).float())
    assert torch.isnan(Y._base[:, V:]).all()
