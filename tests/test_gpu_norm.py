"""The final norm (ember_rmsnorm), its 8-bit output, its gradient and
ember_quantize_rows, through the C ABI, against the formulas in float64.

Bars, with u = 2^-24 (half an ulp of fp32 at 1):
* S is one fp32 addition, rounded once more to its type: the same bits as torch's.
* rstd: the mean is a sum of squares (all positive), added per thread (at most
  64 terms), over a wave (6 levels) and over at most 16 waves, each addition and
  square off by at most u of the result: 64 + 6 + 16 + 1 roundings, halved by the
  root, and the sum's own rounding (2 u in s^2), the division, the addition of eps
  and the root: below 64 u.
* y: rstd's error, the rounding of s, two products: below 68 u |y|; rounded to bf16
  at most 2^-8 |y| more.
* codes: |q - y 127 / a| <= 1/2 + 127 (2 * 68 u + 3 u); the scale within 70 u.
* dx: with A = |rstd dy g| + |rstd^3 s| mean|dy g s| + |ds| its terms are off by at
  most the roundings of the mean (90 u as above) and ten of single operations:
  100 u A, plus the rounding to its type.
* dgain: T terms of three roundings each, added in some order: (T + 3) u sum|terms|.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
EPS = 1e-6
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def em():
    from paper_2607_01455_amd import ember
    return ember


def padded(rows, D, dtype, extra=0):
    """rows x D view whose rows start on 16-byte boundaries, NaN (or code 77) behind them."""
    q = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = ((D + q - 1) // q + extra) * q
    full = torch.full((max(rows, 1), ld), float("nan") if dtype.is_floating_point else 77, dtype=dtype, device=DEV)
    return full[:rows, :D]


def padding_kept(t):
    """The columns behind a padded() view still hold what it put there."""
    pad = t._base[:, t.shape[1]:]
    return bool((torch.isnan(pad.float()) if t.dtype.is_floating_point else pad == 77).all())


def bits(t):
    return t.contiguous().view({2: torch.int16, 4: torch.int32}[t.element_size()])


def store_err(E, dtype):
    return E.abs() * (2.0 ** -8 if dtype == BF else 0.0) + 1e-37


def make(T, D, dtype, seed, residual, extra=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    X = padded(T, D, dtype, extra)
    X.copy_(torch.randn(T, D, generator=g, device=DEV))
    R = None
    if residual:
        R = padded(T, D, dtype, extra + 1)
        R.copy_(3 * torch.randn(T, D, generator=g, device=DEV))
    return X, R, g


def forward64(X, R, gain):
    s = X.double() + (R.double() if R is not None else 0.0)
    rstd = (s.square().mean(dim=1) + EPS).rsqrt()
    return s, rstd, s * rstd[:, None] * gain.double()


def check_codes(Q, qscale, y):
    a = y.abs().amax(dim=1)
    off = (Q.double() - y * (127.0 / a)[:, None]).abs().max().item()
    assert off <= 0.5 + 127 * 139 * U, off
    assert ((qscale.double() - a / 127).abs() <= 70 * U * a / 127).all()
    assert (Q.int().abs().amax(dim=1) == 127).all()


SHAPES = [(1, 1), (3, 7), (5, 8), (2, 64), (130, 200), (4, 512), (9, 513), (33, 1023), (5, 2000), (4, 2048), (6, 2049), (17, 4096), (3, 8192),
          (2, 8200), (2, 16385), (3, 32768)]


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("dtype,ydtype,gdtype,residual", [(BF, BF, F, True), (F, F, F, False), (F, BF, BF, True),
                                                         (BF, F, BF, False)])
def test_forward(em, T, D, dtype, ydtype, gdtype, residual):
    print(f"rmsnorm T={T} D={D} {dtype} {ydtype} gain {gdtype} residual={residual}", flush=True)
    X, R, g = make(T, D, dtype, T * 131 + D, residual)
    gain = (0.5 + torch.rand(D, generator=g, device=DEV)).to(gdtype)
    S = padded(T, D, dtype, 2) if residual else None
    Y, Q = padded(T, D, ydtype, 1), padded(T, D, torch.int8, 1)
    qscale, rstd = torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    em.ember_rmsnorm(X, gain, EPS, R, S, Y, Q, qscale, rstd)
    s, rs, y = forward64(X, R, gain)
    if residual:
        assert torch.equal(bits(S), bits((X.float() + R.float()).to(dtype)))
        assert padding_kept(S)
    assert ((rstd.double() - rs).abs() <= 64 * U * rs).all()
    assert ((Y.double() - y).abs() <= 68 * U * y.abs() + store_err(y, ydtype)).all()
    check_codes(Q, qscale, y)
    assert padding_kept(Y) and padding_kept(Q)
    # each output alone gives the same bits
    Y2, Q2, q2 = padded(T, D, ydtype, 1), padded(T, D, torch.int8, 1), torch.zeros(T, device=DEV)
    em.ember_rmsnorm(X, gain, EPS, R, Y=Y2)
    em.ember_rmsnorm(X, gain, EPS, R, Q=Q2, qscale=q2)
    assert torch.equal(bits(Y2), bits(Y)) and torch.equal(Q2, Q) and torch.equal(q2, qscale)


@pytest.mark.parametrize("T", [1, 63, 300, 2000, 5000])
@pytest.mark.parametrize("D,dtype", [(96, BF), (896, F), (1000, BF), (4096, BF), (699, BF), (1001, F), (2047, BF), (3001, F)])
def test_forward_over_token_counts(em, T, D, dtype):
    print(f"rmsnorm T={T} D={D} {dtype}", flush=True)
    X, R, g = make(T, D, dtype, T + D, True, extra=0)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    S, Y = padded(T, D, dtype), padded(T, D, dtype)
    Q, qscale, rstd = padded(T, D, torch.int8), torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    em.ember_rmsnorm(X, gain, EPS, R, S, Y, Q, qscale, rstd)
    s, rs, y = forward64(X, R, gain)
    assert torch.equal(bits(S), bits((X.float() + R.float()).to(dtype)))
    assert ((rstd.double() - rs).abs() <= 64 * U * rs).all()
    assert ((Y.double() - y).abs() <= 68 * U * y.abs() + store_err(y, dtype)).all()
    check_codes(Q, qscale, y)


def test_outputs_past_what_is_streamed(em):
    """147 MB of Y and as much of dX: these are not stored non-temporally."""
    T, D = 9000, 8192
    print("rmsnorm 9000 x 8192", flush=True)
    X, R, g = make(T, D, BF, 3, True, extra=0)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    norm = em.HeadNorm(gain, EPS, max_tokens=T)
    S, Y, dX, rstd, dgain = padded(T, D, BF), padded(T, D, BF), padded(T, D, BF), torch.zeros(T, device=DEV), torch.zeros(D, device=DEV)
    norm(X, R, S, Y, rstd=rstd)
    norm.grad(R, S, rstd, dX, dgain)
    total = torch.zeros(D, dtype=torch.float64, device=DEV)
    mag = torch.zeros(D, dtype=torch.float64, device=DEV)
    for t0 in range(0, T, 3000):
        at = slice(t0, t0 + 3000)
        s, rs, y = forward64(X[at], R[at], gain)
        assert torch.equal(bits(S[at]), bits((X[at].float() + R[at].float()).to(BF)))
        assert ((Y[at].double() - y).abs() <= 68 * U * y.abs() + store_err(y, BF)).all()
        dx, A, dg, m = grad64(R[at], S[at], gain, rstd[at], None)
        assert ((dX[at].double() - dx).abs() <= 100 * U * A + store_err(dx, BF)).all()
        total, mag = total + dg, mag + m
    assert ((dgain.double() - total).abs() <= (T + 3) * U * mag).all()


def test_outputs_in_place(em):
    """S in the place of the residual stream or of X, Y in the place of X."""
    for D in (1000, 8192, 20000):
        print(f"rmsnorm in place D={D}", flush=True)
        X, R, g = make(9, D, BF, D, True, extra=0)
        R = padded(9, D, BF).copy_(R)
        gain = 0.5 + torch.rand(D, generator=g, device=DEV)
        S, Y = padded(9, D, BF), padded(9, D, BF)
        em.ember_rmsnorm(X, gain, EPS, R, S, Y)
        X2, R2, X3, R3 = (padded(9, D, BF).copy_(t) for t in (X, R, X, R))
        em.ember_rmsnorm(X2, gain, EPS, R2, S=R2, Y=X2)
        assert torch.equal(bits(R2), bits(S)) and torch.equal(bits(X2), bits(Y))
        Y3 = padded(9, D, BF)
        em.ember_rmsnorm(X3, gain, EPS, R3, S=X3, Y=Y3)
        assert torch.equal(bits(X3), bits(S)) and torch.equal(bits(Y3), bits(Y))


@pytest.mark.parametrize("D", [40, 1023, 5000])
def test_rows_of_zeros_tiny_and_not_finite(em, D):
    print(f"rmsnorm special rows D={D}", flush=True)
    X = torch.randn(8, (D + 7) // 8 * 8, device=DEV)[:, :D]
    X[1] = 0.0
    X[2] = 0.0
    X[2, D - 1] = 1e-30
    X[3, 0] = float("nan")
    X[4, D - 1] = float("inf")
    X[5] *= 1e15
    gain = torch.ones(D, device=DEV)
    Y, Q, qs, rstd = padded(8, D, F), padded(8, D, torch.int8), torch.zeros(8, device=DEV), torch.zeros(8, device=DEV)
    em.ember_rmsnorm(X, gain, EPS, Y=Y, Q=Q, qscale=qs, rstd=rstd)
    y = forward64(X, None, gain)[2]
    for row in (0, 5, 6, 7):
        check_codes(Q[row:row + 1], qs[row:row + 1], y[row:row + 1])
        assert ((Y[row].double() - y[row]).abs() <= 68 * U * y[row].abs()).all()
    assert (Y[1] == 0).all() and (Q[1] == 0).all() and qs[1] == 0
    check_codes(Q[2:3], qs[2:3], y[2:3])
    assert torch.isnan(Y[3]).all() and torch.isnan(qs[3]) and (Q[3] == 0).all()
    # an infinity: rstd 0, its own product NaN, the row's others 0, as the formula has them
    assert rstd[4] == 0 and torch.isnan(Y[4, D - 1]) and (Y[4, :D - 1] == 0).all()
    assert torch.isnan(qs[4]) and (Q[4] == 0).all()


@pytest.mark.parametrize("rows,D,dtype", [(1, 1, F), (5, 16, BF), (700, 1000, BF), (300, 4096, F), (3, 32768, BF),
                                          (9, 333, F)])
def test_quantize_rows(em, rows, D, dtype):
    print(f"quantize rows={rows} D={D} {dtype}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(rows + D)
    W = padded(rows, D, dtype, 1)
    W.copy_(0.02 * torch.randn(rows, D, generator=g, device=DEV))
    Q, qs = padded(rows, D, torch.int8, 1), torch.zeros(rows, device=DEV)
    em.ember_quantize_rows(W, Q, qs)
    check_codes(Q, qs, W.double())
    assert padding_kept(Q)
    if rows > 4:
        W[1] = 0
        W[2] = 1e-37 if dtype == F else 0
        W[3, D - 1] = float("-inf")
        em.ember_quantize_rows(W, Q, qs)
        assert (Q[1:4] == 0).all() and (qs[1:3] == 0).all() and torch.isnan(qs[3])


def grad64(dY, S, gain, rstd, dS):
    s, dy, r = S.double(), dY.double(), rstd.double()[:, None]
    u = dy * gain.double()
    dx = r * u - r ** 3 * (u * s).mean(dim=1, keepdim=True) * s
    A = (r * u).abs() + (r ** 3 * s).abs() * (u * s).abs().mean(dim=1, keepdim=True)
    if dS is not None:
        dx, A = dx + dS.double(), A + dS.double().abs()
    terms = dy * s * r
    return dx, A, terms.sum(dim=0), terms.abs().sum(dim=0)


@pytest.mark.parametrize("T,D", SHAPES + [(300, 896), (1500, 72), (2500, 1000), (1100, 4096),
                                          # one block, and a few
                                          (64, 512), (65, 512), (16, 2048), (17, 2048), (8, 4096), (9, 4096), (4, 8192),
                                          (5, 8192), (4, 32768), (5, 32768),
                                          # rows that end inside a chunk, many
                                          (5000, 700), (2000, 2047), (700, 3001), (1500, 300), (5000, 513),
                                          # dgain in the same launch, and the first counts without
                                          (512, 300), (513, 300), (100, 96), (512, 1000), (300, 2047), (512, 4096), (513, 4096),
                                          (200, 8192), (512, 9000), (70, 20000)])
@pytest.mark.parametrize("dtype,gdtype,other", [(BF, F, True), (F, BF, False)])
def test_gradient(em, T, D, dtype, gdtype, other):
    print(f"rmsnorm grad T={T} D={D} {dtype} gain {gdtype} dS={other}", flush=True)
    X, _, g = make(T, D, dtype, T * 7 + D, False)
    gain = (0.5 + torch.rand(D, generator=g, device=DEV)).to(gdtype)
    norm = em.HeadNorm(gain, EPS, max_tokens=T)
    rstd = torch.zeros(T, device=DEV)
    norm(X, Y=padded(T, D, dtype), rstd=rstd)
    dY, dX = padded(T, D, dtype, 2), padded(T, D, dtype, 1)
    dY.copy_(torch.randn(T, D, generator=g, device=DEV))
    dS = padded(T, D, dtype).copy_(torch.randn(T, D, generator=g, device=DEV)) if other else None
    dgain = torch.full((D,), float("nan"), device=DEV)
    norm.grad(dY, X, rstd, dX, dgain, dS=dS)
    dx, A, dg, mag = grad64(dY, X, gain, rstd, dS)
    assert ((dX.double() - dx).abs() <= 100 * U * A + store_err(dx, dtype)).all()
    assert ((dgain.double() - dg).abs() <= (T + 3) * U * mag + 1e-37).all()
    assert padding_kept(dX)
    # in the place of dY, twice with the same bits
    dgain2 = torch.zeros(D, device=DEV)
    dY2 = padded(T, D, dtype).copy_(dY)
    norm.grad(dY2, X, rstd, dY2, dgain2, dS=dS)
    assert torch.equal(bits(dY2), bits(dX)) and torch.equal(bits(dgain2), bits(dgain))


def test_gradient_against_differences(em):
    """Central differences of L = sum(dY y) + sum(dS s) in float64 at D = 65: with
    steps of 1e-5 their own error is below 1e-8 of the gradient's scale, and the
    fp32 gradient's below 100 u times its terms."""
    T, D, h = 4, 65, 1e-5
    X, _, g = make(T, D, F, 5, False)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    dY, dS = torch.randn(T, 68, generator=g, device=DEV)[:, :D], torch.randn(T, 68, generator=g, device=DEV)[:, :D]
    norm = em.HeadNorm(gain, EPS, max_tokens=T)
    rstd, dX, dgain = torch.zeros(T, device=DEV), padded(T, D, F), torch.zeros(D, device=DEV)
    norm(X, Y=padded(T, D, F), rstd=rstd)
    norm.grad(dY, X, rstd, dX, dgain, dS=dS)

    def loss(x, gn):
        y = x * (x.square().mean(dim=1, keepdim=True) + EPS).rsqrt() * gn
        return (dY.double() * y + dS.double() * x).sum()

    x, gn = X.double().clone(), gain.double().clone()
    for t in range(T):
        for j in (0, 1, 31, 63, 64):
            d = torch.zeros_like(x)
            d[t, j] = h
            want = (loss(x + d, gn) - loss(x - d, gn)) / (2 * h)
            assert abs(dX[t, j].item() - want.item()) <= 1e-4
    for j in (0, 17, 64):
        d = torch.zeros_like(gn)
        d[j] = h
        want = (loss(x, gn + d) - loss(x, gn - d)) / (2 * h)
        assert abs(dgain[j].item() - want.item()) <= 1e-4


def test_no_tokens(em):
    D = 48
    norm = em.HeadNorm(torch.ones(D, device=DEV), EPS, max_tokens=0)
    X = torch.empty(0, D, device=DEV)
    norm(X, Y=torch.empty(0, D, device=DEV), rstd=torch.empty(0, device=DEV))
    dgain = torch.ones(D, device=DEV)
    norm.grad(X, X, torch.empty(0, device=DEV), X, dgain)
    assert (dgain == 0).all()
    em.ember_quantize_rows(X, torch.empty(0, D, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV))


def test_on_another_stream_and_in_a_graph(em):
    """The calls run on the current stream; captured, every replay gives the eager bits."""
    T, D = 70, 1000
    X, R, g = make(T, D, BF, 11, True)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    norm = em.HeadNorm(gain, EPS, max_tokens=T)
    S, Y, Q = padded(T, D, BF), padded(T, D, BF), padded(T, D, torch.int8)
    qs, rstd, dgain = torch.zeros(T, device=DEV), torch.zeros(T, device=DEV), torch.zeros(D, device=DEV)
    dX = padded(T, D, BF)
    outs = (S, Y, Q, qs, rstd, dX, dgain)

    def both():
        norm(X, R, S, Y, Q, qs, rstd)
        norm.grad(Y, S, rstd, dX, dgain, dS=R)

    def same(want):
        return all(torch.equal(a, b) for a, b in zip(want, outs))

    both()
    want = [t.clone() for t in outs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in outs:
            t.zero_()
        both()
    side.synchronize()
    assert same(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        X.copy_(torch.randn(T, D, generator=g, device=DEV))
        both()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(want), k


def rows_of_range(T, D, dtype, tiny, g):
    """Rows of magnitudes whose squares, or their sums, leave the fp32 range: above it
    (among them single large values, and numbers next to the largest), or below it."""
    X = padded(T, D, dtype, 1)
    x = torch.randn(T, D, generator=g, device=DEV)
    sizes = [1.0, 1e-20, 1e-24, 1e-30, 1e-36] if tiny else [1.0, 1e18, 2e19, 1e30, 1e37]
    for t in range(T):
        k = t % 7
        if k < 5:
            x[t] *= sizes[k]
        elif k == 5:     # one value apart from the others
            x[t, t % D] = 1e-24 if tiny else 3e19
            if tiny:
                x[t, torch.arange(D, device=DEV) != t % D] = 0.0
        elif not tiny:
            x[t] = (2 * torch.rand(D, generator=g, device=DEV) - 1) * 3e38
        else:
            x[t] *= 1e-15
    return X.copy_(x)


def range_forward(em, T, D, dtype, tiny, eps):
    g = torch.Generator(device=DEV).manual_seed(T + D)
    X = rows_of_range(T, D, dtype, tiny, g)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    norm = em.HeadNorm(gain, eps, max_tokens=T)
    Y, Q, qs, rstd = padded(T, D, F), padded(T, D, torch.int8), torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    norm(X, Y=Y, Q=Q, qscale=qs, rstd=rstd)
    return norm, g, X, gain, Y, Q, qs, rstd


RANGES = [(False, EPS), (False, 0.0), (False, 1e38), (True, 0.0), (True, 1e-44)]
RANGE_SHAPES = [(14, 40), (7, 1023), (9, 2048), (600, 300), (21, 5000), (7, 8192), (8, 20000), (7, 32768)]


@pytest.mark.parametrize("tiny,eps", RANGES)
@pytest.mark.parametrize("T,D", RANGE_SHAPES)
@pytest.mark.parametrize("dtype", [BF, F])
def test_squares_past_the_range_of_fp32(em, T, D, dtype, tiny, eps):
    """A row's mean square, and so everything made of it, is right wherever rstd itself
    is an fp32 number (below 2^-126 it is held to 2^-150)."""
    print(f"rmsnorm range T={T} D={D} {dtype} tiny={tiny} eps={eps}", flush=True)
    _, _, X, gain, Y, Q, qs, rstd = range_forward(em, T, D, dtype, tiny, eps)
    s = X.double()
    rs = (s.square().mean(dim=1) + torch.tensor(eps, dtype=F).double().item()).rsqrt()
    y = s * rs[:, None] * gain.double()
    assert ((rstd.double() - rs).abs() <= 64 * U * rs + 2.0 ** -150).all()
    # (2^-150 is at most 4 u of an rstd above 2.9e-39)
    assert ((Y.double() - y).abs() <= 72 * U * y.abs() + 1e-37).all()
    normal = y.abs().amax(dim=1) > 1e-30
    assert normal.any()
    check_codes(Q[normal], qs[normal], y[normal])


@pytest.mark.parametrize("tiny,eps", RANGES)
@pytest.mark.parametrize("T,D", RANGE_SHAPES)
@pytest.mark.parametrize("dtype", [BF, F])
def test_gradient_past_the_range_of_fp32(em, T, D, dtype, tiny, eps):
    """Rows whose squares leave the fp32 range have a gradient like others."""
    print(f"rmsnorm grad range T={T} D={D} {dtype} tiny={tiny} eps={eps}", flush=True)
    norm, g, X, gain, _, _, _, rstd = range_forward(em, T, D, dtype, tiny, eps)
    dY, dX = padded(T, D, dtype, 2), padded(T, D, dtype)
    dY.copy_(torch.randn(T, D, generator=g, device=DEV))
    dgain, dgain2 = torch.zeros(D, device=DEV), torch.zeros(D, device=DEV)
    norm.grad(dY, X, rstd, dX, dgain)
    dx, A, dg, mag = grad64(dY, X, gain, rstd, None)
    inside = dx.abs() < 1e37      # of tiny rows; beyond lies the end of the range
    assert inside.any()
    # what is below 2^-126 is held to 2^-149 (bf16: 2^-134, after a rounding of 2^-150)
    bar = 100 * U * A + (2.0 ** -8 * dx.abs() + 2.0 ** -133 if dtype == BF else 2.0 ** -148)
    assert ((dX.double() - dx).abs() <= bar)[inside].all()
    assert ((dgain.double() - dg).abs() <= (T + 3) * U * mag + 1e-37).all()
    norm.grad(dY, X, rstd, dY, dgain2)
    assert torch.equal(bits(dY), bits(dX)) and torch.equal(bits(dgain2), bits(dgain))


@pytest.mark.parametrize("T,D", [(1, 96), (40, 96), (40, 100), (600, 101), (9, 5000)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_columns_of_one_buffer(em, T, D, dtype):
    """Inputs and outputs side by side in one buffer's rows: the bits of separate tensors, and
    nothing between them is written."""
    print(f"rmsnorm columns of one buffer T={T} D={D} {dtype}", flush=True)
    W = (D + 7) // 8 * 8 + 8
    big = torch.full((T, 6 * W), float("nan"), dtype=dtype, device=DEV)
    x, r, s, y, dx, ds = (big[:, k * W:k * W + D] for k in (3, 0, 5, 1, 4, 2))
    X, R, g = make(T, D, dtype, T + D, True)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    x.copy_(X), r.copy_(R), ds.copy_(R)
    norm = em.HeadNorm(gain, EPS, max_tokens=T)
    S, Y, dX = padded(T, D, dtype), padded(T, D, dtype), padded(T, D, dtype)
    rstd, dgain = torch.zeros(T, device=DEV), torch.zeros(D, device=DEV)
    rstd2, dgain2 = torch.zeros(T, device=DEV), torch.zeros(D, device=DEV)
    norm(X, R, S, Y, rstd=rstd)
    norm.grad(Y, S, rstd, dX, dgain, dS=R)
    norm(x, r, s, y, rstd=rstd2)
    norm.grad(y, s, rstd2, dx, dgain2, dS=ds)
    for a, b in ((s, S), (y, Y), (dx, dX), (rstd2, rstd), (dgain2, dgain), (x, X), (r, R)):
        assert torch.equal(bits(a), bits(b))
    for k in range(6):
        assert torch.isnan(big[:, k * W + D:(k + 1) * W].float()).all()
    if T > 1:    # S over the last columns of Y, and over X but its first chunk
        for start in (W + (D - 1) // 8 * 8, 3 * W + 8):
            with pytest.raises(em.EmberError) as e:
                norm(x, r, S=big[:, start:start + D], Y=y)
            assert e.value.status == em.EMBER_ERR_ARG


@pytest.mark.parametrize("T,D,dtype", [(16384, 4096, BF), (16385, 4096, BF), (16392, 2047, F), (16393, 2047, F)])
def test_gradient_where_its_stores_change(em, T, D, dtype):
    """dX of 128 MiB, the most that is stored ordinarily, and of a row more, stored non-temporally."""
    print(f"rmsnorm grad T={T} D={D} {dtype}", flush=True)
    X, _, g = make(T, D, dtype, T, False, extra=0)
    gain = 0.5 + torch.rand(D, generator=g, device=DEV)
    dY, dX = padded(T, D, dtype), padded(T, D, dtype)
    dY.copy_(torch.randn(T, D, generator=g, device=DEV))
    norm = em.HeadNorm(gain, EPS, max_tokens=T)
    rstd, dgain = (X.float().square().mean(dim=1) + EPS).rsqrt(), torch.zeros(D, device=DEV)
    norm.grad(dY, X, rstd, dX, dgain, dS=X)
    total, mag = torch.zeros(D, dtype=torch.float64, device=DEV), torch.zeros(D, dtype=torch.float64, device=DEV)
    for t0 in range(0, T, 5000):
        at = slice(t0, t0 + 5000)
        dx, A, dg, m = grad64(dY[at], X[at], gain, rstd[at], X[at])
        assert ((dX[at].double() - dx).abs() <= 100 * U * A + store_err(dx, dtype)).all()
        total, mag = total + dg, mag + m
    assert ((dgain.double() - total).abs() <= (T + 3) * U * mag).all()
    assert padding_kept(dX)
