"""Tokens drawn from logits (ember_sample), through the C ABI, against float64.

Ids and counts are equal: what is summed is 2^-z in fixed point, off by at most half of
2^-n a token (n = min(48, 62 - ceil(log2 V)), 2^-45 at V = 128256), the largest being 1,
and float64's own sums are off by less, so a border is met differently only where a
running sum comes within about V 2^-n of it, of sums of 1 and more.
logp = ln e - ln sum e: each of V terms of the sum is off by 2^-(n+1) at most and the sum is
1 at least, so its logarithm is off by V 2^-(n+1) (2^-29 at V = 128256, 2^-15 at 2^24), and
the result is rounded to fp32 once (2^-24 relative)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F = torch.bfloat16, torch.float32
INF = math.inf


@pytest.fixture(scope="module")
def em():
    from paper_2607_01455_amd import ember
    return ember


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def logits(T, V, dtype, extra=1):
    q = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.full((T, ((V + q - 1) // q + extra) * q), float("nan"), dtype=dtype, device=DEV)[:, :V]


def vec(x, dtype=F):
    return None if x is None else torch.as_tensor(x, dtype=dtype, device=DEV).contiguous()


def one_row(l, u, temperature=1.0, k=0, p=1.0, floor=0.0):
    """id, log-probability, tokens kept, from the definition, in float64 on the host."""
    l = l.double().cpu()
    if torch.isnan(l).any() or (l == INF).any() or not (l > -INF).any():
        return -1, math.nan, 0
    if temperature == 0:
        temperature, k = 1.0, 1
    e = torch.exp((l - l.max()) / temperature)
    order = torch.argsort(l, descending=True, stable=True)[:int((l > -INF).sum())]
    if k:
        order = order[:k]
    w = e[order]
    n = len(order)
    if p < 1:
        before = torch.cumsum(w, 0) - w
        n = max(1, int((before < p * w.sum()).sum()))
    n = max(1, min(n, int((w >= floor).sum())))
    kept = torch.sort(order[:n]).values
    run = torch.cumsum(e[kept], 0)
    i = int(kept[int((run <= u * run[-1]).sum())])
    return i, float((l[i] - l.max()) / temperature - torch.log(e.sum())), n


def draw(em, L, u, temperature=None, k=None, p=None, floor=None, ws=None):
    T, V = L.shape
    ids = torch.full((T,), -7, dtype=torch.int64, device=DEV)
    logp, kept = torch.full((T,), 7.0, device=DEV), torch.full((T,), -7, dtype=torch.int32, device=DEV)
    s = em.Sampler(T, V)
    s.ws.fill_(0xA5)                       # it needs no initialisation
    s(L, u, ids, temperature=temperature, top_k=k, top_p=p, min_p=floor, logp=logp, kept=kept)
    return ids, logp, kept


def check(em, L, u, temperature=None, k=None, p=None, floor=None):
    args = [vec(temperature), vec(k, torch.int32), vec(p), vec(floor)]
    got = [x.cpu() for x in draw(em, L, u, *args)]
    ask = [None if a is None else a.cpu() for a in args]
    for t in range(L.shape[0]):
        v = [a[t].item() if a is not None else d for a, d in zip(ask, (1.0, 0, 1.0, 0.0))]
        i, lp, n = one_row(L[t], u[t].double().item(), *v)
        what = f"row {t}, temperature {v[0]}, k {v[1]}, p {v[2]}, min-p {v[3]}, u {u[t].item()}"
        assert (got[0][t].item(), got[2][t].item()) == (i, n), what
        if i < 0:
            assert math.isnan(got[1][t].item()), what
        else:
            bits = min(48, 62 - (L.shape[1] - 1).bit_length())
            bar = 2.0 ** -24 * abs(lp) + L.shape[1] * 2.0 ** -(bits + 1) + 2.0 ** -40      # 2^-40: fp64's own
            assert abs(got[1][t].item() - lp) <= bar, what
    return got


def zipf(T, V, dtype, seed, power=None):
    """Rows whose probabilities fall with a power of the rank."""
    g = gen(seed)
    L = logits(T, V, dtype)
    a = 0.6 + 1.2 * torch.rand(T, 1, generator=g, device=DEV) if power is None else power
    L.copy_(-torch.log1p(-torch.rand(T, V, generator=g, device=DEV)) * a - 5)
    return L, torch.rand(T, generator=g, device=DEV)


SIZES = [1, 2, 7, 64, 511, 512, 513, 1000, 4096, 8191, 20000, 50257, 128256]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("dtype", [BF, F])
def test_no_filter(em, V, dtype):
    print(f"sample V={V} {dtype}", flush=True)
    L, u = zipf(9, V, dtype, V)
    check(em, L, u)
    check(em, L, u, temperature=[0.0, 0.01, 0.3, 0.7, 1.0, 1.5, 10.0, 1e4, 1e-30])


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("dtype", [BF, F])
def test_each_filter(em, V, dtype):
    print(f"sample filters V={V} {dtype}", flush=True)
    T = 10
    L, u = zipf(T, V, dtype, V + 1)
    check(em, L, u, k=[0, 1, 2, 3, 10, 50, 200, 1000, 100000, 2 ** 31 - 1])
    check(em, L, u, p=[0.0, 0.01, 0.3, 0.5, 0.8, 0.9, 0.95, 0.99, 0.999, 1.0])
    check(em, L, u, floor=[0.0, 1e-30, 1e-10, 1e-5, 1e-3, 0.01, 0.05, 0.1, 0.5, 1.0])


@pytest.mark.parametrize("V", [5, 700, 8192, 32000, 128256, 262144])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("masked", [False, True])
def test_filters_together(em, V, dtype, masked):
    print(f"sample all filters V={V} {dtype} masked={masked}", flush=True)
    T, g = 24, gen(V)
    L, u = zipf(T, V, dtype, V + 2)
    if masked:
        L[torch.rand(T, V, generator=g, device=DEV) < 0.6] = -INF
        L[3] = -INF                         # nothing allowed
        L[5] = -INF
        L[5, V - 1] = -2.0                  # one token allowed
    r = [torch.rand(T, generator=g, device=DEV) for _ in range(4)]
    temperature = 0.2 + 1.5 * r[0]
    temperature[::7] = 0
    k = torch.where(r[1] < 0.4, 0, (10 ** (3 * r[1])).int())
    p = torch.where(r[2] < 0.3, 1.0, 0.6 + 0.4 * r[2])
    floor = torch.where(r[3] < 0.5, 0.0, 0.2 * (r[3] - 0.5))
    check(em, L, u, temperature, k, p, floor)
    check(em, L, u, temperature, None, p, None)
    check(em, L, u, None, k, p, None)


@pytest.mark.parametrize("V", [3, 1000, 8192, 8193, 20000, 128256])
@pytest.mark.parametrize("dtype", [BF, F])
def test_equal_logits(em, V, dtype):
    """Prefixes that end among equal logits: the first by index are kept.  More of them than a list holds."""
    print(f"sample equal V={V} {dtype}", flush=True)
    T = 8
    u = torch.tensor([0, 0.1, 0.25, 0.5, 0.75, 0.9, 0.999, 1 - 2.0 ** -24], device=DEV)
    L = logits(T, V, dtype)
    L.fill_(2.5)
    got = check(em, L, u, k=[1, 2, V // 3, V // 2 + 1, V - 1, V, 0, 300])
    check(em, L, u)
    check(em, L, u, p=[0.0, 2.0 ** -10, 0.125, 0.25, 0.5, 0.75, 1 - 2.0 ** -10, 1.0])
    check(em, L, u, k=[V // 2 + 1] * 8, p=[0.5] * 8, floor=[1.0] * 8)
    # two levels, spread over the row; the lower one ends the prefix
    L[:, ::3] = 1.25
    check(em, L, u, k=[V // 3, V // 2, V - 2, V - 1, 1, 0, V // 3 + 2, 2 * V // 3 + 2])
    check(em, L, u, temperature=[0.5] * 8, p=[0.9, 0.95, 0.97, 0.99, 0.5, 0.1, 1.0, 0.98], k=[0, 0, 0, 0, V - 1, 0, V - 1, V - 1])


def test_values_at_the_ends(em):
    """The type's lowest values as masks, all of them lowest, both zeros, huge spans."""
    for dtype in (BF, F):
        low, top = torch.finfo(dtype).min, torch.finfo(dtype).max
        V = 3000
        L, u = zipf(9, V, dtype, 3)
        L[0] = low
        L[1, 1:] = low
        L[2, ::2] = low
        L[3] = 0.0
        L[3, ::2] = -0.0
        L[4, 7] = top
        L[5] = low
        L[5, 9] = top
        L[6] = top
        L[7] = -INF
        L[7, ::5] = low
        L[8] = torch.linspace(-1e38, 1e38, V, device=DEV).to(dtype)
        for kw in (dict(), dict(k=[5] * 9), dict(p=[0.7] * 9), dict(floor=[0.3] * 9), dict(temperature=[0.0] * 9),
                   dict(temperature=[3e38] * 9, p=[0.5] * 9), dict(temperature=[1e-38] * 9, k=[7] * 9)):
            check(em, L, u, **kw)


def test_rows_without_a_token(em):
    """NaN, infinity, nothing allowed, parameters out of range: -1 there, the other rows as they are."""
    V, T = 2000, 20
    L, u = zipf(T, V, F, 4)
    good = draw(em, L, u)
    bad = L.clone()
    bad[1, 1999] = float("nan")
    bad[2, 0] = INF
    bad[3] = -INF
    for kw in (dict(), dict(k=vec([9] * T, torch.int32)), dict(p=vec([0.9] * T))):
        want = draw(em, L, u, **kw)
        ids, logp, kept = draw(em, bad, u, **kw)
        for t in range(T):
            if t in (1, 2, 3):
                assert ids[t] == -1 and torch.isnan(logp[t]) and kept[t] == 0
            else:
                assert ids[t] == want[0][t] and logp[t] == want[1][t] and kept[t] == want[2][t]
    u2, temp, k = u.clone(), torch.ones(T, device=DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
    p, floor = torch.ones(T, device=DEV), torch.zeros(T, device=DEV)
    u2[0], u2[1], u2[2] = 1.0, -1e-9, float("nan")
    temp[3], temp[4], temp[5] = -1.0, INF, float("nan")
    k[6] = -1
    p[7], p[8], p[9] = -0.1, 1.0001, float("nan")
    floor[10], floor[11], floor[12] = -0.1, 1.5, float("nan")
    ids, logp, kept = draw(em, L, u2, temp, k, p, floor)
    assert (ids[:13] == -1).all() and torch.isnan(logp[:13]).all() and (kept[:13] == 0).all()
    assert torch.equal(ids[13:], good[0][13:]) and torch.equal(logp[13:], good[1][13:]) and (kept[13:] == V).all()


def test_probabilities(em):
    """Random numbers at even steps give every token its share, to one of them."""
    V, n = 300, 20000
    row = torch.randn(V, generator=gen(1), device=DEV) * 2
    L = row.expand(n, V).contiguous()
    u = (torch.arange(n, device=DEV) + 0.5) / n
    for k, p, floor in ((0, 1.0, 0.0), (40, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.05), (60, 0.9, 0.01)):
        ids, _, kept = draw(em, L, u, None, vec([k] * n, torch.int32), vec([p] * n), vec([floor] * n))
        assert (kept == kept[0]).all()
        e = torch.exp((row - row.max()).double())
        left = torch.argsort(row, descending=True)[:int(kept[0])]
        share = torch.zeros(V, dtype=torch.float64, device=DEV)
        share[left] = e[left] / e[left].sum()
        counts = torch.bincount(ids, minlength=V).double()
        # u is fp32: its steps are off by 2^-24, n 2^-24 < 0.002 of a count
        assert ((counts - share * n).abs() <= 1.01).all()


@pytest.mark.parametrize("T,V", [(513, 64), (700, 1000), (1025, 513)])
def test_more_rows_than_a_launch(em, T, V):
    print(f"sample T={T} V={V}", flush=True)
    L, u = zipf(T, V, BF, T)
    check(em, L, u, k=[5] * T, p=[0.9] * T)


def test_more_rows_than_a_grid(em):
    """More than 2^20 rows that are a block each: the same as in two calls."""
    T, V = (1 << 20) + 70, 5
    print(f"sample T={T} V={V}", flush=True)
    L, u = zipf(T, V, F, 3)
    k = torch.full((T,), 3, dtype=torch.int32, device=DEV)
    whole = draw(em, L, u, k=k)
    half = T // 2
    for a, b in ((0, half), (half, T)):
        for x, y in zip(draw(em, L[a:b], u[a:b], k=k[a:b]), whole):
            assert torch.equal(x, y[a:b])
    check(em, L[-50:], u[-50:], k=[3] * 50)


@pytest.mark.parametrize("dtype", [BF, F])
def test_few_values(em, dtype):
    """Thousands of tokens of each of a few logits, at random places: ends among more than a list holds."""
    T, V = 12, 128256
    print(f"sample few values {dtype}", flush=True)
    L = logits(T, V, dtype)
    L.copy_(20 + torch.randint(-3, 4, (T, V), generator=gen(1), device=DEV) * 0.125)
    u = torch.rand(T, generator=gen(2), device=DEV)
    k = [1, 2, 100, 5000, 20000, 60000, 100000, V, 0, 0, 0, 0]
    p = [1.0, 0.9, 0.5, 0.99, 1.0, 0.7, 0.95, 0.999, 0.01, 0.3, 0.9, 0.99]
    check(em, L, u, k=k)
    check(em, L, u, p=p)
    check(em, L, u, k=k, p=p, floor=[0.0, 0.5, 0.7, 0.8, 0.9, 0.95] * 2)
    L[:, 0] = -1e4                       # the bins are 2^-10 of a wide range
    L[:, V // 2] = 21.0
    check(em, L, u, k=k, p=p)


@pytest.mark.parametrize("V", [1000, 30000])
def test_tiny_min_p(em, V):
    """Tokens that min-p keeps although their weights round to nothing count as kept."""
    L, u = zipf(6, V, F, 4)
    L.copy_(-300 * torch.rand(6, V, generator=gen(6), device=DEV))
    check(em, L, u, floor=[1e-30, 1e-20, 1e-38, 1e-10, 1e-44, 1.0])
    check(em, L, u, floor=[1e-30] * 6, k=[0, 3, 2 ** 31 - 1, V // 2, 500, 1], temperature=[0.5, 1.0, 2.0, 3.0, 0.0, 1.0])


def test_row_alone_and_among_others(em):
    """A row's token depends on the row alone, in how many parts it may be worked on."""
    L, u = zipf(300, 40000, F, 8)
    k, p = vec([50] * 300, torch.int32), vec([0.9] * 300)
    for ask in (dict(), dict(k=k), dict(p=p), dict(k=k, p=p)):
        whole = draw(em, L, u, **ask)
        for t in (0, 5, 299):
            one = draw(em, L[t:t + 1], u[t:t + 1], **{n: x[t:t + 1] for n, x in ask.items()})
            for a, b in zip(one, whole):
                assert torch.equal(a, b[t:t + 1])


def test_offsets_past_32_bits(em):
    """2.4 GB of logits in one call; and one row of 2^24."""
    T, V = 2400, 262144
    print("sample 2.5 GB of logits", flush=True)
    L = torch.full((T, V), -20.0, device=DEV)
    at = torch.randint(0, V, (T,), generator=gen(2), device=DEV)
    L[torch.arange(T, device=DEV), at] = 30.0
    u = torch.full((T,), 0.5, device=DEV)
    ids, _, kept = draw(em, L, u, p=vec([0.99] * T))
    assert torch.equal(ids, at) and (kept == 1).all()
    del L
    V = 2 ** 24
    L, u = zipf(2, V, BF, 5)
    L[1] = 1.0
    check(em, L, u, k=[1000, 0], p=[0.9, 1.0])


def test_optional_outputs_and_no_rows(em):
    L, u = zipf(3, 100, F, 1)
    want = draw(em, L, u)
    ids = torch.empty(3, dtype=torch.int64, device=DEV)
    em.Sampler(3, 100)(L, u, ids)
    assert torch.equal(ids, want[0])
    em.Sampler(0, 100)(L[:0], u[:0], ids[:0])
    # a workspace of more tokens serves fewer, and a wider one
    ids.zero_()
    em.Sampler(900, 5000)(L, u, ids)
    assert torch.equal(ids, want[0])


def test_streams_and_graphs(em):
    T, V = 6, 30000
    L, u = zipf(T, V, BF, 7)
    L2, u2 = zipf(T, V, BF, 9)
    k, p, temperature = vec([40] * T, torch.int32), vec([0.9] * T), vec([0.8] * T)
    outs = [torch.empty(T, dtype=torch.int64, device=DEV) for _ in range(2)]
    samplers = [em.Sampler(T, V) for _ in range(2)]
    want = [draw(em, a, b, temperature, k, p)[0] for a, b in ((L, u), (L2, u2))]
    torch.cuda.synchronize()
    # two calls at once, each with its own workspace
    sides = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for s, side, (a, b), o in zip(samplers, sides, ((L, u), (L2, u2)), outs):
            with torch.cuda.stream(side):
                s(a, b, o, temperature=temperature, top_k=k, top_p=p)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    # two graphs that share a workspace, replayed one after the other
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, (a, b), o in zip(graphs, ((L, u), (L2, u2)), outs):
        with torch.cuda.graph(g):
            samplers[0](a, b, o, temperature=temperature, top_k=k, top_p=p)
    for i in range(4):
        u.copy_(torch.rand(T, generator=gen(i), device=DEV))
        L2.copy_(zipf(T, V, BF, i)[0])
        want = [draw(em, a, b, temperature, k, p)[0] for a, b in ((L, u), (L2, u2))]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]), i


@pytest.mark.parametrize("dtype", [BF, F])
def test_short_rows_leave_the_workspace_alone(em, dtype):
    """Rows of up to 8192 tokens with the 4 KiB they ask for, as many rows as there are; nothing of it or
    behind it is written."""
    for T, V in ((1, 8192), (700, 8192), (3000, 40)):
        print(f"sample workspace T={T} V={V} {dtype}", flush=True)
        L, u = zipf(T, V, dtype, V)
        k, p = vec([50] * T, torch.int32), vec([0.9] * T)
        assert em.ember_sample_workspace_bytes(T, V) == 4096
        buf = torch.full((4096 * 2,), 0xA5, dtype=torch.uint8, device=DEV)
        ids, logp, kept = torch.empty(T, dtype=torch.int64, device=DEV), torch.empty(T, device=DEV), vec([0] * T, torch.int32)
        em.ember_sample(L, u, ids, buf[:4096], top_k=k, top_p=p, logp=logp, kept=kept)
        assert (buf == 0xA5).all()
        for t in range(0, T, 97):
            i, lp, n = one_row(L[t], u[t].double().item(), 1.0, 50, vec([0.9])[0].item())
            assert (ids[t].item(), kept[t].item()) == (i, n), t


@pytest.mark.parametrize("T,V,dtype", [(513, 8193, F), (1030, 9001, BF), (520, 30000, BF)])
def test_more_long_rows_than_a_launch(em, T, V, dtype):
    """Rows past the 512 of a launch have their own parameters, in a workspace that the ones before left full."""
    print(f"sample long rows T={T} V={V} {dtype}", flush=True)
    L, u = zipf(T, V, dtype, T)
    r = [torch.rand(T, generator=gen(T + i), device=DEV) for i in range(4)]
    temperature = 0.3 + 1.4 * r[0]
    temperature[::11] = 0
    k = torch.where(r[1] < 0.4, 0, (10 ** (3.5 * r[1])).int())
    p = torch.where(r[2] < 0.3, 1.0, 0.5 + 0.5 * r[2])
    floor = torch.where(r[3] < 0.6, 0.0, 0.1 * (r[3] - 0.6))
    L[::13] = torch.randint(0, 3, (len(L[::13]), V), generator=gen(9), device=DEV).to(dtype) * 0.25      # ends among equal ones
    L[5::17, V // 2:] = -INF
    L[512:, V - 1] = -INF
    L[-1] = -INF
    check(em, L, u, temperature, k, p, floor)
    check(em, L, u)


def ends(V, dtype):
    low, top = torch.finfo(dtype).min, torch.finfo(dtype).max
    L, u = zipf(12, V, dtype, 3)
    L[0] = low
    L[1, 1:] = low
    L[2, ::2] = low
    L[3] = 0.0
    L[3, ::2] = -0.0
    L[4, V - 7] = top
    L[5] = low
    L[5, V // 2] = top
    L[6] = top
    L[7] = -INF
    L[7, ::5] = low
    L[8] = torch.linspace(-1e38, 1e38, V, device=DEV).to(dtype)
    L[9] = -torch.rand(V, generator=gen(5), device=DEV) * 1e-37          # a border about the smallest normal numbers
    L[10] = (torch.rand(V, generator=gen(6), device=DEV) - 0.5) * 1e-40  # subnormal in both types
    L[11] = low
    L[11, V - 1] = torch.nextafter(torch.tensor(low, dtype=dtype), torch.tensor(0.0, dtype=dtype))
    return L, u


@pytest.mark.parametrize("V", [8193, 20000])
@pytest.mark.parametrize("dtype", [BF, F])
def test_values_at_the_ends_of_long_rows(em, V, dtype):
    print(f"sample ends V={V} {dtype}", flush=True)
    L, u = ends(V, dtype)
    T = len(L)
    for kw in (dict(), dict(k=[5] * T), dict(p=[0.7] * T), dict(floor=[0.3] * T), dict(temperature=[0.0] * T),
               dict(temperature=[3e38] * T, p=[0.7] * T), dict(temperature=[1e-38] * T, k=[7] * T),
               dict(temperature=[1e-30] * T, p=[0.9] * T), dict(k=[V // 2] * T, p=[0.6] * T, floor=[0.01] * T),
               dict(temperature=[1e-44] * T, floor=[0.5] * T)):
        check(em, L, u, **kw)


@pytest.mark.parametrize("V", [8193, 20000, 128256])
@pytest.mark.parametrize("dtype", [BF, F])
def test_long_rows_without_a_token(em, V, dtype):
    """NaN or infinity in the first, a middle or the last part of a row, nothing allowed, parameters out of range: -1 there, the
    other rows as they are."""
    T = 20
    print(f"sample without V={V} {dtype}", flush=True)
    L, u = zipf(T, V, dtype, 4)
    want0 = draw(em, L, u)
    bad = logits(T, V, dtype)
    bad.copy_(L)
    for t, (i, x) in enumerate(((0, float("nan")), (V // 2, float("nan")), (V - 1, float("nan")), (0, INF), (V // 2, INF), (V - 1, INF))):
        bad[t, i] = x
    bad[6] = -INF
    bad[7, V // 3] = -float("nan")
    for kw in (dict(), dict(k=vec([9] * T, torch.int32)), dict(p=vec([0.9] * T)), dict(floor=vec([0.05] * T))):
        want = draw(em, L, u, **kw)
        got = draw(em, bad, u, **kw)
        assert (got[0][:8] == -1).all() and torch.isnan(got[1][:8]).all() and (got[2][:8] == 0).all()
        for a, b in zip(got, want):
            assert torch.equal(a[8:], b[8:])
    u2, temp, k = u.clone(), torch.ones(T, device=DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
    p, floor = torch.ones(T, device=DEV), torch.zeros(T, device=DEV)
    u2[0], u2[1], u2[2] = 1.0, -1e-9, float("nan")
    temp[3], temp[4], temp[5] = -1.0, INF, float("nan")
    k[6] = -1
    p[7], p[8], p[9] = -0.1, 1.0001, float("nan")
    floor[10], floor[11], floor[12] = -0.1, 1.5, float("nan")
    ids, logp, kept = draw(em, L, u2, temp, k, p, floor)
    assert (ids[:13] == -1).all() and torch.isnan(logp[:13]).all() and (kept[:13] == 0).all()
    assert torch.equal(ids[13:], want0[0][13:]) and torch.equal(logp[13:], want0[1][13:]) and (kept[13:] == V).all()
