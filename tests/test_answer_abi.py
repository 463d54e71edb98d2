"""Refusals of the entry points that answer from 4-bit tables: bad arguments are rejected
on the host with the documented status codes before the device is touched (no GPU is
needed), and the binding refuses tensors that do not fit."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def em():
    if not os.path.exists(os.path.join(ROOT, "paper_2607_01455_amd", "libember.so")):
        from paper_2607_01455_amd import build
        build.build()
    from paper_2607_01455_amd import ember
    return ember


# Fake, suitably aligned addresses: every call below must fail validation on
# the host, so none of them is ever dereferenced or passed to the device.
A = 1 << 24
X_, XS_, Q_, GS_, B_, Y_, TOK_, TEMP_, K_, P_, MP_, U_, IDS_, LOGP_, KEPT_ = (k * A for k in range(1, 16))
WS_ = 1 << 40        # past all of them


def _quant(em, **kw):
    a = dict(X=X_, xd=1, ldx=304, rows=10, D=300, group=64, Q=Q_, ldq=192, gs=GS_, lds=8)
    a.update(kw)
    return em.LIB.ember_quantize_rows_q4(a["X"], a["xd"], a["ldx"], a["rows"], a["D"], a["group"], a["Q"], a["ldq"],
                                         a["gs"], a["lds"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), "SHAPE"), (dict(rows=2 ** 31), "SHAPE"), (dict(D=0), "SHAPE"), (dict(D=32769, ldx=32776), "SHAPE"),
    (dict(ldx=296), "SHAPE"), (dict(ldq=176), "SHAPE"), (dict(ldq=2 ** 22), "SHAPE"), (dict(lds=4), "SHAPE"),
    (dict(group=32), "SHAPE"),                      # ten scales a row, at a stride of eight
    (dict(group=0), "ARG"), (dict(group=16), "ARG"), (dict(group=256), "ARG"), (dict(group=-64), "ARG"),
    (dict(X=None), "ARG"), (dict(Q=None), "ARG"), (dict(gs=None), "ARG"),
    (dict(X=X_ + 8), "ALIGN"), (dict(Q=Q_ + 4), "ALIGN"), (dict(ldq=200), "ALIGN"), (dict(gs=GS_ + 8), "ALIGN"),
    (dict(lds=12), "ALIGN"), (dict(xd=2), "DTYPE"),
    (dict(Q=X_), "ARG"), (dict(gs=Q_), "ARG"), (dict(Q=X_ + 608), "ARG"),
])
def test_quantize_rejects_bad_arguments_on_host(em, kw, status):
    assert _quant(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def _rows(em, **kw):
    a = dict(Wq=Q_, ldw=192, ws=GS_, lds=8, group=64, V=100, D=300, tok=TOK_, n=10, Y=Y_, yd=1, ldy=304)
    a.update(kw)
    return em.LIB.ember_rows_q4(a["Wq"], a["ldw"], a["ws"], a["lds"], a["group"], a["V"], a["D"], a["tok"], a["n"],
                                a["Y"], a["yd"], a["ldy"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(V=0), "SHAPE"), (dict(V=2 ** 31), "SHAPE"), (dict(D=0), "SHAPE"), (dict(D=32769, ldw=16448, lds=520, ldy=32776), "SHAPE"),
    (dict(n=-1), "SHAPE"), (dict(n=2 ** 26 + 1), "SHAPE"), (dict(tok=None, n=101), "SHAPE"), (dict(ldw=128), "SHAPE"),
    (dict(lds=0), "SHAPE"), (dict(ldy=296), "SHAPE"),
    (dict(group=48), "ARG"), (dict(Wq=None), "ARG"), (dict(ws=None), "ARG"), (dict(Y=None), "ARG"),
    (dict(Wq=Q_ + 8), "ALIGN"), (dict(ldw=196), "ALIGN"), (dict(ws=GS_ + 2), "ALIGN"), (dict(lds=9), "ALIGN"),
    (dict(tok=TOK_ + 4), "ALIGN"), (dict(Y=Y_ + 2), "ALIGN"), (dict(yd=3), "DTYPE"),
    (dict(Y=Q_), "ARG"), (dict(Y=GS_), "ARG"), (dict(Y=TOK_ - 16), "ARG"),
])
def test_rows_reject_bad_arguments_on_host(em, kw, status):
    assert _rows(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def _logits(em, **kw):
    a = dict(Xq=X_, ldx=304, xs=XS_, Wq=Q_, ldw=192, ws=GS_, lds=8, group=64, bias=B_, T=10, V=100, D=300, Y=Y_, yd=1,
             ldy=104)
    a.update(kw)
    return em.LIB.ember_logits_q4(a["Xq"], a["ldx"], a["xs"], a["Wq"], a["ldw"], a["ws"], a["lds"], a["group"],
                                  a["bias"], a["T"], a["V"], a["D"], a["Y"], a["yd"], a["ldy"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "SHAPE"), (dict(T=2 ** 26 + 1), "SHAPE"), (dict(V=0), "SHAPE"), (dict(V=2 ** 31), "SHAPE"), (dict(D=0), "SHAPE"),
    (dict(D=32769, ldx=32784, ldw=16448, lds=520), "SHAPE"), (dict(ldx=288), "SHAPE"), (dict(ldx=2 ** 22), "SHAPE"),
    (dict(ldw=128), "SHAPE"), (dict(ldw=2 ** 22), "SHAPE"), (dict(lds=0), "SHAPE"), (dict(lds=2 ** 22), "SHAPE"), (dict(ldy=96), "SHAPE"),
    (dict(group=31), "ARG"), (dict(Xq=None), "ARG"), (dict(xs=None), "ARG"), (dict(Wq=None), "ARG"), (dict(ws=None), "ARG"),
    (dict(Y=None), "ARG"),
    (dict(Xq=X_ + 8), "ALIGN"), (dict(ldx=312), "ALIGN"), (dict(xs=XS_ + 2), "ALIGN"), (dict(Wq=Q_ + 4), "ALIGN"),
    (dict(ldw=200), "ALIGN"), (dict(ws=GS_ + 8), "ALIGN"), (dict(lds=10), "ALIGN"), (dict(bias=B_ + 2), "ALIGN"),
    (dict(Y=Y_ + 2), "ALIGN"), (dict(ldy=100), "ALIGN"), (dict(yd=2), "DTYPE"),
    (dict(Y=X_), "ARG"), (dict(Y=Q_), "ARG"), (dict(Y=GS_), "ARG"), (dict(bias=Y_), "ARG"), (dict(xs=Y_), "ARG"),
])
def test_logits_reject_bad_arguments_on_host(em, kw, status):
    assert _logits(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def _sample(em, **kw):
    a = dict(L=X_, ld=1, ldl=1000, T=10, V=1000, temp=TEMP_, k=K_, p=P_, mp=MP_, u=U_, ids=IDS_, logp=LOGP_, kept=KEPT_,
             ws=WS_, wsb=None)
    a.update(kw)
    if a["wsb"] is None:
        size = ctypes.c_size_t(0)
        em.LIB.ember_sample_workspace_bytes(max(a["T"], 0), max(a["V"], 1), ctypes.byref(size))
        a["wsb"] = size.value
    return em.LIB.ember_sample(a["L"], a["ld"], a["ldl"], a["T"], a["V"], a["temp"], a["k"], a["p"], a["mp"], a["u"],
                               a["ids"], a["logp"], a["kept"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "SHAPE"), (dict(T=2 ** 26 + 1), "SHAPE"), (dict(V=0), "SHAPE"), (dict(V=2 ** 24 + 1, ldl=2 ** 24 + 8), "SHAPE"),
    (dict(ldl=992), "SHAPE"),
    (dict(L=None), "ARG"), (dict(u=None), "ARG"), (dict(ids=None), "ARG"), (dict(ws=None), "ARG"),
    (dict(L=X_ + 4), "ALIGN"), (dict(ldl=1001), "ALIGN"), (dict(temp=TEMP_ + 2), "ALIGN"), (dict(k=K_ + 1), "ALIGN"),
    (dict(p=P_ + 2), "ALIGN"), (dict(mp=MP_ + 3), "ALIGN"), (dict(u=U_ + 2), "ALIGN"), (dict(ids=IDS_ + 4), "ALIGN"),
    (dict(logp=LOGP_ + 2), "ALIGN"), (dict(kept=KEPT_ + 2), "ALIGN"), (dict(ws=WS_ + 128), "ALIGN"),
    (dict(ld=2), "DTYPE"), (dict(wsb=1000), "WORKSPACE"),
    (dict(ids=X_), "ARG"), (dict(ids=U_), "ARG"), (dict(logp=TEMP_), "ARG"), (dict(kept=LOGP_), "ARG"), (dict(ws=X_), "ARG"),
    (dict(kept=K_), "ARG"),
])
def test_sample_rejects_bad_arguments_on_host(em, kw, status):
    assert _sample(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def test_sample_workspace_bytes(em):
    out = ctypes.c_size_t(0)
    f = em.LIB.ember_sample_workspace_bytes
    assert f(-1, 64, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(10, 0, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(10, 2 ** 24 + 1, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(10, 64, None) == em.EMBER_ERR_ARG
    for V in (1, 1000, 128256, 2 ** 24):
        last = 0
        for T in (0, 1, 5, 100, 1000, 1 << 26):
            assert f(T, V, ctypes.byref(out)) == em.EMBER_OK
            assert out.value % 256 == 0 and out.value >= last    # one for more tokens serves fewer
            last = out.value
    for T in (1, 700):
        last = 0
        for V in (1, 511, 1000, 128256, 2 ** 24):
            assert f(T, V, ctypes.byref(out)) == em.EMBER_OK and out.value >= last
            last = out.value


def test_calls_without_rows_need_no_pointers(em):
    null = dict(Wq=None, ws=None, Y=None)
    assert _quant(em, rows=0, X=None, Q=None, gs=None) == em.EMBER_OK
    assert _rows(em, n=0, tok=None, **null) == em.EMBER_OK
    assert _logits(em, T=0, Xq=None, xs=None, bias=None, **null) == em.EMBER_OK
    assert _sample(em, T=0, L=None, u=None, ids=None, logp=None, kept=None, ws=None, wsb=0) == em.EMBER_OK


def test_binding_refuses_tensors_that_do_not_fit(em):
    """Shapes and types the C entry points cannot see (CPU tensors: refused before any call)."""
    bf, u8, i8 = torch.bfloat16, torch.uint8, torch.int8
    X, Q, s = torch.zeros(4, 200), torch.zeros(4, 128, dtype=u8), torch.zeros(4, 8, dtype=bf)[:, :4]
    for args in ((X, Q[:3], s, 64), (X, Q.to(i8), s, 64), (X, Q[:, :64], s, 64), (X, Q, s[:, :3], 64), (X, Q, s.float(), 64),
                 (X, Q, s, 48), (X, Q, s, 128), (X, Q, s[:2], 64)):
        with pytest.raises((ValueError, TypeError)):
            em.ember_quantize_rows_q4(*args)
    Y = torch.zeros(3, 200)
    for args in ((Q, s, Y, 64, torch.zeros(3, dtype=torch.int32)), (Q, s, Y, 64, torch.zeros(4, dtype=torch.int64)),
                 (Q, s, Y[:, :100], 64), (Q, s, Y, 32), (Q[:2], s, Y, 64), (Q, s.float(), Y, 64)):
        with pytest.raises((ValueError, TypeError)):
            em.ember_rows_q4(*args)
    Xq, xs, L = torch.zeros(3, 200, dtype=i8), torch.zeros(3), torch.zeros(3, 4)
    for args in ((Xq.to(u8), xs, Q, s, L, 64), (Xq, xs[:2], Q, s, L, 64), (Xq, xs, Q, s, L[:, :3], 64), (Xq, xs, Q, s, L[:2], 64),
                 (Xq[:, :100], xs, Q, s, L, 64), (Xq, xs, Q, s, L, 96), (Xq, xs, Q, s, L, 64, torch.zeros(3)),
                 (Xq, xs.double(), Q, s, L, 64)):
        with pytest.raises((ValueError, TypeError)):
            em.ember_logits_q4(*args)
    head = em.HeadQ4(Q, s, 200, 64)
    with pytest.raises(ValueError):
        head.logits(Xq[:, :190], xs, L)       # as many bytes of codes and scales, other columns
    with pytest.raises(ValueError):
        head.rows(None, Y[:, :190])
    L, u, ids, ws = torch.zeros(3, 8), torch.zeros(3), torch.zeros(3, dtype=torch.int64), torch.zeros(1 << 16)
    for kw in (dict(u=u[:2]), dict(u=u.double()), dict(ids=ids.int()), dict(ids=ids[:1]), dict(temperature=torch.zeros(2)),
               dict(top_k=torch.zeros(3, dtype=torch.int64)), dict(top_p=torch.zeros(6)[::2]), dict(min_p=torch.zeros(1)),
               dict(logp=torch.zeros(3, dtype=torch.float64)), dict(kept=torch.zeros(3, dtype=torch.int64)),
               dict(top_k=torch.zeros(3))):
        with pytest.raises((ValueError, TypeError)):
            em.ember_sample(**{**dict(L=L, u=u, ids=ids, ws=ws), **kw})


def test_head_takes_a_table_of_its_own_columns(em):
    """250 columns have as many bytes of codes and as many groups as 200: only the head knows which it has."""
    head = em.HeadQ4(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.bfloat16)[:, :4], 200, 64)
    assert em.q4_shapes(4, 250, 64) == em.q4_shapes(4, 200, 64)
    for D in (193, 199, 201, 250, 256):
        with pytest.raises(ValueError, match=f"{D} columns"):
            head.load(torch.zeros(4, D))


def test_short_rows_ask_for_no_workspace_of_their_own(em):
    """Rows of up to 8192 tokens are one launch without scratch memory: the same 4 KiB for any number of them."""
    out = ctypes.c_size_t(0)
    for V in (1, 64, 5000, 8192):
        for T in (0, 1, 512, 1 << 26):
            assert em.LIB.ember_sample_workspace_bytes(T, V, ctypes.byref(out)) == em.EMBER_OK and out.value == 4096
    assert _sample(em, V=8192, ldl=8192, T=1 << 20, wsb=4095) == em.EMBER_ERR_WORKSPACE
    # longer rows ask for their bins, lists and chunks, and are refused with less
    for T in (0, 1, 600):
        assert em.LIB.ember_sample_workspace_bytes(T, 8193, ctypes.byref(out)) == em.EMBER_OK
        assert out.value >= max(4096, min(T, 512) * (1024 * 12 + 8192 * 8))
        if T:
            args = dict(T=T, V=8193, ldl=8200)
            assert _sample(em, wsb=out.value - 1, **args) == em.EMBER_ERR_WORKSPACE
            assert _sample(em, wsb=4096, **args) == em.EMBER_ERR_WORKSPACE
