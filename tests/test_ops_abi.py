"""Refusals of the norm, 8-bit and clipping entry points: bad arguments are
rejected on the host with the documented status codes before the device is
touched (no GPU is needed), and the binding refuses tensors that do not fit."""
import ctypes
import os
import re

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
X_, R_, GAIN_, S_, Y_, Q_, QS_, RSTD_, WS_, B_ = (k * A for k in range(1, 11))


def _norm(em, **kw):
    a = dict(X=X_, xd=1, ldx=64, R=R_, ldr=64, gain=GAIN_, gd=0, eps=1e-6, T=10, D=64, S=S_, lds=64, Y=Y_, yd=1,
             ldy=64, Q=Q_, ldq=64, qs=QS_, rstd=RSTD_)
    a.update(kw)
    return em.LIB.ember_rmsnorm(a["X"], a["xd"], a["ldx"], a["R"], a["ldr"], a["gain"], a["gd"], a["eps"], a["T"],
                                a["D"], a["S"], a["lds"], a["Y"], a["yd"], a["ldy"], a["Q"], a["ldq"], a["qs"],
                                a["rstd"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "SHAPE"), (dict(T=2 ** 26 + 1), "SHAPE"), (dict(D=0), "SHAPE"),
    (dict(D=32769, ldx=32776, ldr=32776, lds=32776, ldy=32776, ldq=32784), "SHAPE"),
    (dict(ldx=56), "SHAPE"), (dict(ldr=32), "SHAPE"), (dict(lds=8), "SHAPE"), (dict(ldy=56), "SHAPE"),
    (dict(ldq=48), "SHAPE"),
    (dict(X=None), "ARG"), (dict(gain=None), "ARG"), (dict(Q=None), "ARG"), (dict(qs=None), "ARG"),
    (dict(Y=None, Q=None, qs=None), "ARG"), (dict(R=None), "ARG"), (dict(eps=-1e-6), "ARG"),
    (dict(eps=float("nan")), "ARG"), (dict(eps=float("inf")), "ARG"),
    (dict(X=X_ + 8), "ALIGN"), (dict(R=R_ + 2), "ALIGN"), (dict(S=S_ + 4), "ALIGN"), (dict(Y=Y_ + 8), "ALIGN"),
    (dict(Q=Q_ + 8), "ALIGN"), (dict(ldq=72), "ALIGN"), (dict(qs=QS_ + 2), "ALIGN"), (dict(rstd=RSTD_ + 1), "ALIGN"),
    (dict(gain=GAIN_ + 4), "ALIGN"), (dict(ldx=68), "ALIGN"),
    (dict(xd=2), "DTYPE"), (dict(yd=-1), "DTYPE"), (dict(gd=7), "DTYPE"),
    # outputs that overlap an input other than element for element, or each other
    (dict(S=X_ + 128), "ARG"), (dict(S=X_, lds=72), "ARG"), (dict(Y=R_, yd=0), "ARG"), (dict(Q=X_), "ARG"),
    (dict(Y=S_), "ARG"), (dict(rstd=QS_), "ARG"), (dict(qs=GAIN_), "ARG"),
])
def test_norm_rejects_bad_arguments_on_host(em, kw, status):
    assert _norm(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def _grad(em, **kw):
    a = dict(dY=X_, lddy=64, S=S_, xd=1, lds=64, gain=GAIN_, gd=0, rstd=RSTD_, dS=R_, ldds=64, T=10, D=64, dX=Y_,
             lddx=64, dgain=QS_, ws=WS_, wsb=None)
    a.update(kw)
    if a["wsb"] is None:
        out = ctypes.c_size_t(0)
        em.LIB.ember_rmsnorm_grad_workspace_bytes(max(a["T"], 0), max(a["D"], 1), ctypes.byref(out))
        a["wsb"] = out.value
    return em.LIB.ember_rmsnorm_grad(a["dY"], a["lddy"], a["S"], a["xd"], a["lds"], a["gain"], a["gd"], a["rstd"],
                                     a["dS"], a["ldds"], a["T"], a["D"], a["dX"], a["lddx"], a["dgain"], a["ws"],
                                     a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "SHAPE"), (dict(D=0), "SHAPE"), (dict(lddy=56), "SHAPE"), (dict(lds=56), "SHAPE"),
    (dict(ldds=56), "SHAPE"), (dict(lddx=56), "SHAPE"),
    (dict(dY=None), "ARG"), (dict(S=None), "ARG"), (dict(gain=None), "ARG"), (dict(rstd=None), "ARG"),
    (dict(dX=None), "ARG"), (dict(dgain=None), "ARG"), (dict(ws=None), "ARG"),
    (dict(dY=X_ + 2), "ALIGN"), (dict(dS=R_ + 8), "ALIGN"), (dict(dX=Y_ + 4), "ALIGN"), (dict(rstd=RSTD_ + 2), "ALIGN"),
    (dict(dgain=QS_ + 2), "ALIGN"), (dict(ws=WS_ + 128), "ALIGN"), (dict(xd=3), "DTYPE"), (dict(gd=2), "DTYPE"),
    (dict(wsb=0), "WORKSPACE"),
    (dict(dX=X_ + 64), "ARG"), (dict(dX=S_, lddx=72), "ARG"), (dict(dgain=GAIN_), "ARG"), (dict(ws=X_), "ARG"),
])
def test_norm_gradient_rejects_bad_arguments_on_host(em, kw, status):
    assert _grad(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def test_norm_gradient_workspace_bytes(em):
    out = ctypes.c_size_t(0)
    f = em.LIB.ember_rmsnorm_grad_workspace_bytes
    assert f(-1, 64, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(10, 0, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(10, 32769, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(10, 64, None) == em.EMBER_ERR_ARG
    for D in (1, 64, 896, 4096, 32768):
        last = 0
        for T in (0, 1, 5, 100, 1000, 3000, 16384, 1 << 26):
            assert f(T, D, ctypes.byref(out)) == em.EMBER_OK
            assert out.value % 256 == 0 and out.value >= last    # one for more tokens serves fewer
            last = out.value


def _quant(em, **kw):
    a = dict(X=X_, xd=1, ldx=64, rows=10, D=64, Q=Q_, ldq=64, qs=QS_)
    a.update(kw)
    return em.LIB.ember_quantize_rows(a["X"], a["xd"], a["ldx"], a["rows"], a["D"], a["Q"], a["ldq"], a["qs"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), "SHAPE"), (dict(rows=2 ** 31), "SHAPE"), (dict(D=0), "SHAPE"), (dict(ldx=32), "SHAPE"),
    (dict(ldq=48), "SHAPE"), (dict(X=None), "ARG"), (dict(Q=None), "ARG"), (dict(qs=None), "ARG"),
    (dict(Q=None, qs=None), "ARG"), (dict(X=X_ + 2), "ALIGN"), (dict(Q=Q_ + 4), "ALIGN"), (dict(ldq=65), "ALIGN"),
    (dict(xd=9), "DTYPE"), (dict(Q=X_), "ARG"), (dict(qs=Q_), "ARG"),
])
def test_quantize_rows_rejects_bad_arguments_on_host(em, kw, status):
    assert _quant(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def _logits(em, **kw):
    a = dict(Xq=X_, ldx=64, xs=RSTD_, Wq=Q_, ldw=64, ws=QS_, bias=B_, T=10, V=100, D=64, Y=Y_, yd=1, ldy=104)
    a.update(kw)
    return em.LIB.ember_logits_q8(a["Xq"], a["ldx"], a["xs"], a["Wq"], a["ldw"], a["ws"], a["bias"], a["T"], a["V"],
                                  a["D"], a["Y"], a["yd"], a["ldy"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "SHAPE"), (dict(V=0), "SHAPE"), (dict(V=2 ** 31), "SHAPE"), (dict(D=0), "SHAPE"),
    (dict(D=32769, ldx=32784, ldw=32784), "SHAPE"), (dict(ldw=2 ** 22), "SHAPE"), (dict(ldx=48), "SHAPE"), (dict(ldw=48), "SHAPE"),
    (dict(ldy=96), "SHAPE"),
    (dict(Xq=None), "ARG"), (dict(xs=None), "ARG"), (dict(Wq=None), "ARG"), (dict(ws=None), "ARG"),
    (dict(Wq=None, ws=None), "ARG"), (dict(Xq=None, xs=None), "ARG"), (dict(Y=None), "ARG"),
    (dict(Xq=X_ + 8), "ALIGN"), (dict(Wq=Q_ + 4), "ALIGN"), (dict(ldx=72), "ALIGN"), (dict(ldw=68), "ALIGN"),
    (dict(xs=RSTD_ + 2), "ALIGN"), (dict(bias=B_ + 2), "ALIGN"), (dict(Y=Y_ + 2), "ALIGN"), (dict(ldy=100), "ALIGN"),
    (dict(yd=2), "DTYPE"), (dict(Y=X_), "ARG"), (dict(Y=Q_), "ARG"), (dict(bias=Y_), "ARG"),
])
def test_logits_reject_bad_arguments_on_host(em, kw, status):
    assert _logits(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def _clip(em, entries=None, n=None, max_norm=1.0, out=QS_, ws=WS_, wsb=None, **kw):
    a = dict(src=X_, src_dtype=1, lds=64, dst=Y_, dst_dtype=0, ldd=64, rows=10, cols=64, rows_dev=R_)
    a.update(kw)
    arr = (em.Grad * 2)(em.Grad(X_ + (1 << 20), 0, 8, X_ + (1 << 20), 0, 8, 1, 8, None), em.Grad(*a.values()))
    if wsb is None:
        size = ctypes.c_size_t(0)
        assert em.LIB.ember_clip_workspace_bytes(2, ctypes.byref(size)) == em.EMBER_OK
        wsb = size.value
    return em.LIB.ember_clip_grads(arr if entries is None else None, 2 if n is None else n, max_norm, out, ws, wsb,
                                   None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), "SHAPE"), (dict(n=2 ** 16 + 1), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(cols=-3), "SHAPE"),
    (dict(lds=63), "SHAPE"), (dict(ldd=10), "SHAPE"), (dict(rows=2 ** 22, cols=2 ** 21, lds=2 ** 21, ldd=2 ** 21), "SHAPE"),
    (dict(entries=0), "ARG"), (dict(max_norm=-1.0), "ARG"), (dict(max_norm=float("nan")), "ARG"), (dict(out=None), "ARG"),
    (dict(ws=None), "ARG"), (dict(src=None), "ARG"), (dict(dst=None), "ARG"),
    (dict(src=X_ + 1), "ALIGN"), (dict(dst=Y_ + 2), "ALIGN"), (dict(rows_dev=R_ + 4), "ALIGN"), (dict(out=QS_ + 2), "ALIGN"),
    (dict(ws=WS_ + 8), "ALIGN"), (dict(src_dtype=2), "DTYPE"), (dict(dst_dtype=-1), "DTYPE"), (dict(wsb=64), "WORKSPACE"),
    # in place is the same type and stride; otherwise source and destination are apart
    (dict(dst=X_), "ARG"), (dict(dst=X_, dst_dtype=1, ldd=72), "ARG"), (dict(dst=X_ + 16), "ARG"),
])
def test_clip_rejects_bad_arguments_on_host(em, kw, status):
    assert _clip(em, **kw) == getattr(em, "EMBER_ERR_" + status)


def test_clip_workspace_bytes(em):
    out = ctypes.c_size_t(0)
    f = em.LIB.ember_clip_workspace_bytes
    assert f(-1, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(2 ** 16 + 1, ctypes.byref(out)) == em.EMBER_ERR_SHAPE
    assert f(1, None) == em.EMBER_ERR_ARG
    sizes = []
    for n in (0, 1, 48, 49, 300, 2 ** 16):
        assert f(n, ctypes.byref(out)) == em.EMBER_OK
        sizes.append(out.value)
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_binding_refuses_tensors_that_do_not_fit(em):
    """Shapes and types the C entry points cannot see (CPU tensors: refused before any call)."""
    X, g = torch.zeros(4, 64), torch.ones(64)
    cases = [
        dict(gain=torch.ones(63)), dict(R=torch.zeros(3, 64)), dict(R=torch.zeros(4, 64, dtype=torch.bfloat16)),
        dict(R=X, S=torch.zeros(4, 60)), dict(Y=torch.zeros(5, 64)), dict(Q=torch.zeros(4, 64)),
        dict(Q=torch.zeros(4, 64, dtype=torch.int8), qscale=torch.zeros(3)),
        dict(Y=X, rstd=torch.zeros(4, dtype=torch.float64)), dict(Y=X, rstd=torch.zeros(8)[::2]),
    ]
    for kw in cases:
        with pytest.raises((ValueError, TypeError)):
            em.ember_rmsnorm(X, **{"gain": g, **kw})
    q, s = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    for args in ((q, s, torch.zeros(9, 48, dtype=torch.int8), torch.zeros(9), torch.zeros(4, 9)),
                 (q, s, torch.zeros(9, 64), torch.zeros(9), torch.zeros(4, 9)),
                 (q, torch.zeros(3), torch.zeros(9, 64, dtype=torch.int8), torch.zeros(9), torch.zeros(4, 9)),
                 (q, s, torch.zeros(9, 64, dtype=torch.int8), torch.zeros(8), torch.zeros(4, 9)),
                 (q, s, torch.zeros(9, 64, dtype=torch.int8), torch.zeros(9), torch.zeros(4, 8))):
        with pytest.raises((ValueError, TypeError)):
            em.ember_logits_q8(*args)
    ws = torch.zeros(4096)
    for kw in (dict(dX=torch.zeros(4, 63)), dict(dgain=torch.zeros(60)), dict(rstd=torch.zeros(2)),
               dict(dY=torch.zeros(4, 64, dtype=torch.bfloat16)), dict(dS=torch.zeros(1, 64))):
        a = dict(dY=X, S=X, gain=g, rstd=s, dX=X, dgain=torch.zeros(64), ws=ws)
        with pytest.raises((ValueError, TypeError)):
            em.ember_rmsnorm_grad(**{**a, **kw})
    with pytest.raises((ValueError, TypeError)):
        em.ember_quantize_rows(X, torch.zeros(4, 63, dtype=torch.int8), s)
    for args in ((X, torch.zeros(4, 63)), (torch.zeros(64, 4).t(),), (torch.zeros(2, 3, 4).transpose(0, 2),),
                 (X, None, torch.zeros(1)), (torch.zeros(64), None, torch.zeros(1, dtype=torch.int64))):
        with pytest.raises((ValueError, TypeError)):
            em.grad_entry(*args)
    with pytest.raises(ValueError):
        em.GradClipper([])
    with pytest.raises(ValueError):
        em.GradClipper([X, X], out=[X])


def test_profile_takes_every_kernel_the_library_names(em, monkeypatch):
    """ember_profile_collect of the binding has room for all the names that the library times."""
    names = set()
    csrc = os.path.join(ROOT, "paper_2607_01455_amd", "csrc")
    for f in os.listdir(csrc):
        if f.endswith((".cpp", ".hip", ".h")):
            names |= set(re.findall(r'timed\("(\w+)"', open(os.path.join(csrc, f)).read()))
    assert "ember_clip_grads" in names and "ember_stats" in names

    class Lib:
        @staticmethod
        def ember_profile_collect(buf, room, n):
            k = min(room, len(names))
            for i, name in zip(range(k), sorted(names)):
                buf[i].name, buf[i].launches, buf[i].total_ms = name.encode(), 1, 0.5
            n._obj.value = k
            return em.EMBER_OK

    monkeypatch.setattr(em, "LIB", Lib)
    assert set(em.ember_profile_collect()) == names


class OnGpu(torch.Tensor):
    """A host tensor that says it is on a GPU: the others of a call are then the ones to refuse."""
    index, is_cuda = 0, True

    def get_device(self):
        return self.index


class OnSecondGpu(OnGpu):
    index = 1


def test_binding_refuses_tensors_of_another_device(em):
    """An operand on the host, or on another GPU than the call's, is refused: its address
    would be read by the kernel (refused before the stream is asked for or any call is made)."""
    def z(*shape, dtype=torch.float32, cls=OnGpu):
        return torch.zeros(*shape, dtype=dtype).as_subclass(cls)

    def check(f, args, only=None):
        for name in args if only is None else only:
            for cls in (torch.Tensor, OnSecondGpu):
                with pytest.raises(ValueError, match=" on cpu"):
                    f(**{**args, name: args[name].as_subclass(cls)})

    i8 = torch.int8
    args = dict(X=z(4, 64), gain=z(64), R=z(4, 64), S=z(4, 64), Y=z(4, 64), Q=z(4, 64, dtype=i8), qscale=z(4), rstd=z(4))
    check(em.ember_rmsnorm, args)
    args = dict(dY=z(4, 64), S=z(4, 64), gain=z(64), rstd=z(4), dX=z(4, 64), dgain=z(64), ws=z(4096), dS=z(4, 64))
    check(em.ember_rmsnorm_grad, args)
    check(em.ember_quantize_rows, dict(X=z(4, 64), Q=z(4, 64, dtype=i8), qscale=z(4)))
    args = dict(Xq=z(4, 64, dtype=i8), xscale=z(4), Wq=z(9, 64, dtype=i8), wscale=z(9), Y=z(4, 9), bias=z(9))
    check(em.ember_logits_q8, args)
    one = z(1, dtype=torch.int64)
    check(em.grad_entry, dict(src=z(4, 64), dst=z(4, 64), rows_dev=one))
    with pytest.raises(ValueError):
        em.grad_entry(torch.zeros(5))
    entries = [em.grad_entry(z(5)), em.grad_entry(z(4, 8), rows_dev=one)]
    check(lambda **kw: em.ember_clip_grads(entries, 1.0, **kw), dict(out=z(2), ws=z(4096)), only=["ws"])
    for grads in ([z(5), torch.zeros(5)], [z(5), z(5, cls=OnSecondGpu)]):
        with pytest.raises(ValueError):
            em.GradClipper(grads)
    with pytest.raises(ValueError):
        em.ember_clip_grads([em.grad_entry(z(5)), em.grad_entry(z(5, cls=OnSecondGpu))], 1.0, z(2), z(4096))


def test_a_count_is_one_value(em):
    """No value would mean that all rows hold a gradient, more than one is not a count of them."""
    src = torch.zeros(4, 64).as_subclass(OnGpu)
    for n in (0, 2, 4):
        with pytest.raises(TypeError, match="one int64"):
            em.grad_entry(src, rows_dev=torch.zeros(n, dtype=torch.int64).as_subclass(OnGpu))
    assert em.grad_entry(src, rows_dev=torch.zeros((), dtype=torch.int64).as_subclass(OnGpu)).rows_dev


def test_no_rows_need_no_pointers(em):
    """With no tokens (no rows) there is nothing to do: any of the pointers may be NULL, and what
    is given is checked as ever."""
    none = dict(X=None, R=None, gain=None, S=None, Y=None, Q=None, qs=None, rstd=None)
    given = dict(X=X_, R=R_, gain=GAIN_, S=S_, Y=Y_, Q=Q_, qs=QS_, rstd=RSTD_)
    assert _norm(em, T=0, **none) == em.EMBER_OK
    for name in none:
        assert _norm(em, T=0, **{**none, name: given[name]}) == em.EMBER_OK
        assert _norm(em, T=0, **{name: None}) == em.EMBER_OK
    assert _norm(em, T=0, **{**none, "gd": 4}) == em.EMBER_ERR_DTYPE
    assert _norm(em, T=0, **{**none, "gain": GAIN_ + 4}) == em.EMBER_ERR_ALIGN
    assert _norm(em, T=0, **{**none, "D": 0}) == em.EMBER_ERR_SHAPE
    none = dict(X=None, Q=None, qs=None)
    assert _quant(em, rows=0, **none) == em.EMBER_OK
    for name in none:
        assert _quant(em, rows=0, **{name: None}) == em.EMBER_OK
    none = dict(Xq=None, xs=None, Wq=None, ws=None, bias=None, Y=None)
    assert _logits(em, T=0, **none) == em.EMBER_OK
    for name in none:
        assert _logits(em, T=0, **{name: None}) == em.EMBER_OK
    assert _logits(em, T=0, V=0, **none) == em.EMBER_ERR_SHAPE


def test_clip_refuses_gradients_over_what_it_writes(em):
    """out, the workspace and a row count share no memory with a gradient, its destination or each other."""
    n = 10 * 64
    for kw in (dict(out=X_), dict(out=X_ + 2 * n - 4), dict(out=Y_ + 8), dict(out=Y_ + 4 * n - 4), dict(ws=X_), dict(ws=Y_ + 256),
               dict(ws=Y_ - 256), dict(out=WS_ + 8), dict(out=R_), dict(ws=R_), dict(rows_dev=Y_ + 16),
               dict(lds=128, out=X_ + 256 + 120), dict(out=X_ + (1 << 20) + 16)):
        assert _clip(em, **kw) == em.EMBER_ERR_ARG, kw
