"""The operators around a token table's step, as measurable cases.

A model's last hidden states go through a residual addition and a
root-mean-square norm into the LM head; the norm's output is kept in bf16 or
fp32 for training, or in 8 bits with one scale a token for answering, where the
head's table is held in 8 bits with one scale a row.  Backwards, the norm's
gradient joins the tables' gradients, and all of them are clipped by their
global norm before the tables' steps.

A case is a dict of plain values, ``kind`` one of:
  norm       s = x + r, y = s rstd gain           -> s, y, rstd
  norm_q8    the same with y in 8 bits            -> s, the values y's codes stand for
  norm_grad  the norm's gradient                  -> dx, dgain
  logits     8-bit logits of T tokens             -> y
  answer     norm_q8, then logits                 -> s, y
  clip       global norm and clipping             -> gradients, norm, factor
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
NORM_EPS = 1e-6
W_STD, G_STD = 0.02, 1e-3
ZIPF_EXPONENT = 1.1      # token frequencies
CHUNK_ELEMS = 1 << 27    # elements made or checked at a time


def _norm(kind, T, D, x="bf16", residual=True, name=None):
    return _named({"kind": kind, "T": T, "D": D, "x": x, "residual": residual}, name)


def _logits(kind, T, V, D, y="bf16", bias=False, name=None):
    return _named({"kind": kind, "T": T, "V": V, "D": D, "y": y, "bias": bias}, name)


def _clip(V, D, tokens, tensors, elems, g="bf16", out="same", clipped=True, name=None):
    """V x D: a dense table's gradient (V = 0: none); tokens: rows of an
    embedding gradient, of which a count on the device says how many hold a
    token (0: none); tensors, elems: the other parameters' gradients, views of
    one bucket; out: "same" (in place) or the type the clipped gradients go to."""
    return _named({"kind": "clip", "V": V, "D": D, "tokens": tokens, "tensors": tensors, "elems": elems,
                   "g": g, "out": out, "clipped": clipped}, name)


def _named(c, name):
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # A handful of tokens of a small fp32 model of odd width: launches and latency.
        _norm("norm", 7, 1023, "f32", residual=False, name="norm_7x1023_f32"),
        # The final norm of an 8 x 2048 training batch.
        _norm("norm", 16384, 4096, name="norm_16k_x4096"),
        # The same for a prompt that is only answered: 8 bits out, a wide model.
        _norm("norm_q8", 2048, 8192, name="norm_q8_2k_x8192"),
        # Its gradient in training: the 8 x 2048 batch, with the gradient of the residual path ...
        _norm("norm_grad", 16384, 4096, name="norm_grad_16k_x4096"),
        # ... and one sequence of a narrow fp32 model without it.
        _norm("norm_grad", 2048, 896, "f32", residual=False, name="norm_grad_2k_x896_f32"),
        # One token answered by a large vocabulary's head, from the hidden state to the logits.
        _logits("answer", 1, 128256, 4096, name="answer_1_128k"),
        # One token each of sixteen requests.
        _logits("logits", 16, 128256, 4096, name="logits_16_128k"),
        # A ragged validation batch of a small model, fp32 logits with a bias.
        _logits("logits", 333, 8191, 1000, "f32", bias=True, name="logits_333_8k_x1000_f32"),
        # Validation of two 2048-token sequences over a large vocabulary: the largest call.
        _logits("logits", 4096, 128256, 4096, name="logits_4k_128k"),
        # A toy model's gradients, within the limit: in place, nothing to change.
        _clip(1024, 64, 0, 6, 50000, "f32", clipped=False, name="clip_toy_f32"),
        # A small model's 300 fp32 gradients in one bucket beside its table's, written clipped as bf16.
        _clip(32000, 1024, 0, 300, 60_000_000, "f32", "bf16", name="clip_300_tensors_f32_to_bf16"),
        # Both untied tables of a large-vocabulary model: the dense head and the embedding rows of an
        # 8 x 2048 batch, whose count is on the device, beside the norm's gains.
        _clip(128256, 4096, 16384, 2, 8192, "bf16", "bf16", name="clip_head_embed128k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi=8192):
    D = _log_int(rng, 64, hi)
    shape = rng.random()
    if shape < 0.6:      # most widths are multiples of 64
        return max(64, D // 64 * 64)
    if shape < 0.85:     # others whole 16-byte chunks
        return max(64, D // 16 * 16)
    return D


def draw(rng):
    kind = rng.choice(["norm", "norm_q8", "norm_grad", "logits", "logits", "answer", "clip", "clip"])
    while True:
        D = _width(rng)
        if kind in ("norm", "norm_q8", "norm_grad"):
            T = _log_int(rng, 1, 16384)
            if T * D > 16384 * 4096:
                continue
            return _norm(kind, T, D, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.7)
        V = _log_int(rng, 1000, 262144)
        if V * D > 128256 * 4096:
            continue
        if kind in ("logits", "answer"):
            T = _log_int(rng, 1, 4096 if kind == "logits" else 64)
            if T * V * D > 4096 * 128256 * 4096 or T * V > 4096 * 128256:
                continue
            y = "bf16" if kind == "answer" else rng.choice(["bf16", "bf16", "f32"])
            return _logits(kind, T, V, D, y, rng.random() < 0.3)
        g = rng.choice(["bf16", "bf16", "f32"])
        out = rng.choice(["same", "bf16", g])
        tensors = _log_int(rng, 1, 400)
        return _clip(V if rng.random() < 0.7 else 0, D, rng.choice([0, _log_int(rng, 256, 16384)]), tensors,
                     _log_int(rng, 1000 * tensors, 200000 * tensors), g, out, out != "same")


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + part) % (2 ** 63 - 1))
    return g


def _padded(rows, D, dtype):
    """A rows x D tensor whose rows start on 16-byte boundaries."""
    q = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.empty(max(rows, 1), (D + q - 1) // q * q, dtype=dtype, device="cuda")[:rows, :D]


def _normal(rows, D, std, dtype, gen, row_scale=None):
    out = _padded(rows, D, dtype)
    step = max(1, CHUNK_ELEMS // D)
    for r0 in range(0, rows, step):
        r1 = min(rows, r0 + step)
        x = torch.randn(r1 - r0, D, generator=gen, device="cuda") * std
        if row_scale is not None:
            x *= row_scale[r0:r1, None]
        out[r0:r1] = x.to(dtype)
    return out


def _codes(rows, D, std, gen):
    """Rows of normal data held in 8 bits: codes and one scale a row."""
    q, scale = _padded(rows, D, torch.int8), torch.empty(rows, dtype=torch.float32, device="cuda")
    step = max(1, CHUNK_ELEMS // D)
    for r0 in range(0, rows, step):
        r1 = min(rows, r0 + step)
        x = torch.randn(r1 - r0, D, generator=gen, device="cuda") * std
        a = x.abs().amax(dim=1)
        scale[r0:r1] = a / 127
        q[r0:r1] = torch.round(x * (127 / a)[:, None]).to(torch.int8)
    return q, scale


def _body_sizes(case):
    """Sizes of the other parameters' gradients: gains and biases beside
    matrices, in a fixed order, odd ones among them."""
    n = case["tensors"]
    w = [(1 + 7919 * i % 97) * (0.01 if i % 3 == 0 else 1.0) for i in range(n)]
    sizes = [max(1, int(case["elems"] * x / sum(w))) for x in w]
    return sizes


def _hidden(case, seed, part):
    """Hidden states and the residual stream they are added to: rows of
    different size, a few channels much larger than the others."""
    T, D, dt = case["T"], case["D"], DTYPES[case.get("x", "bf16")]
    gen = _gen(seed, part)
    size = 0.5 + torch.rand(T, generator=gen, device="cuda")
    s = {"X": _normal(T, D, 1.0, dt, gen, size)}
    if case.get("residual", True):
        s["R"] = _normal(T, D, 2.0, dt, gen)
        s["R"][:, ::max(1, D // 4)] *= 8
    s["gain"] = 0.5 + torch.rand(D, generator=gen, device="cuda")
    return s


def _norm_state(case, seed):
    T, D, dt = case["T"], case["D"], DTYPES[case["x"]]
    s = _hidden(case, seed, 1)
    if case["kind"] == "norm_grad":
        s["S"] = s.pop("X")
        s["dS"] = s.pop("R", None)
        if s["dS"] is not None:
            s["dS"].mul_(1e-4)
        S = s["S"].float()
        s["rstd"] = torch.rsqrt(S.square().mean(dim=1) + NORM_EPS)
        s["dY"] = _normal(T, D, 1e-4, dt, _gen(seed, 2))
        s["dX"] = _padded(T, D, dt)
        s["dgain"] = torch.empty(D, dtype=torch.float32, device="cuda")
        return s
    s["S"] = _padded(T, D, dt) if case["residual"] else None
    if case["kind"] == "norm":
        s["Y"] = _padded(T, D, dt)
        s["rstd"] = torch.empty(T, dtype=torch.float32, device="cuda")
    else:
        s["Q"], s["qscale"] = _padded(T, D, torch.int8), torch.empty(T, dtype=torch.float32, device="cuda")
    return s


def _logits_state(case, seed):
    T, V, D = case["T"], case["V"], case["D"]
    gen = _gen(seed, 3)
    s = {}
    s["Wq"], s["wscale"] = _codes(V, D, W_STD, gen)
    s["bias"] = torch.randn(V, generator=gen, device="cuda") if case["bias"] else None
    s["L"] = _padded(T, V, DTYPES[case["y"]])
    if case["kind"] == "answer":
        s |= _hidden(case, seed, 4)
        s["S"] = _padded(T, D, torch.bfloat16)
        s["Q"], s["qscale"] = _padded(T, D, torch.int8), torch.empty(T, dtype=torch.float32, device="cuda")
    else:
        s["Q"], s["qscale"] = _codes(T, D, 1.0, gen)
    return s


def _clip_state(case, seed):
    V, D, tokens, dt = case["V"], case["D"], case["tokens"], DTYPES[case["g"]]
    gen = _gen(seed, 5)
    grads, n = [], 0
    if V:
        p = torch.arange(1, V + 1, dtype=torch.float32, device="cuda").pow(-ZIPF_EXPONENT / 2)
        scale = p * math.sqrt(V / float(p.square().sum()))     # rows of frequent tokens are larger
        grads.append(_normal(V, D, G_STD, dt, gen, scale))
        n += V * D
    count = None
    if tokens:
        grads.append(_normal(tokens, D, G_STD, dt, gen))
        held = max(1, int(tokens * (0.25 + 0.5 * torch.rand(1, generator=gen, device="cuda").item())))
        count = torch.tensor([held], dtype=torch.int64, device="cuda")
        n += held * D
    sizes = _body_sizes(case)
    grads.append(torch.randn(sum(sizes), generator=gen, device="cuda").mul_(G_STD).to(dt))
    n += sum(sizes)
    outs = grads
    if case["out"] != "same":
        outs = [_padded(*g.shape, DTYPES[case["out"]]).zero_() if g.dim() == 2 else
                torch.zeros(g.shape, dtype=DTYPES[case["out"]], device="cuda") for g in grads]
    s = {"grads": grads, "outs": outs, "count": count, "sizes": sizes,
         "max_norm": G_STD * math.sqrt(n) * (0.3 if case["clipped"] else 3.0)}
    return s


def prepare(case, seed):
    if case["kind"].startswith("norm"):
        s = _norm_state(case, seed)
    elif case["kind"] == "clip":
        s = _clip_state(case, seed)
    else:
        s = _logits_state(case, seed)
    s["case"] = case
    if own:
        s["own"] = _handles(case, s)
    return s


def _handles(case, s):
    """What a program that uses the framework keeps: the norm with its gains
    and workspace, the 8-bit head, the list of its gradients."""
    from paper_2607_01455_amd import ember

    h = {}
    if case["kind"] != "clip" and "gain" in s:
        h["norm"] = ember.HeadNorm(s["gain"], eps=NORM_EPS, max_tokens=case["T"])
    if "Wq" in s:
        h["head"] = ember.HeadQ8(s["Wq"], s["wscale"], bias=s["bias"])
    if case["kind"] == "clip":
        def views(ts):
            return [t for t in ts if t.dim() == 2] + list(torch.split(ts[-1], s["sizes"]))
        tables = len(s["grads"]) - 1
        counts = [None] * (tables - (s["count"] is not None)) + [s["count"]] * (s["count"] is not None)
        counts += [None] * len(s["sizes"])
        same = case["out"] == "same"
        h["clip"] = ember.GradClipper(views(s["grads"]), out=None if same else views(s["outs"]), counts=counts)
    return h


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _plain_norm(s, eight_bits):
    x = s["X"].float()
    v = x + s["R"].float() if "R" in s else x
    rstd = torch.rsqrt(v.square().mean(dim=1) + NORM_EPS)
    y = v * rstd[:, None] * s["gain"]
    total = v.to(s["X"].dtype) if "R" in s else None
    if not eight_bits:
        return total, y.to(s["X"].dtype), rstd
    a = y.abs().amax(dim=1)
    return total, torch.round(y * (127 / a)[:, None]), a / 127


def _plain_logits(s, q, scale):
    y = q @ s["Wq"].float().t() * scale[:, None] * s["wscale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["L"].dtype)


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "norm":
        return list(_plain_norm(s, False))
    if kind == "norm_q8":
        total, q, scale = _plain_norm(s, True)
        return [total, (q * scale[:, None]).to(torch.bfloat16)]
    if kind == "norm_grad":
        v, dy, rstd = s["S"].float(), s["dY"].float(), s["rstd"][:, None]
        u = dy * s["gain"]
        dx = rstd * u - rstd.pow(3) * (u * v).mean(dim=1, keepdim=True) * v
        if s["dS"] is not None:
            dx = dx + s["dS"].float()
        return [dx.to(s["S"].dtype), (dy * v * rstd).sum(dim=0)]
    if kind == "logits":
        return [_plain_logits(s, s["Q"].float(), s["qscale"])]
    if kind == "answer":
        total, q, scale = _plain_norm(s, True)
        return [total, _plain_logits(s, q, scale)]
    held = [_held(g, s) for g in s["grads"]]
    total = torch.stack([h.square().sum() for h in held]).sum().sqrt()
    factor = torch.where(total > s["max_norm"], s["max_norm"] / total, torch.ones_like(total))
    outs = [o.copy_((h * factor).to(o.dtype)) for h, o in zip(held, s["outs"])]
    return [outs, total, factor]


def _held(g, s):
    """A gradient in 32 bits, without the rows that hold no token."""
    if s["count"] is None or g.dim() == 1 or g is not s["grads"][-2]:
        return g.float()
    at = torch.arange(g.shape[0], device=g.device)[:, None]
    return torch.where(at < s["count"], g.float(), 0.0)


def run(state):
    if not own:
        return _plain(state)
    s, h, kind = state, state["own"], state["case"]["kind"]
    if kind == "norm":
        h["norm"](s["X"], s.get("R"), S=s["S"], Y=s["Y"], rstd=s["rstd"])
        return [s["S"], s["Y"], s["rstd"]]
    if kind == "norm_q8":
        h["norm"](s["X"], s.get("R"), S=s["S"], Q=s["Q"], qscale=s["qscale"])
        return [s["S"], s["Q"] * s["qscale"].to(torch.bfloat16)[:, None]]
    if kind == "norm_grad":
        h["norm"].grad(s["dY"], s["S"], s["rstd"], s["dX"], s["dgain"], dS=s["dS"])
        return [s["dX"], s["dgain"]]
    if kind == "logits":
        h["head"].logits(s["Q"], s["qscale"], s["L"])
        return [s["L"]]
    if kind == "answer":
        h["norm"](s["X"], s["R"], S=s["S"], Q=s["Q"], qscale=s["qscale"])
        h["head"].logits(s["Q"], s["qscale"], s["L"])
        return [s["S"], s["L"]]
    total, factor = h["clip"](s["max_norm"])
    return [s["outs"], total, factor]


# ---------------------------------------------------------------------------
# work, and the same results in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once, each output written once; what is clipped counts as
    read once, and as written where the factor is below one or it goes elsewhere."""
    kind = case["kind"]
    if kind == "clip":
        rows = case["V"] + case["tokens"] // 2
        n = rows * case["D"] + sum(_body_sizes(case))
        w = 0 if case["out"] == "same" and not case["clipped"] else SIZES[case["g" if case["out"] == "same" else "out"]]
        return {"bytes": n * (SIZES[case["g"]] + w) + 8, "flops": 3 * n}
    T, D = case["T"], case["D"]
    es = SIZES[case.get("x", "bf16")]
    streams = 3 if case.get("residual", True) else 1           # x, r and s, or x
    norm = T * D * es * streams + 4 * D
    if kind == "norm":
        return {"bytes": norm + T * D * es + 4 * T, "flops": 5 * T * D}
    if kind == "norm_q8":
        return {"bytes": norm + T * D + 4 * T, "flops": 7 * T * D}
    if kind == "norm_grad":
        return {"bytes": T * D * es * (4 if case["residual"] else 3) + 4 * T + 8 * D, "flops": 10 * T * D}
    V = case["V"]
    head = V * D + 4 * V * (2 if case["bias"] else 1) + T * V * SIZES[case["y"]]
    return {"bytes": head + (norm if kind == "answer" else T * D + 4 * T), "flops": 2 * T * V * D}


def _exact_norm(s):
    v = s["X"].double()
    if "R" in s:
        v = v + s["R"].double()
    rstd = (v.pow(2).sum(dim=1) / v.shape[1] + NORM_EPS).pow(-0.5)
    return v, v * s["gain"].double() * rstd.unsqueeze(1), rstd


def _exact_codes(y):
    top = y.abs().max(dim=1, keepdim=True).values
    return torch.round(y / top * 127), top / 127


def _exact_logits(s, q, scale):
    V = s["Wq"].shape[0]
    out = torch.empty(q.shape[0], V, dtype=torch.float64, device="cuda")
    step = max(1, CHUNK_ELEMS // q.shape[1])
    for v0 in range(0, V, step):
        w = s["Wq"][v0:v0 + step].double() * s["wscale"][v0:v0 + step].double().unsqueeze(1)
        out[:, v0:v0 + step] = (q * scale) @ w.t()
    if s["bias"] is not None:
        out += s["bias"].double()
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind in ("norm", "norm_q8", "norm_grad"):
        s = _norm_state(case, seed)
    elif kind == "clip":
        s = _clip_state(case, seed)
    else:
        s = _logits_state(case, seed)
    if kind in ("norm", "norm_q8", "answer"):
        v, y, rstd = _exact_norm(s)
        total = v if "R" in s else None
        if kind == "norm":
            return [total, y, rstd]
        q, scale = _exact_codes(y)
        return [total, q * scale if kind == "norm_q8" else _exact_logits(s, q, scale)]
    if kind == "logits":
        return [_exact_logits(s, s["Q"].double(), s["qscale"].double().unsqueeze(1))]
    if kind == "norm_grad":
        v, dy, rstd = s["S"].double(), s["dY"].double(), s["rstd"].double().unsqueeze(1)
        h = v * rstd                                # the normed state without its gain
        u = dy * s["gain"].double()
        dx = rstd * (u - h * (u * h).sum(dim=1, keepdim=True) / v.shape[1])
        if s["dS"] is not None:
            dx = dx + s["dS"].double()
        return [dx, (dy * h).sum(dim=0)]
    parts, square = [], 0.0
    for g in s["grads"]:
        g = g.double()
        if s["count"] is not None and g.dim() == 2 and len(parts) == len(s["grads"]) - 2:
            g[int(s["count"]):] = 0.0
        parts.append(g)
        square = square + (g * g).sum()
    total = torch.sqrt(square)
    factor = torch.clamp(s["max_norm"] / total, max=1.0)
    return [[g * factor for g in parts], total, factor]
