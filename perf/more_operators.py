"""The operators that answer from a token table held in 4 bits, as measurable cases.

A model that answers one token after another reads both ends of its token
interface at every step: the row of the last token from the embedding table, and
the whole LM head for the next one's logits.  Both are held in 4 bits here, with a
scale a group of columns; from the logits a token is drawn with temperature,
top-k, top-p and min-p.  The hidden states a head reads are in 8 bits with one
scale a token, as the final norm writes them.

A case is a dict of plain values, ``kind`` one of:
  quantize  a table's rows to 4 bits, and all of them read back  -> values, scales
  rows      the rows of given tokens, read from 4 bits           -> rows
  logits    logits of T tokens from a head in 4 bits             -> logits
  answer    rows, the final norm in 8 bits, logits               -> rows, sum, logits
  sample    a token a row, drawn with given random numbers       -> ids, log-probabilities, kept

Codes: the 128 columns from 128 s on take 64 bytes of their row.  Byte 16 q + 4 w + b
of them holds the code of column 128 s + 32 w + 4 q + b in its lower half and that of
the column 16 further in its upper half, each in two's complement.  A code times the
scale (bf16) of its group of 32, 64 or 128 columns is the value it stands for.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
NORM_EPS = 1e-6
W_STD = 0.02
BLOCK = 128              # columns whose codes are packed together
CHUNK_ELEMS = 1 << 27    # elements made or checked at a time


def _named(c, name):
    if name is not None:
        c["name"] = name
    return c


def _quantize(V, D, group, x="bf16", name=None):
    return _named({"kind": "quantize", "V": V, "D": D, "group": group, "x": x}, name)


def _rows(T, V, D, group, y="bf16", name=None):
    return _named({"kind": "rows", "T": T, "V": V, "D": D, "group": group, "y": y}, name)


def _logits(kind, T, V, D, group, y="bf16", bias=False, name=None):
    return _named({"kind": kind, "T": T, "V": V, "D": D, "group": group, "y": y, "bias": bias}, name)


def _sample(T, V, x, filters, masked=False, name=None):
    """filters: "none" (temperature alone), "top_p", or "all": every row with its own
    temperature (some 0), top-k, top-p and min-p (some off); masked: a share of each
    row's logits is minus infinity."""
    return _named({"kind": "sample", "T": T, "V": V, "x": x, "filters": filters, "masked": masked}, name)


def listed():
    return [
        # A trained fp32 table of odd width, rounded for a device that has little memory.
        _quantize(8191, 1000, 32, "f32", name="quantize_8k_x1000_f32"),
        # A large vocabulary's table after its training, rounded once, and read back for a check.
        _quantize(128256, 4096, 128, name="quantize_128k_x4096"),
        # The embedding of the token that was answered last.
        _rows(1, 32000, 1024, 64, name="rows_1_32k_x1024"),
        # The embeddings of eight prompts of 2048 tokens.
        _rows(16384, 128256, 4096, 128, name="rows_16k_128k"),
        # One token answered by a large vocabulary's head ...
        _logits("logits", 1, 128256, 4096, 128, name="logits_1_128k"),
        # ... and one token each of sixteen requests, finer groups.
        _logits("logits", 16, 128256, 4096, 32, name="logits_16_128k_g32"),
        # A ragged validation batch of a small model, fp32 logits with a bias.
        _logits("logits", 333, 8191, 1000, 64, "f32", bias=True, name="logits_333_8k_x1000_f32"),
        # Validation of a prompt over a large vocabulary: the largest call.
        _logits("logits", 1024, 128256, 4096, 128, name="logits_1k_128k"),
        # One step of four requests: embeddings, the final norm, logits.
        _logits("answer", 4, 32000, 2048, 128, name="answer_4_32k_x2048"),
        # One token of a small model, no filter: latency.
        _sample(1, 8191, "f32", "none", name="sample_1_8k_f32"),
        # Sixteen requests, each with its own filters, some of them bound to a grammar.
        _sample(16, 128256, "bf16", "all", masked=True, name="sample_16_128k"),
        # Rollouts of reinforcement learning: 256 sequences side by side, nucleus sampling.
        _sample(256, 128256, "f32", "top_p", name="sample_256_128k_f32"),
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
    kind = rng.choice(["quantize", "rows", "logits", "logits", "logits", "answer", "sample", "sample"])
    while True:
        V = _log_int(rng, 1000, 262144)
        if kind == "sample":
            T = _log_int(rng, 1, 256)
            if T * V > 256 * 128256:
                continue
            return _sample(T, V, rng.choice(["bf16", "f32"]), rng.choice(["none", "top_p", "all", "all"]),
                           rng.random() < 0.3)
        D, group = _width(rng), rng.choice([32, 64, 128, 128])
        if V * D > 128256 * 4096:
            continue
        if kind == "quantize":
            return _quantize(V, D, group, rng.choice(["bf16", "bf16", "f32"]))
        if kind == "rows":
            T = _log_int(rng, 1, 16384)
            if T * D > 16384 * 4096:
                continue
            return _rows(T, V, D, group, rng.choice(["bf16", "bf16", "f32"]))
        T = _log_int(rng, 1, 1024 if kind == "logits" else 64)
        if T * V * D > 1024 * 128256 * 4096 or T * V > 1024 * 128256:
            continue
        y = "bf16" if kind == "answer" else rng.choice(["bf16", "bf16", "f32"])
        return _logits(kind, T, V, D, group, y, rng.random() < 0.3)


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


def _table(rows, D, dtype, gen):
    """Normal values, columns of different size (what a group's scale is for), a few rows much larger."""
    out = _padded(rows, D, dtype)
    col = W_STD * (0.25 + 2 * torch.rand(D, generator=gen, device="cuda").square())
    step = max(1, CHUNK_ELEMS // D)
    for r0 in range(0, rows, step):
        n = min(step, rows - r0)
        size = 1 + 7 * (torch.rand(n, 1, generator=gen, device="cuda") < 0.01)
        out[r0:r0 + n] = (torch.randn(n, D, generator=gen, device="cuda") * col * size).to(dtype)
    return out


def _groups(D, group):
    return (D + group - 1) // group


def _code_bytes(D):
    return (D + BLOCK - 1) // BLOCK * (BLOCK // 2)


def _scale_rows(V, D, group):
    return _padded(V, _groups(D, group), torch.bfloat16)


def _codes4(V, D, group, gen):
    """A table's codes and scales: each group has a code of 7 or -7."""
    blocks, q4 = _code_bytes(D) // 64, torch.empty(V, _code_bytes(D), dtype=torch.uint8, device="cuda")
    scale = _scale_rows(V, D, group)
    col = W_STD / 2 * (0.25 + 2 * torch.rand(_groups(D, group), generator=gen, device="cuda").square())
    step = max(1, CHUNK_ELEMS // (blocks * BLOCK))
    for v0 in range(0, V, step):
        n = min(step, V - v0)
        x = torch.randn(n, blocks * BLOCK, generator=gen, device="cuda")
        x[:, D:] = 0
        g = x.view(n, -1, group)
        c = torch.round(g * (7 / g.abs().amax(dim=2, keepdim=True).clamp_min(1e-3))).to(torch.int32)
        c = c.view(n, blocks, 4, 2, 4, 4)                        # w, half, q, b
        both = (c[:, :, :, 0] & 15) | ((c[:, :, :, 1] & 15) << 4)
        q4[v0:v0 + n] = both.permute(0, 1, 3, 2, 4).reshape(n, -1).to(torch.uint8)
        scale[v0:v0 + n] = (col * (0.5 + torch.rand(n, len(col), generator=gen, device="cuda"))).to(torch.bfloat16)
    return q4, scale


def _hidden8(T, D, gen):
    """Hidden states in 8 bits: codes and one scale a token."""
    q = _padded(T, D, torch.int8)
    x = torch.randn(T, D, generator=gen, device="cuda")
    a = x.abs().amax(dim=1)
    q.copy_(torch.round(x * (127 / a)[:, None]))
    return q, a / 127


def _state(case, seed):
    kind, V = case["kind"], case["V"]
    gen = _gen(seed, 1)
    if kind == "sample":
        return _sample_state(case, gen)
    D, group = case["D"], case["group"]
    if kind == "quantize":
        dt = DTYPES[case["x"]]
        return {"X": _table(V, D, dt, gen), "Wq": torch.empty(V, _code_bytes(D), dtype=torch.uint8, device="cuda"),
                "wscale": _scale_rows(V, D, group), "Y": _padded(V, D, dt)}
    T = case["T"]
    s = {}
    s["Wq"], s["wscale"] = _codes4(V, D, group, gen)
    if kind in ("rows", "answer"):
        # ids as text has them: frequent ones often, one of them next to itself
        s["tok"] = (V * torch.rand(T, generator=gen, device="cuda", dtype=torch.float64).pow(3)).long()
        s["tok"][T // 2:T // 2 + 1] = s["tok"][:1]
        s["Y"] = _padded(T, D, DTYPES[case["y"]])
    if kind == "answer":
        s["R"] = _padded(T, D, torch.bfloat16).copy_(torch.randn(T, D, generator=gen, device="cuda") * W_STD)
        s["gain"] = 0.5 + torch.rand(D, generator=gen, device="cuda")
        s["S"] = _padded(T, D, torch.bfloat16)
        s["Q"], s["qscale"] = _padded(T, D, torch.int8), torch.empty(T, dtype=torch.float32, device="cuda")
    if kind == "logits":
        s["Q"], s["qscale"] = _hidden8(T, D, gen)
    if kind != "rows":
        s["bias"] = torch.randn(V, generator=gen, device="cuda") if case["bias"] else None
        s["L"] = _padded(T, V, DTYPES[case["y"]])
    return s


def _sample_state(case, gen):
    """Logits whose probabilities fall with the rank's power of 0.8 to 1.8, as those of
    language models do, from nearly flat rows to peaked ones."""
    T, V, dt = case["T"], case["V"], DTYPES[case["x"]]

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    L = _padded(T, V, dt)
    power = 0.8 + rand(T)
    step = max(1, CHUNK_ELEMS // V)
    for t0 in range(0, T, step):
        n = min(step, T - t0)
        x = -torch.log1p(-rand(n, V)) * power[t0:t0 + n, None] - 4.0
        if case["masked"]:
            x[rand(n, V) < 0.5 * rand(n, 1)] = -math.inf
        L[t0:t0 + n] = x.to(dt)
    s = {"L": L, "u": rand(T), "temperature": 0.6 + 0.6 * rand(T), "top_k": None, "top_p": None, "min_p": None,
         "ids": torch.empty(T, dtype=torch.int64, device="cuda"), "logp": torch.empty(T, device="cuda"),
         "kept": torch.empty(T, dtype=torch.int32, device="cuda")}
    if case["filters"] != "none":
        s["top_p"] = 0.8 + 0.18 * rand(T)
    if case["filters"] == "all":
        s["temperature"][rand(T) < 0.1] = 0.0
        s["top_k"] = torch.where(rand(T) < 0.3, 0, (10 ** (1 + 2 * rand(T))).to(torch.int32))
        s["top_k"] = s["top_k"].to(torch.int32)
        s["top_p"][rand(T) < 0.3] = 1.0
        s["min_p"] = torch.where(rand(T) < 0.5, 0.0, 0.1 * rand(T))
    return s


def prepare(case, seed):
    s = _state(case, seed)
    s["case"] = case
    if own:
        s["own"] = _handles(case, s)
    return s


def _handles(case, s):
    """What a program that uses the framework keeps: the table in 4 bits, the norm, the sampler."""
    from paper_2607_01455_amd import ember

    h = {}
    if case["kind"] == "sample":
        h["sampler"] = ember.Sampler(case["T"], case["V"])
        return h
    h["table"] = ember.HeadQ4(s["Wq"], s["wscale"], case["D"], case["group"], bias=s.get("bias"))
    if "gain" in s:
        h["norm"] = ember.HeadNorm(s["gain"], eps=NORM_EPS, max_tokens=case["T"])
    return h


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _unpack(s, rows=None):
    """The values of a table's rows (all, or those of an index), in fp32."""
    q, scale, D, group = s["Wq"], s["wscale"], s["case"]["D"], s["case"]["group"]
    if rows is not None:
        q, scale = q[rows], scale[rows]
    c = q.view(torch.int8).view(q.shape[0], -1, 4, 4, 4)             # q, w, b
    c = torch.stack([(c << 4) >> 4, c >> 4], dim=2)                  # half, q, w, b
    c = c.permute(0, 1, 4, 2, 3, 5).reshape(q.shape[0], -1)[:, :D]
    return c.float() * scale.float().repeat_interleave(group, dim=1)[:, :D]


def _plain_logits(s, q, scale):
    y = q @ _unpack(s).t() * scale[:, None]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["L"].dtype)


def _plain_quantize(s):
    x, group = s["X"].float(), s["case"]["group"]
    V, D = x.shape
    x = torch.nn.functional.pad(x, (0, -D % group)).view(V, -1, group)
    scale = (x.abs().amax(dim=2) / 7).to(torch.bfloat16)
    step = scale.float()[:, :, None]
    c = torch.where(step > 0, torch.round(x / step), 0.0)
    return [(c * step).view(V, -1)[:, :D].to(s["X"].dtype), scale]


def _plain_sample(s):
    l, u = s["L"].double(), s["u"].double()[:, None]
    V = l.shape[1]
    greedy = s["temperature"][:, None] == 0
    heat = torch.where(greedy, 1.0, s["temperature"].double()[:, None])
    e = torch.exp((l - l.amax(dim=1, keepdim=True)) / heat)
    values, order = torch.sort(s["L"], dim=1, descending=True, stable=True)
    rank = torch.arange(V, device=l.device)
    keep = values > -math.inf
    k = torch.full_like(greedy, V, dtype=torch.int64) if s["top_k"] is None else s["top_k"].long()[:, None]
    k = torch.where(greedy, 1, torch.where(k == 0, V, k))
    keep = keep & (rank < k)
    fall = torch.where(keep, e.gather(1, order), 0.0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = fall.cumsum(dim=1) - fall
        keep = keep & ((before < p * fall.sum(dim=1, keepdim=True)) | (rank == 0) | (p >= 1))
    if s["min_p"] is not None:
        keep = keep & (fall >= s["min_p"].double()[:, None])
    part = torch.where(torch.zeros_like(keep).scatter(1, order, keep), e, 0.0).cumsum(dim=1)
    ids = (part <= u * part[:, -1:]).sum(dim=1)
    logp = torch.log(e.gather(1, ids[:, None])[:, 0] / e.sum(dim=1))
    return [ids, logp.float(), keep.sum(dim=1).to(torch.int32)]


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "quantize":
        return _plain_quantize(s)
    if kind == "sample":
        return _plain_sample(s)
    if kind == "logits":
        return [_plain_logits(s, s["Q"].float(), s["qscale"])]
    rows = _unpack(s, s["tok"]).to(s["Y"].dtype)
    if kind == "rows":
        return [rows]
    v = rows.float() + s["R"].float()
    y = v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + NORM_EPS) * s["gain"]
    a = y.abs().amax(dim=1)
    return [rows, v.to(torch.bfloat16), _plain_logits(s, torch.round(y * (127 / a)[:, None]), a / 127)]


def run(state):
    if not own:
        return _plain(state)
    s, h, kind = state, state["own"], state["case"]["kind"]
    if kind == "sample":
        h["sampler"](s["L"], s["u"], s["ids"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                     min_p=s["min_p"], logp=s["logp"], kept=s["kept"])
        return [s["ids"], s["logp"], s["kept"]]
    if kind == "quantize":
        h["table"].load(s["X"])
        h["table"].rows(None, s["Y"])
        return [s["Y"], s["wscale"]]
    if kind in ("rows", "answer"):
        h["table"].rows(s["tok"], s["Y"])
    if kind == "rows":
        return [s["Y"]]
    if kind == "answer":
        h["norm"](s["Y"], s["R"], S=s["S"], Q=s["Q"], qscale=s["qscale"])
    h["table"].logits(s["Q"], s["qscale"], s["L"])
    return [s["L"]] if kind == "logits" else [s["Y"], s["S"], s["L"]]


# ---------------------------------------------------------------------------
# work, and the same results in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once, each output written once; reading a table back reads what was just written."""
    kind, V = case["kind"], case["V"]
    if kind == "sample":
        T = case["T"]
        # one difference, exponential (12) and two sums a logit
        return {"bytes": T * V * SIZES[case["x"]] + 32 * T, "flops": 16 * T * V}
    D = case["D"]
    row = (D + 1) // 2 + 2 * _groups(D, case["group"])               # bytes of a row in 4 bits
    if kind == "quantize":
        return {"bytes": V * (2 * D * SIZES[case["x"]] + 2 * row), "flops": 5 * V * D}
    T = case["T"]
    fetch = {"bytes": T * (row + 8 + D * SIZES[case["y"]]), "flops": T * D}
    if kind == "rows":
        return fetch
    head = V * row + (4 * V if case["bias"] else 0) + T * V * SIZES[case["y"]]
    if kind == "logits":
        return {"bytes": head + T * D + 4 * T, "flops": 2 * T * V * D}
    return {"bytes": head + fetch["bytes"] + 4 * T * D + 4 * D, "flops": 2 * T * V * D + 8 * T * D}


def _exact_values(case, s, rows):
    """The values of some rows, column by column from where the codes' bytes are."""
    D = case["D"]
    k = torch.arange(D, device="cuda")
    at = k // 128 * 64 + k % 16 // 4 * 16 + k % 128 // 32 * 4 + k % 4
    nibble = (s["Wq"][rows][:, at].to(torch.int16) >> (4 * (k % 32 // 16)).to(torch.int16)) % 16
    code = torch.where(nibble > 7, nibble - 16, nibble)
    return code.double() * s["wscale"][rows][:, k // case["group"]].double()


def _exact_logits(case, s, q, scale):
    T, V = q.shape[0], case["V"]
    out = torch.empty(T, V, dtype=torch.float64, device="cuda")
    step = max(1, CHUNK_ELEMS // case["D"])
    for v0 in range(0, V, step):
        w = _exact_values(case, s, slice(v0, v0 + step))
        out[:, v0:v0 + step] = (q * scale) @ w.t()
    return out if s["bias"] is None else out + s["bias"].double()


def _exact_quantize(case, s):
    V, D, group = case["V"], case["D"], case["group"]
    values = torch.empty(V, D, dtype=torch.float64, device="cuda")
    scales = torch.empty(V, _groups(D, group), dtype=torch.bfloat16, device="cuda")
    for g in range(_groups(D, group)):
        x = s["X"][:, g * group:(g + 1) * group].double()
        step = (x.abs().max(dim=1).values / 7).to(torch.bfloat16)
        scales[:, g] = step
        values[:, g * group:(g + 1) * group] = torch.round(x / step.double()[:, None]) * step.double()[:, None]
    return [values, scales.double()]


def _exact_sample(s):
    """Row by row: the kept tokens are the first few of a list in falling order."""
    ids, logps, kepts = [], [], []
    for t in range(s["L"].shape[0]):
        l = s["L"][t].double()
        heat = s["temperature"][t].item()
        k = 0 if s["top_k"] is None else int(s["top_k"][t])
        p = 1.0 if s["top_p"] is None else s["top_p"][t].item()
        floor = 0.0 if s["min_p"] is None else s["min_p"][t].item()
        k, heat = (1, 1.0) if heat == 0 else (k, heat)
        best = torch.argsort(-l, stable=True)[:int((l > -math.inf).sum())]
        if k:
            best = best[:k]
        w = torch.exp(l[best] / heat - l.max() / heat)
        n = len(best)
        if p < 1:
            n = min(n, int(torch.searchsorted(torch.cumsum(w, 0), p * w.sum())) + 1)
        n = max(1, min(n, int((w >= floor).sum())))
        index, at = torch.sort(best[:n])
        part = torch.cumsum(w[at], 0)
        ids.append(index[torch.searchsorted(part, s["u"][t].double() * part[-1], right=True)])
        logps.append((l[ids[-1]] - l.max()) / heat - torch.log(torch.exp((l - l.max()) / heat).sum()))
        kepts.append(n)
    return [torch.stack(ids), torch.stack(logps), torch.tensor(kepts, dtype=torch.int32, device="cuda")]


def exact(case, seed):
    s, kind = _state(case, seed), case["kind"]
    if kind == "quantize":
        return _exact_quantize(case, s)
    if kind == "sample":
        return _exact_sample(s)
    if kind == "logits":
        return [_exact_logits(case, s, s["Q"].double(), s["qscale"].double().unsqueeze(1))]
    rows = _exact_values(case, s, s["tok"])
    if kind == "rows":
        return [rows]
    # the norm reads what was stored: rows rounded to bf16
    v = rows.to(torch.bfloat16).double() + s["R"].double()
    y = v * (v.pow(2).sum(dim=1, keepdim=True) / v.shape[1] + NORM_EPS).pow(-0.5) * s["gain"].double()
    scale = y.abs().max(dim=1, keepdim=True).values / 127
    return [rows, v, _exact_logits(case, s, torch.round(y / scale), scale)]
