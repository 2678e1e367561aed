"""Timed cases of a stage's model operators, through the torch-facing public API.

  rope, rope_back    the norm of every query and key head with the rotation by position, and its gradients
  loss, loss_grad    the tail stage's loss against a teacher's top logits, alone and with the gradient of the logits
  int8               a projection of a frozen model in 8 bits: the activations quantised per token, the product with
                     weights quantised per output channel

Sizes: d = 2048 and 4096, vocabularies 32000 and 128256 and the token counts are those of this repository's workloads
(synth.py); heads of 64 to 256 columns, odd token counts and odd vocabularies are generic.
"""

from __future__ import annotations

import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_EPS = 1e-6
_MAX_POS = 8192


def _rope(kind, tokens, q_heads, k_heads, head_dim, rot_dim, dtype="bf16", pairing="halves", layout="packed", positions="implicit", seq=2048):
    """layout: "packed" (views of one [tokens, q|k|v] buffer, as a fused projection leaves them), "heads" (head-major, each
    head's tokens contiguous) or "plain"; positions: "implicit" (token t at t mod seq) or "packed" (documents, one int each)."""
    return {"kind": kind, "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "head_dim": head_dim, "rot_dim": rot_dim, "dtype": dtype,
            "pairing": pairing, "layout": layout, "positions": positions, "seq": seq}


def _loss(kind, tokens, vocab, top, dtype="bf16", tau=1.0, absent=0.0, masked=0.0):
    """absent: share of a row's teacher entries that are padding; masked: share of rows of weight 0."""
    return {"kind": kind, "tokens": tokens, "vocab": vocab, "top": top, "dtype": dtype, "tau": tau, "absent": absent, "masked": masked}


def _int8(tokens, inner, outer, dtype="bf16"):
    return {"kind": "int8", "tokens": tokens, "inner": inner, "outer": outer, "dtype": dtype}


def listed():
    cases = {
        # one token of a sequence that is being continued: latency only
        "rope_one_token": _rope("rope", 1, 32, 8, 128, 128, positions="packed"),
        # the wide model's microbatch, queries and keys as views of the fused projection's output
        "rope_microbatch": _rope("rope", 65536, 32, 8, 128, 128),
        # packed documents kept in fp32, three quarters of a head rotated, adjacent pairs, head-major
        "rope_back_ragged_fp32": _rope("rope_back", 3001, 12, 4, 80, 64, "f32", "adjacent", "heads", "packed"),
        # the backward pass of half a microbatch
        "rope_back_microbatch": _rope("rope_back", 32768, 32, 8, 128, 128),
        # a few tokens of an evaluation, the small model's vocabulary in fp32
        "loss_few_tokens_fp32": _loss("loss", 61, 32000, 32, "f32", tau=2.0, absent=0.2),
        # one sequence evaluated against the teacher
        "loss_one_sequence": _loss("loss", 2048, 128256, 64),
        # a vocabulary with odd rows, padded teacher rows, padding tokens
        "loss_grad_odd_vocab": _loss("loss_grad", 1023, 32003, 20, tau=2.0, absent=0.3, masked=0.1),
        # the tail stage's microbatch: loss and the gradient of 8192 rows of logits
        "loss_grad_microbatch": _loss("loss_grad", 8192, 128256, 64, tau=1.5),
        # one token through an output projection: latency and the weights' bytes
        "int8_one_token": _int8(1, 4096, 4096),
        # a ragged batch of sequences, an odd number of channels
        "int8_ragged": _int8(777, 2000, 5003),
        # the teacher's head for a few sequences' last tokens
        "int8_head": _int8(64, 4096, 128256),
        # an up-projection of the wide model over a microbatch
        "int8_microbatch": _int8(16384, 4096, 14336),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(("rope", "rope_back", "loss", "loss_grad", "int8"))
    if kind in ("rope", "rope_back"):
        head = rng.choice((64, 80, 96, 128, 192, 256))
        rot = head if rng.random() < 0.6 else 2 * rng.randint(1, head // 2)
        k_heads = rng.randint(1, 16)
        return _rope(kind, _log(rng, 1, 65536), k_heads * rng.randint(1, 8), k_heads, head, rot, rng.choice(("bf16", "bf16", "f32")),
                     rng.choice(("halves", "adjacent")), rng.choice(("packed", "plain", "heads")), rng.choice(("implicit", "packed")),
                     _log(rng, 64, _MAX_POS))
    if kind in ("loss", "loss_grad"):
        return _loss(kind, _log(rng, 1, 8192), _log(rng, 500, 200000), _log(rng, 1, 128), rng.choice(("bf16", "bf16", "f32")),
                     rng.choice((1.0, 1.5, 2.0, 4.0)), rng.choice((0.0, 0.3)), rng.choice((0.0, 0.1)))
    inner = _log(rng, 64, 16384)
    inner += -inner % rng.choice((1, 16, 128))
    return _int8(_log(rng, 1, 16384), inner, _log(rng, 64, 128256), rng.choice(("bf16", "bf16", "f32")))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 6e13   # a full-rate fp32 product, which is what the plain form runs at


def draw(rng):
    most = {}
    for c in listed():
        group = c["kind"][:4]
        most[group] = max(most.get(group, 0.0), _cost(c))
    while True:
        case = _draw(rng)
        if _cost(case) <= most[case["kind"][:4]]:
            return case


# ---- inputs -------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    """Normal values in the stored type, made in blocks so that no fp32 copy of a large tensor is kept."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.normal_(0.0, scale, generator=g)


def _heads(buf, case, heads, first):
    """The [tokens, heads, head_dim] view of a tensor made by _head_buffer, from head `first` on."""
    return buf[:, first:first + heads] if case["layout"] != "heads" else buf[first:first + heads].transpose(0, 1)


def _head_buffer(g, case, heads, dtype):
    t, d = case["tokens"], case["head_dim"]
    return _normal(g, (heads, t, d) if case["layout"] == "heads" else (t, heads, d), dtype)


def _positions(g, case):
    t = case["tokens"]
    if case["positions"] == "implicit":
        return None
    # documents of unequal length one after the other: the position starts again at each
    start = torch.randint(0, _MAX_POS, (1,), generator=g, device="cuda")
    at = torch.arange(t, device="cuda")
    length = 1 + torch.randint(0, case["seq"], (1,), generator=g, device="cuda")
    return ((at + start) % torch.clamp(length, min=7)).to(torch.int32) if t > 1 else start.to(torch.int32)


def _rope_table(rot_dim):
    """[positions, rot_dim] fp32: cosines, then sines, of the angles in 64 bits."""
    freq = 10000.0 ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device="cuda") / rot_dim)
    angle = torch.arange(_MAX_POS, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat((angle.cos(), angle.sin()), dim=1).float()


def _prepare_rope(case, g):
    dt, qh, kh, d = _TORCH[case["dtype"]], case["q_heads"], case["k_heads"], case["head_dim"]
    if case["layout"] == "plain":
        q, k = _head_buffer(g, case, qh, dt), _head_buffer(g, case, kh, dt)
    else:
        buf = _head_buffer(g, case, qh + (2 if case["layout"] == "packed" else 1) * kh, dt)
        q, k = _heads(buf, case, qh, 0), _heads(buf, case, kh, qh)
    s = {"q": q, "k": k, "pos": _positions(g, case), "table": _rope_table(case["rot_dim"]),
         "wq": (1 + _normal(g, (d,), torch.float32, 0.2)).to(dt), "wk": (1 + _normal(g, (d,), torch.float32, 0.2)).to(dt)}
    if case["kind"] == "rope_back":   # attention's gradients arrive as they are, in one piece each
        s["dq"], s["dk"] = _normal(g, (case["tokens"], qh, d), dt), _normal(g, (case["tokens"], kh, d), dt)
    if own:
        from paper_2607_13332_b200.stage_ops import QKNormRope
        s["op"] = QKNormRope(case["dtype"], d, s["wq"], s["wk"], s["table"], eps=_EPS, pairing=case["pairing"])
    return s


def _prepare_loss(case, g):
    t, v, k = case["tokens"], case["vocab"], case["top"]
    k = min(k, v)
    logits = _normal(g, (t, v), _TORCH[case["dtype"]], 2.5)
    # the teacher's best entries: distinct ids of a row (an odd step through the vocabulary), falling logits
    first = torch.randint(0, v, (t, 1), generator=g, device="cuda")
    ids = (first + torch.arange(k, device="cuda") * max(1, v // max(k, 1) - 1)) % v
    top = (8.0 + 1.5 * _normal(g, (t, k), torch.float32)).sort(dim=1, descending=True).values.contiguous()
    if case["absent"]:   # rows end early, some at once
        keep = torch.randint(0, k + 1, (t, 1), generator=g, device="cuda")
        cut = torch.rand((t, 1), generator=g, device="cuda") < 2 * case["absent"]
        ids = torch.where(cut & (torch.arange(k, device="cuda") >= keep), -1, ids)
    weight = torch.full((t,), 1.0 / t, device="cuda")
    if case["masked"]:
        weight = torch.where(torch.rand((t,), generator=g, device="cuda") < case["masked"], 0.0, weight)
    return {"logits": logits, "ids": ids.to(torch.int32).contiguous(), "top": top, "weight": weight}


def _prepare_int8(case, g):
    dt = _TORCH[case["dtype"]]
    x = _normal(g, (case["tokens"], case["inner"]), dt)
    x[:, ::97] *= 8.0   # the few wide columns that activations have
    w = _normal(g, (case["outer"], case["inner"]), torch.bfloat16, 1.0 / math.sqrt(case["inner"]))
    wq = torch.empty(w.shape, dtype=torch.int8, device="cuda")
    ws = torch.empty((case["outer"],), dtype=torch.float32, device="cuda")
    for at in range(0, case["outer"], 16384):
        ws[at:at + 16384] = w[at:at + 16384].abs().amax(dim=1).float() / 127.0
        wq[at:at + 16384] = torch.round(w[at:at + 16384].float() / ws[at:at + 16384, None]).to(torch.int8)
    return {"x": x, "wq": wq, "ws": ws}


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    make = _prepare_rope if kind.startswith("rope") else _prepare_loss if kind.startswith("loss") else _prepare_int8
    return dict(make(case, g), case=case)


# ---- plain forms --------------------------------------------------------------------------------------------------------------
def _angles(s, dtype=torch.float32):
    """Cosine and sine [tokens, 1, rot_dim / 2] of every token."""
    case = s["case"]
    pos = s["pos"]
    if pos is None:
        pos = torch.arange(case["tokens"], device="cuda") % case["seq"]
    row = s["table"][pos.long()].to(dtype)[:, None, :]
    half = case["rot_dim"] // 2
    return row[..., :half], row[..., half:]


def _rotate(x, cos, sin, case, sign):
    """x with the pairs of its first rot_dim columns turned by sign times the angle."""
    rot = case["rot_dim"]
    if case["pairing"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat((a * cos - sign * b * sin, b * cos + sign * a * sin, x[..., rot:]), dim=-1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    turned = torch.stack((a * cos - sign * b * sin, b * cos + sign * a * sin), dim=-1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _rope_forward(s, x, w, dtype=torch.float32):
    x, cos_sin = x.to(dtype), _angles(s, dtype)
    n = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + _EPS) * w.to(dtype)
    return _rotate(n, *cos_sin, s["case"], 1.0)


def _rope_backward(s, x, w, dy, dtype=torch.float32):
    x, w = x.to(dtype), w.to(dtype)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + _EPS)
    xh = x * r
    g = _rotate(dy.to(dtype), *_angles(s, dtype), s["case"], -1.0)
    h = g * w
    dx = r * (h - xh * (h * xh).mean(dim=-1, keepdim=True))
    return dx, (g * xh).sum(dim=(0, 1))


def _run_rope(s):
    case = s["case"]
    dt = _TORCH[case["dtype"]]
    if own:
        if case["kind"] == "rope":
            return s["op"].forward(s["q"], s["k"], pos=s["pos"], seq_len=case["seq"])
        return s["op"].backward(s["dq"], s["dk"], s["q"], s["k"], pos=s["pos"], seq_len=case["seq"])
    if case["kind"] == "rope":
        return _rope_forward(s, s["q"], s["wq"]).to(dt), _rope_forward(s, s["k"], s["wk"]).to(dt)
    dq, dwq = _rope_backward(s, s["q"], s["wq"], s["dq"])
    dk, dwk = _rope_backward(s, s["k"], s["wk"], s["dk"])
    return dq.to(dt), dk.to(dt), dwq, dwk


def _run_loss(s):
    case = s["case"]
    tau, grad = case["tau"], case["kind"] == "loss_grad"
    if own:
        from paper_2607_13332_b200 import stage_ops
        if grad:
            return stage_ops.distill_loss_grad(s["logits"], s["ids"], s["top"], s["weight"], temperature=tau)
        return stage_ops.distill_loss(s["logits"], s["ids"], s["top"], s["weight"], temperature=tau)
    x = s["logits"].float() / tau
    m = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(dim=1, keepdim=True)
    there = s["ids"] >= 0
    ids = torch.where(there, s["ids"], 0).long()
    a = torch.where(there, s["top"] / tau, -math.inf)
    am = a.amax(dim=1, keepdim=True)
    rows = there.any(dim=1) & (s["weight"] != 0)
    p = torch.where(there, torch.exp(a - torch.where(am > -math.inf, am, 0.0)), 0.0)
    ptotal = p.sum(dim=1, keepdim=True)
    p = torch.where(ptotal > 0, p / ptotal, 0.0)
    logp = a - am - torch.log(ptotal)
    logq = x.gather(1, ids) - m - torch.log(total)
    per_row = torch.where(there & (p > 0), p * (logp - logq), 0.0).sum(dim=1)
    loss = torch.where(rows, tau * tau * s["weight"] * per_row, 0.0)
    if not grad:
        return loss
    d = e / total
    d.scatter_add_(1, ids, -p)
    d *= torch.where(rows, tau * s["weight"], 0.0)[:, None]
    return loss, d.to(s["logits"].dtype)


def _run_int8(s):
    if own:
        from paper_2607_13332_b200 import stage_ops
        xq, xs = stage_ops.int8_quantize(s["x"])
        return stage_ops.int8_matmul(xq, xs, s["wq"], s["ws"], dtype=s["case"]["dtype"])
    x = s["x"].float()
    scale = x.abs().amax(dim=1, keepdim=True) / 127.0
    q = torch.round(x.double() / scale.double()).float()   # in 64 bits: a quotient beside one half may round either way in 32
    y = q @ s["wq"].float().t()
    return (y * scale * s["ws"]).to(s["x"].dtype)


def run(state):
    kind = state["case"]["kind"]
    return (_run_rope if kind.startswith("rope") else _run_loss if kind.startswith("loss") else _run_int8)(state)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------
def _exact_rope(s):
    """Every pair of columns as a complex number, turned by multiplication with cos + i sin."""
    case = s["case"]
    t, rot, d = case["tokens"], case["rot_dim"], case["head_dim"]
    at = torch.arange(t, device="cuda") % case["seq"] if s["pos"] is None else s["pos"].long()
    row = s["table"].double()[at]
    turn = torch.complex(row[:, :rot // 2], row[:, rot // 2:])[:, None, :]
    cols = torch.arange(rot, device="cuda")
    re, im = (cols[:rot // 2], cols[rot // 2:]) if case["pairing"] == "halves" else (cols[0::2], cols[1::2])

    def turned(x, by):
        y = x.clone()
        z = torch.complex(x[..., re], x[..., im]) * by
        y[..., re], y[..., im] = z.real, z.imag
        return y

    outs, sums = [], []
    for x, w, dy in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        out = torch.empty((t,) + tuple(x.shape[1:]), dtype=torch.float64, device="cuda")
        total = torch.zeros((d,), dtype=torch.float64, device="cuda")
        for lo in range(0, t, 8192):
            hi = min(t, lo + 8192)
            xx, ww, by = x[lo:hi].double(), w.double(), turn[lo:hi]
            norm = torch.sqrt(xx.pow(2).sum(dim=-1, keepdim=True) / d + _EPS)
            unit = xx / norm
            if dy is None:
                out[lo:hi] = turned(unit * ww, by)
                continue
            back = turned(dy[lo:hi].double(), by.conj())
            total += torch.einsum("thd,thd->d", back, unit)
            inner = (back * ww * unit).sum(dim=-1, keepdim=True) / d
            out[lo:hi] = (back * ww - unit * inner) / norm
        outs.append(out)
        sums.append(total)
    return tuple(outs) if case["kind"] == "rope" else tuple(outs + sums)


def _exact_loss(s):
    case = s["case"]
    t, v, tau = case["tokens"], case["vocab"], case["tau"]
    loss = torch.zeros((t,), dtype=torch.float64, device="cuda")
    d = torch.zeros((t, v), dtype=torch.float64, device="cuda") if case["kind"] == "loss_grad" else None
    ids = s["ids"].long()
    for lo in range(0, t, 1024):
        hi = min(t, lo + 1024)
        logq = torch.log_softmax(s["logits"][lo:hi].double() / tau, dim=1)
        # the teacher's distribution over the whole vocabulary: one spare column takes the padding
        full = torch.full((hi - lo, v + 1), -math.inf, dtype=torch.float64, device="cuda")
        full.scatter_(1, torch.where(ids[lo:hi] >= 0, ids[lo:hi], v), s["top"][lo:hi].double() / tau)
        full = full[:, :v]
        on = torch.isfinite(full).any(dim=1) & (s["weight"][lo:hi] != 0)
        logp = torch.log_softmax(torch.where(on[:, None], full, 0.0), dim=1)
        p = logp.exp()
        w = torch.where(on, s["weight"][lo:hi].double(), 0.0)
        loss[lo:hi] = tau * tau * w * torch.where(p > 0, p * (logp - logq), 0.0).sum(dim=1)
        if d is not None:
            d[lo:hi] = tau * w[:, None] * (logq.exp() - p)
    return loss if d is None else (loss, d)


def _exact_int8(s):
    """The quantised values are whole numbers of the scale, which is an fp32 number by definition."""
    y = torch.empty((s["case"]["tokens"], s["case"]["outer"]), dtype=torch.float64, device="cuda")
    top = s["x"].abs().amax(dim=1).float()
    scale = (top / 127.0).double()[:, None]
    q = torch.round(s["x"].double() / scale)
    for lo in range(0, s["case"]["outer"], 16384):
        hi = min(s["case"]["outer"], lo + 16384)
        y[:, lo:hi] = (q @ s["wq"][lo:hi].double().t()) * scale * s["ws"][lo:hi].double()
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    return (_exact_rope if kind.startswith("rope") else _exact_loss if kind.startswith("loss") else _exact_int8)(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], _BYTES[case["dtype"]]
    if kind.startswith("rope"):
        t, d = case["tokens"], case["head_dim"]
        values = t * (case["q_heads"] + case["k_heads"]) * d
        rows = min(t, _MAX_POS if case["positions"] == "packed" else case["seq"])
        small = rows * case["rot_dim"] * 4 + 2 * d * e + (4 * t if case["positions"] == "packed" else 0)
        if kind == "rope":
            return {"bytes": 2 * values * e + small, "flops": 7 * values}
        return {"bytes": 3 * values * e + small + 8 * d, "flops": 16 * values}
    if kind.startswith("loss"):
        t, v, k = case["tokens"], case["vocab"], min(case["top"], case["vocab"])
        passes = 2 if kind == "loss_grad" else 1
        return {"bytes": passes * t * v * e + t * (8 * k + 8), "flops": (4 if passes == 1 else 7) * t * v}
    t, k, n = case["tokens"], case["inner"], case["outer"]
    return {"bytes": t * k * e + n * k + 4 * n + t * n * e, "flops": 2 * t * k * n}
