"""The training operators beside the gradient synchronisation, as cases to be measured.

A data-parallel worker computes the gradients that the library synchronises.  Three families of
operators are measured here, each in a plain form (elementary torch operations in 32 bits,
rounded once at the end) and through the library's entry points (``own = True``):

  norm_forward, norm_backward   layer norm over rows, optionally with the normalised rows kept in
                                8 bits and the backward pass reading them; the weight's and the
                                bias' gradients are reduced over all rows
  act_forward, act_backward     GELU or SiLU that keeps its input in 8 bits for the backward pass
  attn_forward, attn_backward   softmax attention with shared key/value heads, causal masks and
                                sequences of different lengths in one batch; the backward pass
                                recomputes the probabilities from the saved logarithms of the sums

Checkpoints in 8 bits hold signed codes -127 ... 127 with one fp32 scale per 128 columns of a row.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128                # columns of a row that share a scale
SMALLEST = 2.0 ** -100     # a block whose largest magnitude is below this is kept as zeros
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------- cases
def _norm(name, op, rows, cols, dtype, keep):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "keep": keep}


def _act(name, op, rows, cols, dtype, kind):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "kind": kind}


def _attn(name, op, batch, len_q, len_kv, heads, heads_kv, dim, causal, ragged):
    return {"name": name, "op": op, "batch": batch, "len_q": len_q, "len_kv": len_kv, "heads": heads,
            "heads_kv": heads_kv, "dim": dim, "causal": causal, "ragged": ragged}


def listed():
    return [
        # one short micro-batch of a small fp32 model: the launch is what counts
        _norm("norm fwd 64x512 f32", "norm_forward", 64, 512, "f32", False),
        # a rank's tokens of one step in bf16, normalised rows kept in 8 bits for the backward pass
        _norm("norm fwd keep 16384x4096", "norm_forward", 16384, 4096, "bf16", True),
        # an odd number of tokens, a width that is no power of two
        _norm("norm bwd 4999x1000 f32", "norm_backward", 4999, 1000, "f32", False),
        # the same step's backward pass from the rows themselves
        _norm("norm bwd 16384x4096", "norm_backward", 16384, 4096, "bf16", False),
        # a backward pass that reads the 8-bit rows instead
        _norm("norm bwd kept 16384x2048", "norm_backward", 16384, 2048, "bf16", True),
        # the hidden activation of a small micro-batch
        _act("gelu fwd 128x2048", "act_forward", 128, 2048, "bf16", "gelu"),
        # the hidden activation of a rank's step: the largest tensor that a block keeps
        _act("gelu bwd 16384x8192", "act_backward", 16384, 8192, "bf16", "gelu"),
        # short sentences of different lengths in one batch, an odd padded length, heads of 80
        _attn("attn fwd 4x333 h12/4 d80", "attn_forward", 4, 333, 333, 12, 4, 80, True, True),
        # one long sequence, four query heads to a key/value head
        _attn("attn fwd 1x8192 h16/4 d128", "attn_forward", 1, 8192, 8192, 16, 4, 128, True, False),
        # a small micro-batch of ragged sequences
        _attn("attn bwd 2x200 h4/2 d64", "attn_backward", 2, 200, 200, 4, 2, 64, False, True),
        # an ordinary training batch
        _attn("attn bwd 8x1024 h16 d64", "attn_backward", 8, 1024, 1024, 16, 16, 64, True, False),
        # one long sequence, four query heads to a key/value head
        _attn("attn bwd 1x8192 h16/4 d128", "attn_backward", 1, 8192, 8192, 16, 4, 128, True, False),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], uniform in its logarithm."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(("norm_forward", "norm_backward", "act_forward", "act_backward", "attn_forward", "attn_backward"))
    if op.startswith("attn"):
        dim = rng.choice((64, 64, 128, 128, 8 * rng.randint(2, 16)))
        heads_kv = rng.choice((1, 2, 3, 4, 8))
        heads = heads_kv * rng.choice((1, 1, 2, 4))
        len_q = _spread(rng, 1, 8192)
        len_kv = len_q if rng.random() < 0.7 else _spread(rng, 1, 8192)
        room = 8 * 8192 * 8192 // (heads * len_q * len_kv)       # half of the largest listed case
        while room < 1:
            len_q, len_kv = (len_q + 1) // 2, (len_kv + 1) // 2
            room = 8 * 8192 * 8192 // (heads * len_q * len_kv)
        batch = _spread(rng, 1, min(16, room))
        case = _attn("", op, batch, len_q, len_kv, heads, heads_kv, dim, rng.random() < 0.6, rng.random() < 0.4)
    else:
        cols = _spread(rng, 16, 8192)
        if rng.random() < 0.6:
            cols = -(-cols // 8) * 8
        rows = _spread(rng, 1, 16384)
        dtype = rng.choice(("f32", "bf16", "bf16"))
        if op.startswith("norm"):
            case = _norm("", op, rows, cols, dtype, rng.random() < 0.5)
        else:
            case = _act("", op, rows, cols, dtype, rng.choice(("gelu", "silu")))
    del case["name"]
    return case


# ------------------------------------------------------------------------------------ inputs
def _blocks(cols):
    return -(-cols // BLOCK)


def _pitch(cols):
    return -(-cols // 16) * 16


def _lengths(case, device):
    """Tokens in use of every sequence: the longest fills the batch, the others are shorter."""
    if not case["ragged"]:
        return None, None
    part = torch.linspace(1.0, 0.3, case["batch"], dtype=torch.float64)
    used = [torch.clamp((part * case[k]).to(torch.int32), min=1).to(device) for k in ("len_q", "len_kv")]
    return used[0], used[1]


def prepare(case, seed):
    """Inputs of the path on the GPU, and the buffers that a training loop keeps from step to step."""
    device = torch.device("cuda")
    gen = torch.Generator(device).manual_seed(int(seed))

    def normal(*shape, dtype=torch.float32, std=1.0, mean=0.0):
        return (torch.randn(*shape, device=device, generator=gen) * std + mean).to(dtype)

    s = {"case": dict(case)}
    if case["op"].startswith("attn"):
        B, Lq, Lk, H, Hk, D = (case[k] for k in ("batch", "len_q", "len_kv", "heads", "heads_kv", "dim"))
        bf16 = torch.bfloat16
        s["q"], s["k"], s["v"] = normal(B, Lq, H, D, dtype=bf16), normal(B, Lk, Hk, D, dtype=bf16), normal(B, Lk, Hk, D, dtype=bf16)
        s["scale"] = 1.0 / math.sqrt(D)
        s["used_q"], s["used_kv"] = _lengths(case, device)
        s["out"] = torch.empty(B, Lq, H, D, dtype=bf16, device=device)
        s["lse"] = torch.empty(B, H, Lq, device=device)
        if case["op"] == "attn_backward":
            s["dout"] = normal(B, Lq, H, D, dtype=bf16)
            s["out"], s["lse"] = _attn_forward(s)                # what the forward pass has left
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[k]) for k in ("q", "k", "v"))
        return s
    rows, cols, dtype = case["rows"], case["cols"], TYPES[case["dtype"]]
    s["codes"] = torch.zeros(rows, _pitch(cols), dtype=torch.int8, device=device)
    s["scales"] = torch.zeros(rows, _blocks(cols), device=device)
    s["kept"] = torch.empty(rows, cols, dtype=torch.bfloat16, device=device)      # what matrix products read
    s["x"] = normal(rows, cols, dtype=dtype, std=1.5, mean=0.2)
    s["out"] = torch.empty_like(s["x"])
    if case["op"].startswith("norm"):
        s["weight"], s["bias"] = normal(cols, std=0.2, mean=1.0), normal(cols, std=0.1)
        s["mean"], s["rstd"] = torch.empty(rows, device=device), torch.empty(rows, device=device)
        if case["op"] == "norm_backward":
            s["dout"] = normal(rows, cols, dtype=dtype)
            x = s["x"].float()
            s["mean"], s["rstd"] = _moments(x)
            if case["keep"]:
                s["codes"][:, :cols], s["scales"] = _encode((x - s["mean"][:, None]) * s["rstd"][:, None])
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
    elif case["op"] == "act_backward":
        s["dout"] = normal(rows, cols, dtype=dtype)
        s["codes"][:, :cols], s["scales"] = _encode(s["x"].float())
        s["dx"] = torch.empty_like(s["x"])
    return s


# -------------------------------------------------------------------------------- plain forms
def _encode(x):
    """Codes (int8) and scales of x (fp32): per 128 columns of a row, the largest magnitude is 127."""
    rows, cols = x.shape
    blocks = torch.nn.functional.pad(x, (0, _blocks(cols) * BLOCK - cols)).view(rows, -1, BLOCK)
    top = blocks.abs().amax(2)
    used = top >= SMALLEST
    per_unit = torch.where(used, 127.0 * (1.0 / torch.where(used, top, 1.0)), 0.0)
    codes = torch.round(blocks * per_unit[:, :, None]).to(torch.int8)
    return codes.view(rows, -1)[:, :cols], torch.where(used, top * (1.0 / 127.0), 0.0)


def _decode(codes, scales, cols):
    """The values that codes and scales stand for (fp32)."""
    return codes[:, :cols].float() * scales.repeat_interleave(BLOCK, 1)[:, :cols]


def _moments(x):
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, 1.0 / torch.sqrt(var + EPS)


def _norm_forward(s):
    x, dtype = s["x"].float(), s["x"].dtype
    mean, rstd = _moments(x)
    unit = (x - mean[:, None]) * rstd[:, None]
    got = {"out": (unit * s["weight"] + s["bias"]).to(dtype), "mean": mean, "rstd": rstd}
    if s["case"]["keep"]:
        got["kept"] = _decode(*_encode(unit), unit.shape[1]).to(torch.bfloat16)
    return got


def _norm_backward(s):
    dout = s["dout"].float()
    if s["case"]["keep"]:
        unit = _decode(s["codes"], s["scales"], dout.shape[1])
    else:
        unit = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dout * s["weight"]
    dx = (g - g.mean(1, keepdim=True) - unit * (g * unit).mean(1, keepdim=True)) * s["rstd"][:, None]
    return {"dx": dx.to(s["dout"].dtype), "dweight": (dout * unit).sum(0), "dbias": dout.sum(0)}


def _act_forward(s):
    x = s["x"].float()
    y = x * 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) if s["case"]["kind"] == "gelu" else x / (1.0 + torch.exp(-x))
    return {"out": y.to(s["x"].dtype), "kept": _decode(*_encode(x), x.shape[1]).to(torch.bfloat16)}


def _act_backward(s):
    x = _decode(s["codes"], s["scales"], s["dout"].shape[1])
    if s["case"]["kind"] == "gelu":
        slope = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    else:
        gate = 1.0 / (1.0 + torch.exp(-x))
        slope = gate * (1.0 + x * (1.0 - gate))
    return {"dx": (s["dout"].float() * slope).to(s["dout"].dtype)}


def _seen(s):
    """Which keys a query sees, as truth values [batch or 1, 1, len_q, len_kv]; and the queries in use."""
    case, device = s["case"], s["q"].device
    i = torch.arange(case["len_q"], device=device).view(1, 1, -1, 1)
    j = torch.arange(case["len_kv"], device=device).view(1, 1, 1, -1)
    used_q = torch.full((1,), case["len_q"], device=device) if s["used_q"] is None else s["used_q"]
    used_kv = torch.full((1,), case["len_kv"], device=device) if s["used_kv"] is None else s["used_kv"]
    used_q, used_kv = used_q.view(-1, 1, 1, 1), used_kv.view(-1, 1, 1, 1)
    seen = (i < used_q) & (j < used_kv)
    return seen & (j <= i + used_kv - used_q) if case["causal"] else seen


def _heads_first(x, heads):
    """[batch, tokens, heads or a divisor, dim] as fp32 [batch, heads, tokens, dim]."""
    return x.float().transpose(1, 2).repeat_interleave(heads // x.shape[2], 1)


def _attn_forward(s):
    H = s["case"]["heads"]
    q, k, v = (_heads_first(s[n], H) for n in ("q", "k", "v"))
    scores = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~_seen(s), -math.inf)
    top = scores.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    scores.sub_(top).exp_()
    total = scores.sum(3, keepdim=True)
    out = torch.matmul(scores, v) / torch.where(total == 0, 1.0, total)
    return out.transpose(1, 2).to(s["q"].dtype).contiguous(), (top + torch.log(total)).squeeze(3)


def _attn_backward(s):
    case = s["case"]
    B, Lk, H, Hk, D = case["batch"], case["len_kv"], case["heads"], case["heads_kv"], case["dim"]
    q, k, v, out, dout = (_heads_first(s[n], H) for n in ("q", "k", "v", "out", "dout"))
    probs = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).sub_(s["lse"][..., None]).exp_().masked_fill_(~_seen(s), 0.0)
    dv = torch.matmul(probs.transpose(2, 3), dout)
    dscores = torch.matmul(dout, v.transpose(2, 3)).sub_((dout * out).sum(3, keepdim=True)).mul_(probs).mul_(s["scale"])
    dq, dk = torch.matmul(dscores, k), torch.matmul(dscores.transpose(2, 3), q)
    dk, dv = (g.view(B, Hk, H // Hk, Lk, D).sum(2) for g in (dk, dv))
    return {n: g.transpose(1, 2).to(s["q"].dtype).contiguous() for n, g in (("dq", dq), ("dk", dk), ("dv", dv))}


# ----------------------------------------------------------------------------- the library's own
def _run_own(s):
    from paper_2505_10183_b200 import binding as kt
    case = s["case"]
    op = case["op"]
    if op == "norm_forward":
        keep = {"codes": s["codes"], "scales": s["scales"]} if case["keep"] else {}
        kt.kt_norm_forward(s["x"], s["weight"], s["bias"], s["out"], s["mean"], s["rstd"], EPS, **keep)
        got = {"out": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
        if case["keep"]:
            kt.kt_ckpt_restore(s["codes"], s["scales"], s["kept"])
            got["kept"] = s["kept"]
        return got
    if op == "norm_backward":
        source = {"codes": s["codes"], "scales": s["scales"]} if case["keep"] else {"x": s["x"], "mean": s["mean"]}
        work = torch.empty(kt.kt_norm_workspace(case["rows"], case["cols"]), dtype=torch.uint8, device="cuda")
        kt.kt_norm_backward(s["dout"], s["weight"], s["rstd"], s["dx"], s["dweight"], s["dbias"], work, **source)
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if op == "act_forward":
        kt.kt_act_forward(s["x"], s["out"], s["codes"], s["scales"], case["kind"])
        kt.kt_ckpt_restore(s["codes"], s["scales"], s["kept"])
        return {"out": s["out"], "kept": s["kept"]}
    if op == "act_backward":
        kt.kt_act_backward(s["dout"], s["codes"], s["scales"], s["dx"], case["kind"])
        return {"dx": s["dx"]}
    mask = {"scale": s["scale"], "causal": case["causal"], "used_q": s["used_q"], "used_kv": s["used_kv"]}
    if op == "attn_forward":
        kt.kt_attn_forward(s["q"], s["k"], s["v"], s["out"], s["lse"], **mask)
        return {"out": s["out"], "lse": s["lse"]}
    work = torch.empty(kt.kt_attn_workspace(s["q"], s["k"]), dtype=torch.uint8, device="cuda")
    kt.kt_attn_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dq"], s["dk"], s["dv"], work, **mask)
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


_PLAIN = {"norm_forward": _norm_forward, "norm_backward": _norm_backward, "act_forward": _act_forward,
          "act_backward": _act_backward, "attn_backward": _attn_backward,
          "attn_forward": lambda s: dict(zip(("out", "lse"), _attn_forward(s)))}


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------- work
def _pairs(case):
    """Query-key pairs of one head over the batch that the mask leaves."""
    used_q, used_kv = _lengths(case, "cpu")
    lens_q = [case["len_q"]] * case["batch"] if used_q is None else used_q.tolist()
    lens_kv = [case["len_kv"]] * case["batch"] if used_kv is None else used_kv.tolist()
    total = 0
    for n, m in zip(lens_q, lens_kv):
        if not case["causal"]:
            total += n * m
        else:                                   # query i sees min(m, max(0, i + 1 + m - n)) keys
            first = max(0, n - m)               # queries before it see nothing
            low = 1 + m - n + first
            total += (n - first) * (low + m) // 2
    return total


def work(case):
    if case["op"].startswith("attn"):
        B, Lq, Lk, H, Hk, D = (case[k] for k in ("batch", "len_q", "len_kv", "heads", "heads_kv", "dim"))
        q, kv, stats = 2 * B * Lq * H * D, 2 * B * Lk * Hk * D, 4 * B * H * Lq
        product = 2 * _pairs(case) * H * D
        if case["op"] == "attn_forward":
            return {"bytes": 2 * q + 2 * kv + stats, "flops": 2 * product}
        return {"bytes": 4 * q + 4 * kv + stats, "flops": 5 * product}
    rows, cols = case["rows"], case["cols"]
    size = 4 if case["dtype"] == "f32" else 2
    full, kept = rows * cols * size, rows * (cols + 4 * _blocks(cols))
    if case["op"] == "norm_forward":            # keeping: codes written, read again and restored
        return {"bytes": 2 * full + 8 * cols + 8 * rows + (2 * kept + 2 * rows * cols if case["keep"] else 0), "flops": 8 * rows * cols}
    if case["op"] == "norm_backward":
        source = kept + 4 * rows if case["keep"] else full + 8 * rows
        return {"bytes": 2 * full + source + 12 * cols, "flops": 12 * rows * cols}
    if case["op"] == "act_forward":
        return {"bytes": 2 * full + 2 * kept + 2 * rows * cols, "flops": 12 * rows * cols}
    return {"bytes": 2 * full + kept, "flops": 14 * rows * cols}


# --------------------------------------------------------------------------------------- exact
def _exact_norm(s, case):
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"] == "norm_forward":
        var, mean = torch.var_mean(f["x"], 1, correction=0)
        rstd = (var + EPS) ** -0.5
        out = torch.addcmul(f["bias"], (f["x"] - mean[:, None]) * rstd[:, None], f["weight"])
        return {"out": out, "mean": mean, "rstd": rstd, **({"kept": None} if case["keep"] else {})}
    n = case["cols"]
    if case["keep"]:
        at = torch.arange(n, device=f["codes"].device)
        unit = f["codes"][:, :n] * f["scales"][:, at // BLOCK]
    else:
        unit = (f["x"] - f["mean"][:, None]) * f["rstd"][:, None]
    # y = w u + b with u = (x - m(x)) r(x): J^T of u applied to w dy, column by column summed for w and b
    g = f["dout"] * f["weight"]
    along = torch.einsum("rc,rc->r", g, unit) / n
    dx = f["rstd"][:, None] * (g - (g.sum(1) / n)[:, None] - along[:, None] * unit)
    return {"dx": dx, "dweight": torch.einsum("rc,rc->c", f["dout"], unit), "dbias": torch.einsum("rc->c", f["dout"])}


def _exact_act(s, case):
    n = case["cols"]
    if case["op"] == "act_forward":
        x = s["x"].double()
        gate = torch.special.ndtr(x) if case["kind"] == "gelu" else torch.sigmoid(x)
        return {"out": x * gate, "kept": None}                # rounding to a code has no value in more bits
    at = torch.arange(n, device=s["codes"].device) // BLOCK
    x = s["codes"][:, :n].double() * s["scales"].double()[:, at]
    if case["kind"] == "gelu":
        slope = torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / (2 * math.pi) ** 0.5
    else:
        slope = torch.sigmoid(x) + x * torch.sigmoid(x) * torch.sigmoid(-x)
    return {"dx": s["dout"].double() * slope}


def _exact_attn(s, case):
    """Head group by head group: [batch, kv head, query head of the group, token, dim]."""
    B, Lq, Lk, H, Hk, D = (case[k] for k in ("batch", "len_q", "len_kv", "heads", "heads_kv", "dim"))
    split = lambda x: x.double().view(B, -1, Hk, x.shape[2] // Hk, D).permute(0, 2, 3, 1, 4)  # noqa: E731
    merge = lambda x: x.permute(0, 3, 1, 2, 4).reshape(B, x.shape[3], -1, D)  # noqa: E731
    q, k, v = split(s["q"]), split(s["k"]), split(s["v"])
    device = q.device
    n = s["used_q"].long() if s["used_q"] is not None else torch.full((B,), Lq, device=device)
    m = s["used_kv"].long() if s["used_kv"] is not None else torch.full((B,), Lk, device=device)
    at_q, at_k = torch.arange(Lq, device=device), torch.arange(Lk, device=device)
    last = (m[:, None] - 1).expand(B, Lq)                     # the last key that a query sees
    if case["causal"]:
        last = torch.minimum(last, at_q[None, :] + (m - n)[:, None])
    last = torch.where(at_q[None, :] < n[:, None], last, -1)
    hidden = (at_k[None, None, :] > last[:, :, None])[:, None, None]
    scores = torch.einsum("bgrid,bgsjd->bgrij", q, k).mul_(s["scale"]).masked_fill_(hidden, -math.inf)
    if case["op"] == "attn_forward":
        lse = torch.logsumexp(scores, -1)
        probs = scores.sub_(lse[..., None]).exp_().nan_to_num_(nan=0.0)      # an empty row: -inf - -inf
        return {"out": merge(torch.einsum("bgrij,bgsjd->bgrid", probs, v)), "lse": lse.reshape(B, H, Lq)}
    # the saved output and logarithms are inputs of the backward pass, as they are
    lse = s["lse"].double().view(B, Hk, H // Hk, Lq, 1)
    probs = scores.sub_(lse).exp_().nan_to_num_(nan=0.0)
    dout, out = split(s["dout"]), split(s["out"])
    dv = torch.einsum("bgrij,bgrid->bgjd", probs, dout)[:, :, None]
    dprobs = torch.einsum("bgrid,bgsjd->bgrij", dout, v)
    dscores = dprobs.sub_(torch.einsum("bgrid,bgrid->bgri", dout, out)[..., None]).mul_(probs).mul_(s["scale"])
    dq = torch.einsum("bgrij,bgsjd->bgrid", dscores, k)
    dk = torch.einsum("bgrij,bgrid->bgjd", dscores, q)[:, :, None]
    return {"dq": merge(dq), "dk": merge(dk), "dv": merge(dv)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("attn"):
        return _exact_attn(s, case)
    return (_exact_norm if case["op"].startswith("norm") else _exact_act)(s, case)
