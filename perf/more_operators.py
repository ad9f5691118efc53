"""Operators at both ends of a language model's training step, and of its update, as cases to be measured.

A worker that trains a language model needs, around the blocks whose operators the library has, the
embedding of its tokens and the loss over the vocabulary with their gradients, and after the
synchronisation the update of its matrices.  Each operator in a plain form (elementary torch
operations in 32 bits, rounded once at the end) and through the library's entry points (``own = True``):

  embed_forward, embed_backward   rows of a table, scaled, for the tokens of a batch; the table's gradient
                                  sums the tokens that share a row, or adds them to a gradient that is
                                  there already (a table that is the output layer too)
  xent_forward, xent_backward     softmax cross entropy of hidden rows against a vocabulary's weights,
                                  without keeping the logits; tokens with a negative target do not count
  orth_update                     a matrix-shaped update orthogonalised by Newton-Schulz products, as the
                                  Muon optimiser does it
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEPS, COEFFICIENTS = 5, (3.4445, -4.7750, 2.0315)


# ------------------------------------------------------------------------------------- cases
def _embed(name, op, tokens, cols, vocab, dtype, accumulate=False):
    return {"name": name, "op": op, "tokens": tokens, "cols": cols, "vocab": vocab, "dtype": dtype, "accumulate": accumulate}


def _xent(name, op, rows, dim, vocab, ignored, penalty=False):
    return {"name": name, "op": op, "rows": rows, "dim": dim, "vocab": vocab, "ignored": ignored, "penalty": penalty}


def _orth(name, batch, rows, cols, dtype):
    return {"name": name, "op": "orth_update", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # one short micro-batch of a small fp32 model: the launch is what counts
        _embed("embed fwd 77x512 f32", "embed_forward", 77, 512, 8000, "f32"),
        # a rank's tokens of one step
        _embed("embed fwd 16384x4096", "embed_forward", 16384, 4096, 50257, "bf16"),
        # a micro-batch of odd length and width in fp32
        _embed("embed bwd 999x500 f32", "embed_backward", 999, 500, 8001, "f32"),
        # a rank's step with a table that is the output layer too: added to the gradient that the loss left
        _embed("embed bwd add 16384x2048", "embed_backward", 16384, 2048, 50257, "bf16", True),
        # evaluating the loss of one short sentence: the vocabulary's weights are read once, little else happens
        _xent("xent fwd 24x512 v32000", "xent_forward", 24, 512, 32000, 0.0),
        # a fine-tuning batch, whose prompts do not count, on a vocabulary of odd size
        _xent("xent fwd 4096x2048 v50257 masked", "xent_forward", 4096, 2048, 50257, 0.4),
        # a rank's step of a large model
        _xent("xent fwd 8192x4096 v65536", "xent_forward", 8192, 4096, 65536, 0.0),
        # a short ragged micro-batch of a small model
        _xent("xent bwd 200x768 v8001", "xent_backward", 200, 768, 8001, 0.1),
        # an ordinary batch, with a penalty on the logarithm of the sum too
        _xent("xent bwd 4096x1024 v50257", "xent_backward", 4096, 1024, 50257, 0.05, True),
        # a rank's step of a large model
        _xent("xent bwd 8192x4096 v65536", "xent_backward", 8192, 4096, 65536, 0.0),
        # a small model's projection: a chain of short products
        _orth("orth 256x384 f32", 1, 256, 384, "f32"),
        # the four hidden matrices of a group of layers
        _orth("orth 4x4096x2048", 4, 4096, 2048, "bf16"),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], uniform in its logarithm."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(("embed_forward", "embed_backward", "xent_forward", "xent_backward", "orth_update"))
    if op.startswith("embed"):
        cols = _spread(rng, 16, 4096)
        if rng.random() < 0.6:
            cols = -(-cols // 8) * 8
        case = _embed("", op, _spread(rng, 1, 16384), cols, _spread(rng, 100, 50257), rng.choice(("f32", "bf16", "bf16")),
                      op == "embed_backward" and rng.random() < 0.4)
    elif op.startswith("xent"):
        case = _xent("", op, _spread(rng, 1, 8192), 8 * _spread(rng, 4, 512), _spread(rng, 2, 65536), rng.choice((0.0, 0.0, 0.1, 0.5)),
                     op == "xent_backward" and rng.random() < 0.3)
    else:
        rows, cols = _spread(rng, 1, 4096), _spread(rng, 1, 4096)
        room = max(1, 4 * 4096 * 2048 * 2048 // (rows * cols * min(rows, cols)))
        case = _orth("", _spread(rng, 1, min(8, room)), rows, cols, rng.choice(("f32", "bf16")))
        if rows * cols * min(rows, cols) > 4 * 4096 * 2048 * 2048:
            case["rows"], case["cols"] = min(rows, 2048), min(cols, 4096)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------ inputs
def _tokens(case, count, gen, device):
    """Ids as a text has them: the commonest take a good part, most of the vocabulary is rare; one in
    fifty is padding."""
    u = torch.rand(count, device=device, generator=gen, dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["vocab"])) - 1.0).long().clamp_(0, case["vocab"] - 1)
    order = torch.randperm(case["vocab"], device=device, generator=gen)       # common tokens lie anywhere in the table
    ids = order[ids]
    return torch.where(torch.rand(count, device=device, generator=gen) < 0.02, -1, ids)


def prepare(case, seed):
    """Inputs of the path on the GPU, and the buffers that a training loop keeps from step to step."""
    device = torch.device("cuda")
    gen = torch.Generator(device).manual_seed(int(seed))

    def normal(*shape, dtype=torch.float32, std=1.0):
        return (torch.randn(*shape, device=device, generator=gen) * std).to(dtype)

    s = {"case": dict(case)}
    if own:
        from paper_2505_10183_b200 import binding as kt
    if case["op"].startswith("embed"):
        dtype = TYPES[case["dtype"]]
        s["ids"] = _tokens(case, case["tokens"], gen, device)
        s["scale"] = math.sqrt(case["cols"])
        if case["op"] == "embed_forward":
            s["weight"] = normal(case["vocab"], case["cols"], dtype=dtype, std=case["cols"] ** -0.5)
            s["out"] = torch.empty(case["tokens"], case["cols"], dtype=dtype, device=device)
        else:
            s["dout"] = normal(case["tokens"], case["cols"], dtype=dtype, std=0.01)
            s["before"] = normal(case["vocab"], case["cols"], dtype=dtype, std=0.1) if case["accumulate"] else None
            s["dweight"] = torch.empty(case["vocab"], case["cols"], dtype=dtype, device=device)
            if own:
                s["work"] = torch.empty(kt.kt_embed_workspace(case["tokens"], case["cols"], case["vocab"]), dtype=torch.uint8, device=device)
    elif case["op"].startswith("xent"):
        N, D, V = case["rows"], case["dim"], case["vocab"]
        bf16 = torch.bfloat16
        s["hidden"], s["weight"] = normal(N, D, dtype=bf16), normal(V, D, dtype=bf16, std=1.5 * D ** -0.5)
        targets = torch.randint(V, (N,), device=device, generator=gen)
        s["targets"] = torch.where(torch.rand(N, device=device, generator=gen) < case["ignored"], -100, targets)
        s["loss"], s["lse"] = torch.empty(N, device=device), torch.empty(N, device=device)
        if case["op"] == "xent_backward":
            s["loss"], s["lse"] = _xent_forward(s)               # what the forward pass has left
            counted = (s["targets"] >= 0).sum().clamp(min=1)
            s["dloss"] = torch.full((N,), 1.0, device=device) / counted
            s["dlse"] = 2e-4 * s["lse"] / counted if case["penalty"] else None
            s["dhidden"], s["dweight"] = torch.empty_like(s["hidden"]), torch.empty_like(s["weight"])
        if own:
            s["work"] = torch.empty(kt.kt_xent_workspace(N, D, V, case["op"] == "xent_backward"), dtype=torch.uint8, device=device)
    else:
        shape = (case["batch"], case["rows"], case["cols"])
        # a gradient's momentum: a few strong directions above noise
        strong = torch.bmm(normal(shape[0], shape[1], 8), normal(shape[0], 8, shape[2])) / 8.0
        s["x"] = (1e-3 * (strong + normal(*shape))).to(TYPES[case["dtype"]])
        s["scale"] = max(1.0, case["rows"] / case["cols"]) ** 0.5
        s["out"] = torch.empty(shape, dtype=torch.bfloat16, device=device)
        if own:
            s["work"] = torch.empty(kt.kt_orth_workspace(*shape), dtype=torch.uint8, device=device)
    return s


# -------------------------------------------------------------------------------- plain forms
def _embed_forward(s):
    rows = s["weight"][s["ids"].clamp(min=0)].float() * s["scale"]
    return torch.where(s["ids"][:, None] >= 0, rows, 0.0).to(s["weight"].dtype)


def _embed_backward(s):
    used = s["ids"] >= 0
    sums = torch.zeros(s["dweight"].shape, device=s["ids"].device)
    sums.index_add_(0, s["ids"].clamp(min=0), torch.where(used[:, None], s["dout"].float(), 0.0))
    sums = sums * s["scale"]
    return (sums if s["before"] is None else s["before"].float() + sums).to(s["dweight"].dtype)


def _logits(s):
    return s["hidden"].float() @ s["weight"].float().t()


def _xent_forward(s):
    logits, used = _logits(s), s["targets"] >= 0
    top = logits.amax(1)
    at = logits.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0]
    lse = top + torch.log(logits.sub_(top[:, None]).exp_().sum(1))
    return torch.where(used, lse - at, 0.0), torch.where(used, lse, 0.0)


def _xent_backward(s):
    used = s["targets"] >= 0
    dloss = torch.where(used, s["dloss"], 0.0)
    both = dloss if s["dlse"] is None else dloss + torch.where(used, s["dlse"], 0.0)
    grad = _logits(s).sub_(s["lse"][:, None]).exp_().mul_(both[:, None])
    grad = torch.where(used[:, None], grad, 0.0)
    grad[torch.arange(grad.shape[0], device=grad.device), s["targets"].clamp(min=0)] -= dloss
    return (grad @ s["weight"].float()).to(torch.bfloat16), (grad.t() @ s["hidden"].float()).to(torch.bfloat16)


def _orth_update(s):
    a, b, c = COEFFICIENTS
    x = s["x"].float()
    x = x / x.square().sum((1, 2), keepdim=True).sqrt()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    if tall:
        x = x.transpose(1, 2)
    return (x * s["scale"]).to(torch.bfloat16)


def _plain(s):
    op = s["case"]["op"]
    if op == "embed_forward":
        return {"out": _embed_forward(s)}
    if op == "embed_backward":
        return {"dweight": _embed_backward(s)}
    if op == "xent_forward":
        return dict(zip(("loss", "lse"), _xent_forward(s)))
    if op == "xent_backward":
        return dict(zip(("dhidden", "dweight"), _xent_backward(s)))
    return {"out": _orth_update(s)}


def _own(s):
    from paper_2505_10183_b200 import binding as kt

    op = s["case"]["op"]
    if op == "embed_forward":
        kt.kt_embed_forward(s["ids"], s["weight"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "embed_backward":
        kt.kt_embed_backward(s["dout"], s["ids"], s["dweight"], s["work"], scale=s["scale"], base=s["before"])
        return {"dweight": s["dweight"]}
    if op == "xent_forward":
        kt.kt_xent_forward(s["hidden"], s["weight"], s["targets"], s["loss"], s["lse"], s["work"])
        return {"loss": s["loss"], "lse": s["lse"]}
    if op == "xent_backward":
        kt.kt_xent_backward(s["dloss"], s["hidden"], s["weight"], s["targets"], s["lse"], s["dhidden"], s["dweight"], s["work"],
                            dlse=s["dlse"])
        return {"dhidden": s["dhidden"], "dweight": s["dweight"]}
    kt.kt_orth_update(s["x"], s["out"], s["work"], steps=STEPS, coefficients=COEFFICIENTS, scale=s["scale"])
    return {"out": s["out"]}


def run(state):
    return _own(state) if own else _plain(state)


# -------------------------------------------------------------------------------------- work
def work(case):
    if case["op"].startswith("embed"):
        size = 4 if case["dtype"] == "f32" else 2
        tokens, table = case["tokens"] * case["cols"] * size, case["vocab"] * case["cols"] * size
        if case["op"] == "embed_forward":            # no row of the table has to be read twice
            return {"bytes": tokens + min(tokens, table) + 8 * case["tokens"], "flops": case["tokens"] * case["cols"]}
        return {"bytes": tokens + 8 * case["tokens"] + table * (2 if case["accumulate"] else 1), "flops": 2 * case["tokens"] * case["cols"]}
    if case["op"].startswith("xent"):
        V, D = case["vocab"], case["dim"]
        N = case["rows"] * (1.0 - case["ignored"])
        inputs = 2 * (N * D + V * D) + 16 * case["rows"]
        if case["op"] == "xent_forward":
            return {"bytes": int(inputs), "flops": int(2 * N * V * D)}
        return {"bytes": int(2 * inputs), "flops": int(6 * N * V * D)}
    m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": case["batch"] * m * n * (size + 2), "flops": case["batch"] * STEPS * (3 * m * m * n + m * m * m)}


# --------------------------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "embed_forward":
        table = torch.cat((f["weight"], torch.zeros_like(f["weight"][:1])))        # padding reads the row of zeros
        return {"out": s["scale"] * table.index_select(0, s["ids"] % (case["vocab"] + 1))}
    if case["op"] == "embed_backward":
        order = torch.argsort(s["ids"], stable=True)
        ids, rows = s["ids"][order], f["dout"][order]
        first = torch.ones_like(ids, dtype=torch.bool)
        first[1:] = ids[1:] != ids[:-1]
        starts = torch.nonzero(first)[:, 0]
        lengths = torch.diff(starts, append=torch.tensor([len(ids)], device=ids.device))
        sums = torch.segment_reduce(rows, "sum", lengths=lengths, axis=0)
        out = f["before"].clone() if s["before"] is not None else torch.zeros(case["vocab"], case["cols"], dtype=torch.float64, device=ids.device)
        real = ids[starts] >= 0
        out[ids[starts][real]] += s["scale"] * sums[real]
        return {"dweight": out}
    if case["op"].startswith("xent"):
        counted = torch.nonzero(s["targets"] >= 0)[:, 0]
        targets, hidden = s["targets"][counted], f["hidden"][counted]
        outs = [torch.zeros(case["rows"], dtype=torch.float64, device=counted.device) for _ in range(2)]
        dhidden, dweight = torch.zeros_like(f["hidden"]), torch.zeros_like(f["weight"])
        for i in range(0, len(counted), 2048):
            at, t, h = counted[i:i + 2048], targets[i:i + 2048, None], hidden[i:i + 2048]
            logp = torch.einsum("nd,vd->nv", h, f["weight"])
            if case["op"] == "xent_forward":
                lse = torch.logsumexp(logp, 1)
                outs[0][at], outs[1][at] = lse - torch.take_along_dim(logp, t, 1)[:, 0], lse
                continue
            # the saved logarithms are inputs of the backward pass, as they are
            logp.sub_(f["lse"][at][:, None]).exp_()
            if s["dlse"] is not None:
                logp.mul_((1.0 + f["dlse"][at] / f["dloss"][at])[:, None])
            logp.scatter_add_(1, t, torch.full_like(t, -1.0, dtype=torch.float64)).mul_(f["dloss"][at][:, None])
            dhidden[at] = torch.einsum("nv,vd->nd", logp, f["weight"])
            dweight += torch.einsum("nv,nd->vd", logp, h)
        return {"loss": outs[0], "lse": outs[1]} if case["op"] == "xent_forward" else {"dhidden": dhidden, "dweight": dweight}
    a, b, c = COEFFICIENTS
    y = f["x"] / torch.linalg.matrix_norm(f["x"], keepdim=True)
    left = case["rows"] <= case["cols"]
    for _ in range(STEPS):                                       # the polynomial of the shorter side's Gram matrix
        gram = torch.einsum("bij,bkj->bik", y, y) if left else torch.einsum("bji,bjk->bik", y, y)
        factor = torch.einsum("bij,bjk->bik", gram, c * gram + b * torch.eye(gram.shape[1], dtype=gram.dtype, device=gram.device))
        factor.diagonal(dim1=1, dim2=2).add_(a)
        y = torch.einsum("bij,bjk->bik", factor, y) if left else torch.einsum("bij,bjk->bik", y, factor)
    return {"out": s["scale"] * y}
