"""A training step of a small language model on simulated ranks of unequal speed, from token ids to updated matrices:

    python -m paper_2505_10183_b200.language_step [--tokens 512] [--width 1024] [--layers 2] [--vocab 32000] [--steps 5]

Around the blocks of block_step.py: the embedding of the tokens, a last layer norm, and the cross entropy of its rows
against the embedding's table, which is the output layer too (no logits are kept, and the embedding's gradient is added
to what the loss leaves).  The ranks' gradients are combined with the shares' weights in one pass
(kt_sync_direct) and compared with those of the whole batch from a plain fp32 model; the blocks' matrices then take
a step along their orthogonalised momentum, all layers' matrices of a shape in one call.
"""
from __future__ import annotations

import argparse
from typing import Dict, List, Tuple

import torch

from . import binding as kt
from .block_step import NAMES, Block, Shape, _Kept
from .block_step import parameters as block_parameters

MATRICES = ("qkv", "proj", "up", "down")


def names(layers: int) -> List[str]:
    return ["embed", "norm.weight", "norm.bias"] + ["%d.%s" % (i, n) for i in range(layers) for n in NAMES]


def parameters(shape: Shape, layers: int, vocab: int, seed: int, device="cuda") -> Dict[str, torch.Tensor]:
    """bf16 parameters: the table (tokens in, logits out), the last norm, and the blocks."""
    gen = torch.Generator().manual_seed(seed + 1000)
    C = shape.width
    p = {"embed": torch.randn(vocab, C, generator=gen) * C ** -0.5, "norm.weight": torch.randn(C, generator=gen) * 0.1 + 1.0,
         "norm.bias": torch.randn(C, generator=gen) * 0.1}
    p = {n: t.to(device=device, dtype=torch.bfloat16) for n, t in p.items()}
    for i in range(layers):
        p.update({"%d.%s" % (i, n): t for n, t in block_parameters(shape, seed + i, device).items()})
    return p


def batch_of(vocab: int, sequences: int, tokens: int, seed: int, device="cuda"):
    """ids and targets [sequences, tokens] (the next token; -1 and -100 where there is none) and the tokens in use of each."""
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(vocab, (sequences, tokens + 1), generator=gen)
    used = torch.linspace(tokens, tokens // 3, sequences).to(torch.int32).clamp(min=1)
    there = torch.arange(tokens)[None, :] < used[:, None]
    return (torch.where(there, ids[:, :-1], -1).to(device), torch.where(there, ids[:, 1:], -100).to(device), used.to(device))


class Model:
    """Forward and backward pass of one rank.  The loss is the mean over sequences of the mean over their tokens;
    `grads` receives the gradients of all parameters, in the order of names()."""

    def __init__(self, shape: Shape, layers: int, params: Dict[str, torch.Tensor]):
        self.shape, self.params = shape, params
        self.scale = shape.width ** 0.5                       # of the embedding: the table's rows have the norm 1
        self.blocks = [Block(shape, {n: params["%d.%s" % (i, n)] for n in NAMES}) for i in range(layers)]
        self.grads = {n: torch.empty_like(params[n]) for n in ("embed", "norm.weight", "norm.bias")}
        for i, block in enumerate(self.blocks):
            self.grads.update({"%d.%s" % (i, n): block.grads[n] for n in NAMES})

    def forward(self, ids: torch.Tensor, targets: torch.Tensor, used: torch.Tensor) -> torch.Tensor:
        """The loss of each token (0 where there is no target)."""
        p, (B, L), C, dev = self.params, ids.shape, self.shape.width, ids.device
        self.size, self.ids, self.targets = (B, L, C), ids.reshape(-1), targets.reshape(-1)
        x = torch.empty(B * L, C, dtype=torch.bfloat16, device=dev)
        kt.kt_embed_forward(self.ids, p["embed"], x, scale=self.scale)
        x = x.view(B, L, C)
        for block in self.blocks:
            x = block.forward(x, used)
        rows = x.reshape(-1, C)
        self.hidden, self.rstd, self.kept = torch.empty_like(rows), torch.empty(B * L, device=dev), _Kept(B * L, C, dev)
        kt.kt_norm_forward(rows, p["norm.weight"], p["norm.bias"], self.hidden, None, self.rstd, codes=self.kept.codes, scales=self.kept.scales)
        loss, self.lse = torch.empty(B * L, device=dev), torch.empty(B * L, device=dev)
        work = torch.empty(kt.kt_xent_workspace(B * L, C, p["embed"].size(0)), dtype=torch.uint8, device=dev)
        kt.kt_xent_forward(self.hidden, p["embed"], self.targets, loss, self.lse, work)
        return loss.view(B, L)

    def backward(self) -> None:
        p, g, dev = self.params, self.grads, self.hidden.device
        B, L, C = self.size
        counted = (self.targets.view(B, L) >= 0).sum(1, keepdim=True).clamp(min=1)
        dloss = (1.0 / (B * counted)).expand(B, L).reshape(-1).contiguous()
        dh = torch.empty_like(self.hidden)
        work = torch.empty(kt.kt_xent_workspace(*self.hidden.shape, p["embed"].size(0), True), dtype=torch.uint8, device=dev)
        kt.kt_xent_backward(dloss, self.hidden, p["embed"], self.targets, self.lse, dh, g["embed"], work)
        dx = torch.empty_like(dh)
        work = torch.empty(kt.kt_norm_workspace(*dh.shape), dtype=torch.uint8, device=dev)
        kt.kt_norm_backward(dh, p["norm.weight"], self.rstd, dx, g["norm.weight"], g["norm.bias"], work, codes=self.kept.codes, scales=self.kept.scales)
        dx = dx.view(B, L, C)
        for block in reversed(self.blocks):
            dx = block.backward(dx)
        work = torch.empty(kt.kt_embed_workspace(B * L, C, p["embed"].size(0)), dtype=torch.uint8, device=dev)
        kt.kt_embed_backward(dx.reshape(-1, C), self.ids, g["embed"], work, scale=self.scale, base=g["embed"])


def plain_gradients(shape: Shape, layers: int, params: Dict[str, torch.Tensor], ids: torch.Tensor, targets: torch.Tensor,
                    used: torch.Tensor) -> Dict[str, torch.Tensor]:
    """The same model on the whole batch in fp32 with stock operations and automatic differentiation."""
    p = {n: t.detach().float().requires_grad_() for n, t in params.items()}
    (B, L), C, D = ids.shape, shape.width, shape.head_dim
    norm = torch.nn.functional.layer_norm
    x = torch.where(ids[..., None] >= 0, p["embed"][ids.clamp(min=0)] * C ** 0.5, 0.0)
    i = torch.arange(L, device=ids.device)
    seen = (i[None, :] < used[:, None])[:, None, None, :]
    if shape.causal:
        seen = seen & (i[None, :] <= i[:, None])[None, None]
    for b in range(layers):
        q = {n: p["%d.%s" % (b, n)] for n in NAMES}
        heads = (norm(x, (C,), q["norm1.weight"], q["norm1.bias"]) @ q["qkv"]).view(B, L, -1, D).transpose(1, 2)
        k, v = (t.repeat_interleave(shape.heads // shape.heads_kv, 1) for t in (heads[:, shape.heads:shape.heads + shape.heads_kv], heads[:, shape.heads + shape.heads_kv:]))
        probs = torch.softmax((heads[:, :shape.heads] @ k.transpose(2, 3) * D ** -0.5).masked_fill(~seen, float("-inf")), 3)
        y = x + (probs @ v).transpose(1, 2).reshape(B, L, C) @ q["proj"]
        x = y + torch.nn.functional.gelu(norm(y, (C,), q["norm2.weight"], q["norm2.bias"]) @ q["up"]) @ q["down"]
    logits = norm(x, (C,), p["norm.weight"], p["norm.bias"]) @ p["embed"].t()
    each = torch.nn.functional.cross_entropy(logits.view(B * L, -1), targets.reshape(-1), reduction="none", ignore_index=-100).view(B, L)
    (each.sum(1) / (targets >= 0).sum(1).clamp(min=1)).mean().backward()
    return {n: t.grad for n, t in p.items()}


def synchronised_step(shape: Shape, layers: int, params: Dict[str, torch.Tensor], batch, shares: List[int], group_of: List[int]) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
    """(loss of each token, gradients of the mean over all sequences): rank r does the next shares[r] of them."""
    lists, losses, at, given_up, order = [], [], 0, kt.kt_waits_given_up(), names(layers)
    for share in shares:
        model = Model(shape, layers, params)
        losses.append(model.forward(*(t[at:at + share] for t in batch)))
        model.backward()
        at += share
        lists.append([model.grads[n] for n in order])
    if kt.kt_waits_given_up() != given_up:          # gradients that are not right reach no replica
        raise RuntimeError("a wait inside a kernel was given up: the step has no result")
    ctx = kt.kt_groups_init(group_of, shares)
    kt.kt_bucket_pack(ctx, lists, 25 << 20)
    out = [torch.empty_like(params[n]) for n in order]
    kt.kt_sync_direct(ctx, [out])
    torch.cuda.current_stream().synchronize()       # the ranks' gradients go out of use with this call
    kt.kt_destroy(ctx)
    return torch.cat(losses), dict(zip(order, out))


class Update:
    """One step of all parameters: the blocks' matrices along their orthogonalised momentum, the others along the gradient.  A matrix with
    more outputs than inputs moves by the root of their ratio more.  `inputs_first`: whether matrices are [inputs, outputs], as
    those of Model are (x @ up), or [outputs, inputs], as stock linear layers have them."""

    def __init__(self, layers: int, params: Dict[str, torch.Tensor], rate: float = 0.02, momentum: float = 0.95, rate_others: float = 0.1, inputs_first: bool = False):
        self.layers, self.params, self.rate, self.momentum, self.rate_others, self.inputs_first = layers, params, rate, momentum, rate_others, inputs_first
        self.state = {n: torch.zeros(layers, *params["0." + n].shape, device=params["0." + n].device) for n in MATRICES} if layers else {}
        self.work = {n: torch.empty(kt.kt_orth_workspace(*s.shape), dtype=torch.uint8, device=s.device) for n, s in self.state.items()}

    def directions(self, grads: Dict[str, torch.Tensor]) -> Dict[str, torch.Tensor]:
        """Orthogonalised momentum of the matrices, [layers, rows, cols] for each name."""
        out = {}
        for n, s in self.state.items():
            s.mul_(self.momentum).add_(torch.stack([grads["%d.%s" % (i, n)] for i in range(self.layers)]))
            out[n] = torch.empty_like(s, dtype=torch.bfloat16)
            inputs, outputs = s.shape[1:] if self.inputs_first else s.shape[:0:-1]
            kt.kt_orth_update(s, out[n], self.work[n], scale=max(1.0, outputs / inputs) ** 0.5)
        return out

    def step(self, grads: Dict[str, torch.Tensor]) -> None:
        turned = self.directions(grads)
        for n, p in self.params.items():
            layer, _, name = n.partition(".")
            if name in turned:
                p.sub_(turned[name][int(layer)], alpha=self.rate)
            else:
                p.sub_(grads[n], alpha=self.rate_others)


def example(tokens: int = 512, width: int = 1024, layers: int = 2, vocab: int = 32000, batch: int = 16, seed: int = 0):
    """One step on four ranks in two groups, the second group 1.6 times slower; sequences of different lengths.
    Returns (shares, relative error of each gradient against the plain fp32 model on the whole batch)."""
    shape = Shape(width=width, heads=width // 64, heads_kv=max(1, width // 256), hidden=4 * width)
    shares = kt.kt_schedule([1.0, 1.0, 1.6, 1.6], batch)
    params, data = parameters(shape, layers, vocab, seed), batch_of(vocab, batch, tokens, seed + 1)
    _, got = synchronised_step(shape, layers, params, data, shares, [0, 0, 1, 1])
    want = plain_gradients(shape, layers, params, *data)
    errors = {n: float((got[n].float() - want[n]).norm() / want[n].norm()) for n in got}
    Update(layers, params, inputs_first=True).step(got)
    return shares, errors


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--steps", type=int, default=5, help="timed steps of one rank")
    a = ap.parse_args()
    shares, errors = example(a.tokens, a.width, a.layers, a.vocab)
    print("shares %s" % shares)
    for n, e in errors.items():
        print("%-16s relative error against the fp32 model %.4f" % (n, e))
    shape = Shape(width=a.width, heads=a.width // 64, heads_kv=max(1, a.width // 256), hidden=4 * a.width)
    params, data = parameters(shape, a.layers, a.vocab, 0), batch_of(a.vocab, 8, a.tokens, 1)
    model, update = Model(shape, a.layers, params), Update(a.layers, params, inputs_first=True)

    def step():
        model.forward(*data)
        model.backward()
        update.step(model.grads)

    for _ in range(3):
        step()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.steps):
        step()
    end.record()
    end.synchronize()
    print("forward, backward and update on 8 x %d tokens: %.3f ms" % (a.tokens, start.elapsed_time(end) / a.steps))


if __name__ == "__main__":
    main()
