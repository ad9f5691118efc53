"""A training step of a transformer block on simulated ranks of unequal speed, from the shares to the
synchronised gradients:

    python -m paper_2505_10183_b200.block_step [--tokens 512] [--width 1024] [--steps 5]

Every rank runs the block forward and backward on its share of the batch with the library's training
operators: layer norm, attention and GELU, of which only 8-bit checkpoints are kept (normalised rows, the
hidden activation's input); the matrix products between them are the stock ones.  Its gradients, the means
over its own sequences, are then combined with the shares' weights in one pass (kt_sync_direct), and the
result is compared with the gradient of the whole batch from a plain fp32 block.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

from . import binding as kt

NAMES = ("norm1.weight", "norm1.bias", "qkv", "proj", "norm2.weight", "norm2.bias", "up", "down")


@dataclass
class Shape:
    width: int = 1024
    heads: int = 16
    heads_kv: int = 4
    hidden: int = 4096
    causal: bool = True

    @property
    def head_dim(self) -> int:
        return self.width // self.heads


def parameters(shape: Shape, seed: int, device="cuda") -> Dict[str, torch.Tensor]:
    """bf16 parameters of one block: x + proj(attention(norm1(x))), then y + down(gelu(up(norm2(y))))."""
    gen = torch.Generator().manual_seed(seed)
    C, D, F = shape.width, shape.head_dim, shape.hidden

    def normal(*size, std, mean=0.0):
        return (torch.randn(*size, generator=gen) * std + mean).to(device=device, dtype=torch.bfloat16)

    return {"norm1.weight": normal(C, std=0.1, mean=1.0), "norm1.bias": normal(C, std=0.1),
            "qkv": normal(C, (shape.heads + 2 * shape.heads_kv) * D, std=C ** -0.5), "proj": normal(C, C, std=C ** -0.5),
            "norm2.weight": normal(C, std=0.1, mean=1.0), "norm2.bias": normal(C, std=0.1),
            "up": normal(C, F, std=C ** -0.5), "down": normal(F, C, std=F ** -0.5)}


class _Kept:
    """Rows in 8 bits."""

    def __init__(self, rows: int, cols: int, device):
        self.rows, self.cols = rows, cols
        self.codes = torch.empty(rows, kt.kt_ckpt_pitch(cols), dtype=torch.int8, device=device)
        self.scales = torch.empty(rows, kt.kt_ckpt_blocks(cols), device=device)

    def restore(self, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> torch.Tensor:
        out = torch.empty(self.rows, self.cols, dtype=torch.bfloat16, device=self.codes.device)
        kt.kt_ckpt_restore(self.codes, self.scales, out, weight, bias)
        return out


class Block:
    """Forward and backward pass of one rank on x [sequences, tokens, width] (bf16); used: tokens of each
    sequence (int32), or None.  `grads` receives the gradients, as tensors that kt_bucket_pack can take."""

    def __init__(self, shape: Shape, params: Dict[str, torch.Tensor]):
        self.shape, self.params = shape, params
        self.grads = {n: torch.empty_like(params[n]) for n in NAMES}

    def _heads(self, qkv: torch.Tensor, B: int, L: int):
        s = self.shape
        t = qkv.view(B, L, s.heads + 2 * s.heads_kv, s.head_dim)
        return t[:, :, :s.heads], t[:, :, s.heads:s.heads + s.heads_kv], t[:, :, s.heads + s.heads_kv:]

    def _norm(self, x: torch.Tensor, which: str):
        """(output, kept normalised rows, rstd) of the layer norm `which`."""
        out, rstd, kept = torch.empty_like(x), torch.empty(x.size(0), device=x.device), _Kept(*x.shape, x.device)
        kt.kt_norm_forward(x, self.params[which + ".weight"], self.params[which + ".bias"], out, None, rstd,
                           codes=kept.codes, scales=kept.scales)
        return out, kept, rstd

    def _norm_backward(self, dout: torch.Tensor, which: str, kept: _Kept, rstd: torch.Tensor) -> torch.Tensor:
        dx = torch.empty_like(dout)
        work = torch.empty(kt.kt_norm_workspace(*dout.shape), dtype=torch.uint8, device=dout.device)
        kt.kt_norm_backward(dout, self.params[which + ".weight"], rstd, dx, self.grads[which + ".weight"],
                            self.grads[which + ".bias"], work, codes=kept.codes, scales=kept.scales)
        return dx

    def forward(self, x: torch.Tensor, used: Optional[torch.Tensor] = None) -> torch.Tensor:
        s, p = self.shape, self.params
        B, L, C = x.shape
        rows = x.reshape(-1, C)
        h, self.kept1, self.rstd1 = self._norm(rows, "norm1")
        self.qkv = h @ p["qkv"]
        q, k, v = self._heads(self.qkv, B, L)
        self.attn = torch.empty(B, L, s.heads, s.head_dim, dtype=x.dtype, device=x.device)
        self.lse = torch.empty(B, s.heads, L, device=x.device)
        kt.kt_attn_forward(q, k, v, self.attn, self.lse, causal=s.causal, used_q=used, used_kv=used)
        y = rows + self.attn.view(-1, C) @ p["proj"]
        h, self.kept2, self.rstd2 = self._norm(y, "norm2")
        u = h @ p["up"]
        self.kept_u = _Kept(*u.shape, x.device)
        kt.kt_act_forward(u, u, self.kept_u.codes, self.kept_u.scales, "gelu")        # in place: u is kept in 8 bits only
        self.used, self.size = used, (B, L, C)
        return (y + u @ p["down"]).view(B, L, C)

    def backward(self, dz: torch.Tensor) -> torch.Tensor:
        s, p, g = self.shape, self.params, self.grads
        B, L, C = self.size
        dz = dz.reshape(-1, C)
        a = self.kept_u.restore()
        kt.kt_act_forward(a, a, kind="gelu")
        torch.mm(a.t(), dz, out=g["down"])
        du = dz @ p["down"].t()
        kt.kt_act_backward(du, self.kept_u.codes, self.kept_u.scales, du, "gelu")
        torch.mm(self.kept2.restore(p["norm2.weight"], p["norm2.bias"]).t(), du, out=g["up"])
        dy = self._norm_backward(du @ p["up"].t(), "norm2", self.kept2, self.rstd2).add_(dz)
        torch.mm(self.attn.view(-1, C).t(), dy, out=g["proj"])
        dattn = (dy @ p["proj"].t()).view(B, L, s.heads, s.head_dim)
        dqkv = torch.empty_like(self.qkv)                                             # the three gradients side by side
        work = torch.empty(kt.kt_attn_workspace(self.attn, self.attn), dtype=torch.uint8, device=dz.device)
        kt.kt_attn_backward(dattn, *self._heads(self.qkv, B, L), self.attn, self.lse, *self._heads(dqkv, B, L), work,
                            causal=s.causal, used_q=self.used, used_kv=self.used)
        torch.mm(self.kept1.restore(p["norm1.weight"], p["norm1.bias"]).t(), dqkv, out=g["qkv"])
        dx = self._norm_backward(dqkv @ p["qkv"].t(), "norm1", self.kept1, self.rstd1).add_(dy)
        return dx.view(B, L, C)


def plain_gradients(shape: Shape, params: Dict[str, torch.Tensor], x: torch.Tensor, dz: torch.Tensor,
                    used: Optional[torch.Tensor] = None) -> Dict[str, torch.Tensor]:
    """The same block in fp32 with stock operations and automatic differentiation."""
    p = {n: t.detach().float().requires_grad_() for n, t in params.items()}
    B, L, C = x.shape
    s = shape

    def norm(t, which):
        return torch.nn.functional.layer_norm(t, (C,), p[which + ".weight"], p[which + ".bias"], 1e-5)

    y = x.float()
    qkv = (norm(y, "norm1") @ p["qkv"]).view(B, L, s.heads + 2 * s.heads_kv, s.head_dim).transpose(1, 2)
    q, k, v = qkv[:, :s.heads], qkv[:, s.heads:s.heads + s.heads_kv], qkv[:, s.heads + s.heads_kv:]
    k, v = (t.repeat_interleave(s.heads // s.heads_kv, 1) for t in (k, v))
    i = torch.arange(L, device=x.device)
    seen = (i[None, :] <= i[:, None]) if s.causal else torch.ones(L, L, dtype=torch.bool, device=x.device)
    seen = seen[None, None]
    if used is not None:
        seen = seen & (i[None, :] < used[:, None])[:, None, None, :]
    probs = torch.softmax((q @ k.transpose(2, 3) * s.head_dim ** -0.5).masked_fill(~seen, float("-inf")), 3)
    y = y + (probs @ v).transpose(1, 2).reshape(B, L, C) @ p["proj"]
    z = y + torch.nn.functional.gelu(norm(y, "norm2") @ p["up"]) @ p["down"]
    (z * dz.float()).sum().backward()
    return {n: t.grad for n, t in p.items()}


def synchronised_step(shape: Shape, params: Dict[str, torch.Tensor], x: torch.Tensor, dz: torch.Tensor, shares: List[int],
                      group_of: List[int], used: Optional[torch.Tensor] = None) -> Dict[str, torch.Tensor]:
    """Gradients of the mean over all sequences of x: rank r does the next shares[r] of them.  dz: gradient of
    one sequence's loss with respect to its output."""
    lists, at, given_up = [], 0, kt.kt_attn_given_up()
    for share in shares:
        mine = slice(at, at + share)
        at += share
        block = Block(shape, params)
        block.forward(x[mine], None if used is None else used[mine])
        block.backward((dz[mine].float() / share).to(dz.dtype))
        lists.append([block.grads[n] for n in NAMES])
    if kt.kt_attn_given_up() != given_up:           # gradients that are not right reach no replica
        raise RuntimeError("a wait inside an attention kernel was given up: the step has no result")
    ctx = kt.kt_groups_init(group_of, shares)
    kt.kt_bucket_pack(ctx, lists, 25 << 20)
    out = [torch.empty_like(params[n]) for n in NAMES]
    kt.kt_sync_direct(ctx, [out])
    torch.cuda.current_stream().synchronize()       # the ranks' gradients go out of use with this call
    kt.kt_destroy(ctx)
    return dict(zip(NAMES, out))


def example(tokens: int = 512, width: int = 1024, batch: int = 16, seed: int = 0):
    """One step on four ranks in two groups, the second group 1.6 times slower; sequences of different lengths.
    Returns (shares, relative error of each gradient against the plain fp32 block on the whole batch)."""
    shape = Shape(width=width, heads=width // 64, heads_kv=max(1, width // 256), hidden=4 * width)
    shares = kt.kt_schedule([1.0, 1.0, 1.6, 1.6], batch)
    params = parameters(shape, seed)
    gen = torch.Generator().manual_seed(seed + 1)
    x, dz = (torch.randn(batch, tokens, width, generator=gen).to(device="cuda", dtype=torch.bfloat16) for _ in range(2))
    used = torch.linspace(tokens, tokens // 3, batch).to(torch.int32).clamp(min=1).cuda()
    dz.masked_fill_((torch.arange(tokens, device="cuda")[None, :] >= used[:, None])[..., None], 0.0)
    got = synchronised_step(shape, params, x, dz, shares, [0, 0, 1, 1], used)
    want = plain_gradients(shape, params, x, dz / batch, used)
    return shares, {n: float((got[n].float() - want[n]).norm() / want[n].norm()) for n in NAMES}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=5, help="timed steps of one rank")
    a = ap.parse_args()
    shares, errors = example(a.tokens, a.width)
    print("shares %s" % shares)
    for n, e in errors.items():
        print("%-14s relative error against the fp32 block %.4f" % (n, e))
    shape = Shape(width=a.width, heads=a.width // 64, heads_kv=max(1, a.width // 256), hidden=4 * a.width)
    block = Block(shape, parameters(shape, 0))
    x = torch.randn(8, a.tokens, a.width, device="cuda", dtype=torch.bfloat16)
    for _ in range(3):
        block.backward(block.forward(x))
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(a.steps):
        block.backward(block.forward(x))
    end.record()
    end.synchronize()
    print("forward and backward of 8 x %d tokens: %.3f ms" % (a.tokens, start.elapsed_time(end) / a.steps))


if __name__ == "__main__":
    main()
