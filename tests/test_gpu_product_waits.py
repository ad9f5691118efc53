"""Waits inside the kernels of the loss and of matrix updates that give up: results that are not right are NaN, the count
tells, the device stays usable.  The limit is set to 0, so that whatever is not there at the first look is given up; nothing hangs
or faults.  In processes of their own, whose counts end with them."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

START = """
import torch
from paper_2505_10183_b200 import binding as kt
BF16, SENTINEL, SECOND = torch.bfloat16, 77.0, 10 ** 9
torch.cuda.set_device(0)


def buffer(*shape, dtype=BF16):
    return torch.full(shape, SENTINEL, dtype=dtype, device="cuda")


def nan_or_right(got, want):
    got, want = got.float(), want.float()
    bad = torch.isnan(got)
    assert not (got == SENTINEL).any()                      # what the buffer held before
    assert torch.equal(got[~bad], want[~bad])
    return int(bad.sum())


def check(run):
    want = run()
    count = kt.kt_waits_given_up()
    kt.kt_attn_wait_limit(0)
    got = run()
    kt.kt_attn_wait_limit(2 * SECOND)
    after = kt.kt_waits_given_up()
    assert after > count and kt.kt_attn_given_up() == 0
    assert sum(nan_or_right(a, b) for a, b in zip(got, want)) > 0
    again = run()                                           # as if nothing had been
    assert all(torch.equal(a, b) for a, b in zip(again, want)) and kt.kt_waits_given_up() == after
"""

LOSS = START + """
# one CTA to a tile, pairs, rows left out, shares of dhidden, pieces of the vocabulary
for N, D, V, ignored in ((24, 64, 3000, 0.0), (200, 136, 5003, 0.2), (2600, 256, 4001, 0.0), (3000, 128, 5000, 0.4), (8192, 16, 40000, 0.0)):
    gen = torch.Generator().manual_seed(N)
    hidden, weight = (torch.randn(n, D, generator=gen).to(BF16).cuda() for n in (N, V))
    targets = torch.randint(V, (N,), generator=gen)
    targets[torch.rand(N, generator=gen) < ignored] = -1
    targets, dloss = targets.cuda(), torch.ones(N, device="cuda")
    work = [torch.empty(kt.kt_xent_workspace(N, D, V, back), dtype=torch.uint8, device="cuda") for back in (False, True)]

    def forward():
        loss, lse = buffer(N, dtype=torch.float32), buffer(N, dtype=torch.float32)
        kt.kt_xent_forward(hidden, weight, targets, loss, lse, work[0], scale=D ** -0.5)
        torch.cuda.synchronize()
        return loss, lse

    lse = forward()[1]

    def backward():
        dh, dw = buffer(N, D), buffer(V, D)
        kt.kt_xent_backward(dloss, hidden, weight, targets, lse, dh, dw, work[1], scale=D ** -0.5)
        torch.cuda.synchronize()
        return dh, dw

    check(forward)
    check(backward)
print("done")
"""

UPDATE = START + """
for shape in ((1, 100, 60), (1, 300, 500), (2, 640, 200), (75, 200, 136), (75, 130, 300)):
    x = torch.randn(*shape, generator=torch.Generator().manual_seed(1)).cuda()
    work = torch.empty(kt.kt_orth_workspace(*shape), dtype=torch.uint8, device="cuda")

    def run():
        out = buffer(*shape)
        kt.kt_orth_update(x, out, work)
        torch.cuda.synchronize()
        return (out,)

    check(run)
print("done")
"""


@pytest.mark.parametrize("program", [LOSS, UPDATE], ids=["loss", "update"])
def test_given_up(program):
    done = subprocess.run([sys.executable, "-c", program], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=240)
    assert done.returncode == 0 and done.stdout.endswith("done\n"), done.stdout[-3000:]
