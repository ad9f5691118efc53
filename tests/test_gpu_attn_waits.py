"""Waits inside the attention kernels that give up: results that are not right are NaN, the count tells, the device
stays usable.  The limit is set to 0, so that whatever is not there at the first look is given up; nothing hangs
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


def heads(*shape):
    return torch.randn(*shape, generator=gen).to(BF16).cuda()


def buffer(*shape, dtype=BF16):
    return torch.full(shape, SENTINEL, dtype=dtype, device="cuda")


def nan_or_right(got, want):
    got, want = got.float(), want.float()
    bad = torch.isnan(got)
    assert not (got == SENTINEL).any()                      # what the buffer held before
    assert torch.equal(got[~bad], want[~bad])
    return int(bad.sum())
"""

PASSES = START + """
# sizes whose items one CTA does each, and sizes whose keys or queries the CTAs of a cluster share
for B, Lq, Lk, H, Hk, D in ((3, 300, 300, 8, 4, 64), (3, 300, 300, 8, 4, 128), (1, 1, 4100, 4, 2, 64), (1, 5, 2000, 4, 2, 128), (2, 700, 700, 8, 1, 64), (1, 1500, 300, 4, 1, 128)):
    gen = torch.Generator().manual_seed(Lq + D)
    q, k, v, dout = heads(B, Lq, H, D), heads(B, Lk, Hk, D), heads(B, Lk, Hk, D), heads(B, Lq, H, D)
    work = torch.empty(kt.kt_attn_workspace(q, k), dtype=torch.uint8, device="cuda")

    def forward():
        out, lse = buffer(B, Lq, H, D), buffer(B, H, Lq, dtype=torch.float32)
        kt.kt_attn_forward(q, k, v, out, lse, causal=True)
        torch.cuda.synchronize()
        return out, lse

    def backward(out, lse):
        grads = buffer(B, Lq, H, D), buffer(B, Lk, Hk, D), buffer(B, Lk, Hk, D)
        kt.kt_attn_backward(dout, q, k, v, out, lse, *grads, work, causal=True)
        torch.cuda.synchronize()
        return grads

    want = forward()
    want_grads = backward(*want)
    count = kt.kt_attn_given_up()
    kt.kt_attn_wait_limit(0)
    got = forward()
    after = kt.kt_attn_given_up()
    assert after > count and sum(nan_or_right(a, b) for a, b in zip(got, want)) > 0
    got = backward(*want)
    kt.kt_attn_wait_limit(2 * SECOND)
    assert kt.kt_attn_given_up() > after and sum(nan_or_right(a, b) for a, b in zip(got, want_grads)) > 0
    count = kt.kt_attn_given_up()
    again = forward()                                       # as if nothing had been
    assert all(torch.equal(a, b) for a, b in zip((*again, *backward(*again)), (*want, *want_grads)))
    assert kt.kt_attn_given_up() == count
print("done")
"""

STEP = START + """
from paper_2505_10183_b200 import block_step as step
shape = step.Shape(width=256, heads=4, heads_kv=2, hidden=512)
params = step.parameters(shape, 3)
gen = torch.Generator().manual_seed(4)
x, dz = heads(4, 64, 256), heads(4, 64, 256)
want = step.synchronised_step(shape, params, x, dz, [3, 1], [0, 1])
kt.kt_attn_wait_limit(0)
try:
    step.synchronised_step(shape, params, x, dz, [3, 1], [0, 1])
    raise SystemExit("gradients of waits that gave up were synchronised")
except RuntimeError as e:
    assert "given up" in str(e)
kt.kt_attn_wait_limit(2 * SECOND)
got = step.synchronised_step(shape, params, x, dz, [3, 1], [0, 1])
assert all(torch.equal(got[n], want[n]) for n in step.NAMES)
print("done")
"""

COUNT = START + """
gen = torch.Generator().manual_seed(5)
q = heads(1, 300, 4, 64)
out, lse = buffer(1, 300, 4, 64), buffer(1, 4, 300, dtype=torch.float32)
kt.kt_attn_forward(q, q, q, out, lse)
assert kt.kt_attn_given_up() == 0
kt.kt_attn_wait_limit(0)
s = torch.cuda.Stream()
with torch.cuda.stream(s):
    torch.cuda._sleep(200 * 1000 * 1000)                    # the kernel starts a tenth of a second after the call has returned
    kt.kt_attn_forward(q, q, q, out, lse)
count = kt.kt_attn_given_up()
torch.cuda.synchronize()
assert count == kt.kt_attn_given_up() > 0, count
print("done")
"""


def run(source):
    done = subprocess.run([sys.executable, "-c", source], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.endswith("done\n"), done.stdout[-3000:]


def test_results_that_are_not_right_are_nan():
    run(PASSES)


def test_a_step_whose_waits_gave_up_synchronises_nothing():
    run(STEP)


def test_the_count_waits_for_every_stream():
    run(COUNT)
