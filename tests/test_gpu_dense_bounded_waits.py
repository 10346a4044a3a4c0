"""A wait that runs out inside the products of 8-bit rows and of the class loss: every block still ends, the status is reported, and the
device stays usable.  In a process of its own, because the reported flag stays up."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Tiles of one block and of a pair, of 32, 64, 128 and 256 columns (four, two and one group of epilogue warps); several tiles to a block and
# more stages than the ring has.
CHILD = """
import torch
from paper_2210_13149_b200 import binding as B
ctx = B.BiGCN(0)
gen = torch.Generator(device="cuda").manual_seed(1)
cases = []
for n, d, m in ((40000, 700, 40), (30000, 900, 100), (3000, 1500, 8000), (20, 2000, 60000), (50, 2000, 60000)):
    x = torch.randn((n, d), device="cuda", generator=gen).bfloat16()
    q, s = ctx.quantize_rows(torch.randn((m, d), device="cuda", generator=gen))
    cases.append(lambda a=(x, q, s): (ctx.quantized_product(*a),))
for n, d, m in ((40000, 700, 40), (30000, 900, 100), (3000, 1500, 8000), (20, 1000, 60000)):
    x = torch.randn((n, d), device="cuda", generator=gen).bfloat16()
    W = (torch.randn((m, d), device="cuda", generator=gen) / d ** 0.5).bfloat16()
    y = torch.randint(0, m, (n,), device="cuda", generator=gen)
    g = torch.full((n,), 1.0 / n, device="cuda")
    lse = ctx.class_loss(x, W, y)[1]
    cases.append(lambda a=(x, W, y): ctx.class_loss(*a))
    cases.append(lambda a=(x, W, y, lse, g): ctx.class_loss_backward(*a))
want = [f() for f in cases]
ctx.sync_check()
for tries in (1, 2, 3):
    ctx.set_option(B.OPT_WAIT_TRIES, tries)
    for f in cases:
        f()
    torch.cuda.synchronize()
try:
    ctx.sync_check()
    print("no wait ran out")
except B.BigcnError as e:
    print("status", e.status, e)
ctx.set_option(B.OPT_WAIT_TRIES, 0)
for f, w in zip(cases, want):
    assert all(torch.equal(a, b) for a, b in zip(f(), w))
print("usable")
"""


def test_a_wait_that_runs_out_ends_every_block_and_is_reported():
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "status 8" in r.stdout and ("a bounded wait ran out (class loss)" in r.stdout or "a bounded wait ran out (product of 8-bit rows)" in r.stdout), r.stdout
    assert r.stdout.endswith("usable\n")
