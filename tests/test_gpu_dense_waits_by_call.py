"""A wait that runs out in each kind of dense product by itself: the status is reported under that product's own name, so that none hides behind another's.
Each in a process of its own, because the reported flag stays up."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys
import torch
from paper_2210_13149_b200 import binding as B
kind = sys.argv[1]
ctx = B.BiGCN(0)
gen = torch.Generator(device="cuda").manual_seed(1)
cases = []
sizes = {"few rows": ((20, 2000, 60000), (50, 2000, 60000)), "rows": ((40000, 700, 40), (30000, 900, 100), (3000, 1500, 8000))}
for n, d, m in sizes.get(kind, ((40000, 700, 40), (30000, 900, 100), (3000, 1500, 8000), (20, 1000, 60000))):
    x = torch.randn((n, d), device="cuda", generator=gen).bfloat16()
    W = (torch.randn((m, d), device="cuda", generator=gen) / d ** 0.5).bfloat16()
    if kind in sizes:
        q, s = ctx.quantize_rows(W)
        cases.append(lambda a=(x, q, s): (ctx.quantized_product(*a),))
        continue
    y = torch.randint(0, m, (n,), device="cuda", generator=gen)
    g = torch.full((n,), 1.0 / n, device="cuda")
    lse = ctx.class_loss(x, W, y)[1]
    cases.append((lambda a=(x, W, y): ctx.class_loss(*a)) if kind == "loss" else (lambda a=(x, W, y, lse, g): ctx.class_loss_backward(*a)))
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


@pytest.mark.parametrize("kind,name", [("few rows", "product of 8-bit rows"), ("rows", "product of 8-bit rows"), ("loss", "class loss"), ("gradients", "class loss")])
def test_a_wait_that_runs_out_is_reported_as_what_it_was(kind, name):
    r = subprocess.run([sys.executable, "-c", CHILD, kind], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "status 8" in r.stdout and "a bounded wait ran out (%s)" % name in r.stdout, r.stdout
    assert r.stdout.endswith("usable\n")
