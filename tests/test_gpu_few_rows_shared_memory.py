"""Products of three and four rows whose quantised rows take about 48 KB of shared memory, beside the kernel's own: more than a kernel has without
being allowed more.  Each length in a process of its own, since what one call allows a kernel it keeps."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# The integers are exact (at most 2^28: 24 bits of fp32 round them once), then two products: 3 roundings of 2^-24.
CHILD = """
import torch
from paper_2210_13149_b200 import binding as B
ctx = B.BiGCN(0)
d = %d
gen = torch.Generator(device="cuda").manual_seed(d)
q_w, s_w = ctx.quantize_rows(torch.randn((500, d), device="cuda", generator=gen))
for n in (3, 4):
    x = torch.randn((n, d), device="cuda", generator=gen)
    before = ctx.launch_count()
    got = ctx.quantized_product(x, q_w, s_w)
    assert ctx.launch_count() == before + 1            # the one launch that this is about
    q_x, s_x = ctx.quantize_rows(x)
    ctx.sync_check()
    want = (q_x.double() @ q_w.double().t()) * s_x.double()[:, None] * s_w.double()
    assert ((got.double() - want).abs() <= want.abs() * 3.01 * 2.0 ** -24 + 2.0 ** -140).all()
print("right")
"""


@pytest.mark.parametrize("d", [12256, 12257, 12288, 16384])
def test_few_long_rows_first_in_their_process(d):
    r = subprocess.run([sys.executable, "-c", CHILD % d], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.endswith("right\n"), r.stderr[-2000:]
