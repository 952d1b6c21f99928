"""Cross-entropy as the first call of its kind in a process: whether a launch is accepted does not depend on the calls before it."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Rows of six 16-byte units a thread, 48 KB a block beside what the kernels have of their own, shared by one, two and eight blocks; and
# of five and seven.
PROGRAM = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2010_16165_b200 import binding as B
gen = torch.Generator(device="cuda").manual_seed(1)
for M, C, dtype in {sizes}:
    dtype = getattr(torch, dtype)
    x = torch.randn(M, C, generator=gen, device="cuda").to(dtype)
    lab = torch.randint(0, C, (M,), generator=gen, device="cuda")
    loss, dx = torch.empty(M, device="cuda"), torch.empty_like(x)
    B.fp_cross_entropy(x, lab, loss, dlogits=dx)
    X = x.double()
    p = torch.softmax(X, 1)
    r = (C / 16 + 60) * 2.0 ** -22
    want = -torch.log_softmax(X, 1).gather(1, lab[:, None])[:, 0]
    assert ((loss.double() - want).abs() <= r + 2.0 ** -22 * want).all()
    err = (r + 2.0 ** -18) * p + 2.0 ** -25
    p[torch.arange(M, device="cuda"), lab] -= 1
    assert ((dx.double() - p).abs() <= err + (torch.finfo(dtype).eps / 2 + 2.0 ** -22) * p.abs()).all()
print("done")
"""


@pytest.mark.parametrize("sizes", [[(256, 10450, "float32"), (256, 21841, "float32"), (256, 21841, "bfloat16"), (4, 180000, "float16")],
                                   [(256, 11221, "float32"), (4096, 21128, "bfloat16"), (256, 21841, "float16")],
                                   [(300, 10000, "float32"), (300, 12500, "float32"), (300, 19000, "float16"), (300, 25000, "bfloat16")]])
def test_in_a_process_of_its_own(sizes):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    r = subprocess.run([sys.executable, "-c", PROGRAM.format(root=ROOT, sizes=sizes)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr[-2000:]
