"""A process's first calls on the 8-bit cache, captured into a CUDA graph without a call before them: the kernels are
opted into their shared memory at their first launch, which a capture has to allow."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CODE = """
import sys
sys.path[:0] = ["tests"]
import torch
import kv8_cases as kc
from paper_2609_09338_gb300 import binding as ob
R, dt = int(sys.argv[1]), getattr(torch, sys.argv[2])
ctx = kc.make_ctx(8, 2, 128)
tab, n = kc.table(3, 20, 1)
kv = ob.alloc_kv8(ctx.shape, tab, n)
gen = torch.Generator(device="cuda").manual_seed(0)
rows = [kc.rows(gen, (1, 3 * R + 200, 2, 128), dt) for _ in range(2)]
q = kc.rows(gen, (3, R, 8, 128), dt)
cnt = torch.tensor([R, R + 200, R], dtype=torch.int32, device="cuda")
qn = torch.full((3,), R, dtype=torch.int32, device="cuda")
st = torch.zeros(1, dtype=torch.int32, device="cuda")
out = [torch.zeros_like(q) for _ in range(2)]
torch.cuda.synchronize()
def go(o):
    kv.seq_len.zero_()
    ob.osprey_kv8_append(ctx, kv, cnt, *rows, st)
    ob.osprey_kv8_attend(ctx, kv, 0, qn, q, o, st, rotate=True)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    go(out[0])
g.replay()
torch.cuda.synchronize()
go(out[1])
torch.cuda.synchronize()
assert int(st.item()) == 0 and torch.equal(out[0], out[1]) and out[0].any()
print("captured")
"""


@pytest.mark.parametrize("R,dtype", [(1, "bfloat16"), (7, "bfloat16"), (3, "float32")])
def test_first_call_captured(R, dtype):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CODE, str(R), dtype], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
