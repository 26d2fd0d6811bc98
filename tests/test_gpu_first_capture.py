"""The first call that a process ever makes of an operator on rows may be a captured one: nothing is set up on the side that a capture
forbids, and a replay gives what the call itself gives.  Each in a process of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COMMON = """
import torch
from paper_2609_37007_gb300 import mcd
D, F8 = torch.device("cuda:0"), torch.float8_e4m3fn
g = torch.Generator(device=D).manual_seed(0)
z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device=D)
x = lambda *s, dtype=torch.float32: torch.randn(s, generator=g, device=D).to(dtype)
err = z(1, dtype=torch.int32)
"""
END = """
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=side):
    call(side)
assert all((o == 0).all().item() for o in seen())
graph.replay()
torch.cuda.synchronize()
first = [o.clone() for o in seen()]
for o in seen():
    o.zero_()
call(None)
torch.cuda.synchronize()
assert err.item() == 0 and all(torch.equal(a, b) and (a != 0).any().item() for a, b in zip(first, seen()))
print("same")
"""
CALLS = {
    "norm": """
a, y, s = x(300, 4096), z(300, 4096, dtype=F8), z(300)
call = lambda st: mcd.mcd_norm_rows(a, y, y_scale=s, stream=st)
seen = lambda: [y.view(torch.uint8), s]
""",
    "gemm_tile": """
a, b, y = x(1024, 512).to(F8), x(4, 512).to(F8), z(4, 1024)
call = lambda st: mcd.mcd_tc_gemm_e4m3(a, b, y, err, stream=st)
seen = lambda: [y]
""",
    "gemm_pair": """
a, b, y = x(4096, 256).to(F8), x(1500, 256).to(F8), z(1500, 4096, dtype=torch.bfloat16)
call = lambda st: mcd.mcd_tc_gemm_e4m3(a, b, y, err, stream=st)
seen = lambda: [y]
""",
    "sample": """
a, u, ids, p = x(6, 50000), torch.rand(6, dtype=torch.float64, device=D), z(6, dtype=torch.int32), z(6)
t = torch.full((6,), 0.9, device=D)
call = lambda st: mcd.mcd_sample_rows(a, u, ids, err, top_p=t, probs=p, stream=st)
seen = lambda: [ids, p]
""",
    "window": """
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=D)
k, v = x(1, 90, 2, 16, 64, dtype=torch.bfloat16), x(1, 90, 2, 16, 64, dtype=torch.bfloat16)
kv, ch = mcd.paged_kv(k, v), mcd.chunks(i32([list(range(45)), list(range(45, 90))]), i32([600, 500]), i32([0, 1, 101]), 101, 100, 720)
q, o = x(101, 256, dtype=torch.bfloat16), z(101, 256, dtype=torch.bfloat16)
space = torch.zeros(mcd.mcd_paged_attention_window_workspace(kv, ch, 4, 100, 4), dtype=torch.uint8, device=D)
call = lambda st: mcd.mcd_paged_attention_window(kv, 0, ch, 4, q, o, 0.125, 100, 4, space, err, stream=st)
seen = lambda: [o]
""",
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_first_call_that_is_captured(name):
    r = subprocess.run([sys.executable, "-c", COMMON + CALLS[name] + END], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
