"""Group norm and the 4-bit operators where nothing has run before: first calls into a capture, and from several threads at once."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

COMMON = """
import sys, threading
sys.path.insert(0, {root!r})
import torch
import paper_2109_00170_b200 as A
dev = torch.device("cuda:0")
def calls(seed, stream, out):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = r(4, 196, 256).to(torch.bfloat16); dy = r(4, 196, 256).to(torch.bfloat16); big = r(1, 150 * 120, 64); w = r(300, 256); deep = r(3, 4096); wd = r(200, 4096)
    y, dx, z = torch.empty_like(x), torch.empty_like(x), torch.empty_like(big)
    mean, rstd, dg, db = torch.empty(4, 32, device="cuda"), torch.empty(4, 32, device="cuda"), torch.empty(256, device="cuda"), torch.empty(256, device="cuda")
    n1, n2 = A.alcs_group_norm_workspace(4, 14, 14, 256, 32, 2), A.alcs_group_norm_workspace(1, 150, 120, 64, 2, 0)
    ws1, ws2 = torch.empty(n1, dtype=torch.uint8, device="cuda"), torch.empty(n2, dtype=torch.uint8, device="cuda")
    q = lambda rows, cols: [torch.empty(b, dtype=torch.uint8, device="cuda") for b in A.alcs_mx4_bytes(rows, cols)]
    qx, qw, qd, qwd = q(784, 256), q(300, 256), q(3, 4096), q(200, 4096)
    p, pd, back = torch.empty(784, 300, device="cuda"), torch.empty(3, 200, device="cuda"), torch.empty(300, 256, device="cuda")
    torch.cuda.synchronize()
    def run(stream):
        A.alcs_group_norm(x, y, 4, 14, 14, 256, 32, None, None, 1e-5, A.ALCS_SILU, 2, mean, rstd, ws1, n1, stream)
        A.alcs_group_norm_backward(x, dy, dx, 4, 14, 14, 256, 32, mean, rstd, None, None, dg, db, A.ALCS_SILU, 2, ws1, n1, stream)
        A.alcs_group_norm(big, z, 1, 150, 120, 64, 2, None, None, 1e-5, 0, 0, None, None, ws2, n2, stream)
        A.alcs_mx4_quantize(y, 784, 256, 256, 2, *qx, stream)
        A.alcs_mx4_quantize(w, 300, 256, 256, 0, *qw, stream)
        A.alcs_mx4_quantize(deep, 3, 4096, 4096, 0, *qd, stream)
        A.alcs_mx4_quantize(wd, 200, 4096, 4096, 0, *qwd, stream)
        A.alcs_mx4_dequantize(*qw, 300, 256, back, 256, 0, stream)
        A.alcs_mx4_product(*qx, 784, *qw, 300, 256, p, None, None, 0, 0, stream)
        A.alcs_mx4_product(*qd, 3, *qwd, 200, 4096, pd, None, None, 0, 0, stream)
    out.extend((run, [y, dx, z, dg, db, back, p, pd]))
"""

CAPTURE = COMMON + """
out, s = [], torch.cuda.Stream()
calls(1, s, out)
run, results = out
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=s):
    run(s)
g.replay()
torch.cuda.synchronize()
first = [t.clone() for t in results]
for t in results: t.fill_(float("nan"))
run(torch.cuda.current_stream())
torch.cuda.synchronize()
assert all(torch.equal(a, b) and not a.isnan().any() for a, b in zip(first, results))
"""

THREADS = COMMON + """
outs = [[] for _ in range(4)]
streams = [torch.cuda.Stream() for _ in outs]
for i, (o, s) in enumerate(zip(outs, streams)): calls(i, s, o)
def work(o, s):
    for _ in range(30): o[0](s)
ts = [threading.Thread(target=work, args=a) for a in zip(outs, streams)]
for t in ts: t.start()
for t in ts: t.join()
torch.cuda.synchronize()
for run, results in outs:
    got = [t.clone() for t in results]
    run(torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and not a.isnan().any() for a, b in zip(got, results))
assert A.alcs_mx4_status() == 0
"""


@pytest.mark.parametrize("script", [CAPTURE, THREADS], ids=["capture", "threads"])
def test_first_calls(alcs, script):
    r = subprocess.run([sys.executable, "-c", script.format(root=ROOT)], capture_output=True, text=True, timeout=120, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
