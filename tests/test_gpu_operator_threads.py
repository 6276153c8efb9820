"""Calls without a handle from several host threads at once, each on a stream of its own, from the first use on: results are those of
one thread.  In a new process, where nothing about the device is known yet."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import threading
import torch
from paper_2607_27591_b200 import binding as pb

g = torch.Generator(device="cuda").manual_seed(1)
def w4(rows, cols, group):
    return (torch.randint(0, 256, (rows, cols // 2), device="cuda", generator=g, dtype=torch.uint8),
            (torch.rand(rows, cols // group, device="cuda", generator=g) * 0.02).half(), None)

N, K, D, F, k2, V = 1000, 8192, 512, 1408, 300, 50000
w, m = w4(N, K, 64), [w4(F, D, 128) for _ in range(3)]
x = torch.randn(8, K, device="cuda", generator=g).bfloat16()
xd = x[:, :D].contiguous()
sel = torch.rand(8, F, device="cuda", generator=g).argsort(1)[:, :k2].sort(1).values.to(torch.int32).contiguous()
z = torch.randn(3, V, device="cuda", generator=g)

def work(stream, out):
    s = stream.cuda_stream
    for B in (1, 3, 8):
        y = out[f"linear{B}"]
        pb.prox_w4_linear(w, N, K, 64, x, K, 0, B, y, N, 1, s)
        pb.prox_w4_stage2_ffn(*m, D, F, 128, xd, B, sel, k2, None, k2, out[f"ffn{B}"], 1, out[f"ws{B}"], out[f"ws{B}"].numel(), s)
    pb.prox_token_logprobs(z, 1, 3, V, V, 1.0, None, 0, None, out["entropy"], 9, out["top"], out["index"], s)

def buffers():
    out = {}
    for B in (1, 3, 8):
        out[f"linear{B}"], out[f"ffn{B}"] = torch.zeros(B, N, device="cuda"), torch.zeros(B, D, device="cuda")
        out[f"ws{B}"] = torch.zeros(pb.prox_w4_stage2_workspace(D, F, B), dtype=torch.uint8, device="cuda")
    out["entropy"], out["top"], out["index"] = torch.zeros(3, device="cuda"), torch.zeros(3, 9, device="cuda"), torch.zeros(3, 9, dtype=torch.int32, device="cuda")
    return out

outs, streams, failed = [buffers() for _ in range(6)], [torch.cuda.Stream() for _ in range(6)], []
torch.cuda.synchronize()
start = threading.Barrier(6)
def run(i):
    try:
        torch.cuda.set_device(0)
        start.wait()
        for _ in range(20):
            work(streams[i], outs[i])
    except Exception as e:
        failed.append(repr(e))
threads = [threading.Thread(target=run, args=(i,)) for i in range(6)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
assert not failed, failed
one = buffers()
work(streams[0], one)
torch.cuda.synchronize()
for out in outs:
    for key in one:
        assert key.startswith("ws") or torch.equal(out[key], one[key]), key
print("same")
"""


def test_threads_find_the_same():
    import __graft_entry__ as entry
    entry.build()
    res = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip().endswith("same"), res.stderr[-2000:]
