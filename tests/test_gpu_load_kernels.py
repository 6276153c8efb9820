"""Calls without a handle take no device memory once prox_load_kernels (or prox_ffn_create) has been called.  CUDA loads a
kernel's code when it is first used, so this runs in a process of its own, where nothing has used any of them yet."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import json, sys, time
import torch
from paper_2607_27591_b200 import binding as pb

def w4(rows, cols, group, zeros):
    n = -(-cols // group) if group else 1
    t = lambda *s, dtype: torch.ones(s, dtype=dtype, device="cuda")
    return t(rows, cols // 2, dtype=torch.uint8), t(rows, n, dtype=torch.float16), t(rows, n, dtype=torch.uint8) if zeros else None

calls = {}
N, K = 192, 256
y, x, x16 = torch.empty(8, N, device="cuda"), torch.ones(8, K, device="cuda", dtype=torch.bfloat16), torch.ones(8, K, device="cuda", dtype=torch.float16)
for group in (0, 32, 64, 128):
    for zeros in (False, True):
        w = w4(N, K, group, zeros)
        for B in (1, 4, 5, 8):
            for xt, xb in ((0, x), (2, x16)):
                calls[f"linear {group} {zeros} {B} {xt}"] = lambda w=w, g=group, B=B, xt=xt, xb=xb: pb.prox_w4_linear(w, N, K, g, xb, K, xt, B, y, N, 1)
D, F, k2 = 256, 640, 300
sel = torch.arange(k2, device="cuda", dtype=torch.int32).expand(8, k2).contiguous()
for zeros in (False, True):
    m = [w4(F, D, 128, zeros) for _ in range(3)]
    for B in (1, 2, 3, 5, 8):
        n = pb.prox_w4_stage2_workspace(D, F, B)
        ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(B, D, device="cuda")
        calls[f"ffn {zeros} {B}"] = lambda m=m, B=B, ws=ws, out=out, n=n: pb.prox_w4_stage2_ffn(*m, D, F, 128, x, B, sel, k2, None, k2, out, 1, ws, n)
wb = torch.ones(F, D, device="cuda", dtype=torch.bfloat16)
codes, scales, _ = w4(F, D, 128, False)
calls["quantize"] = lambda: pb.prox_w4_quantize(wb, F, D, 128, codes, scales)
for dt, t in ((0, torch.bfloat16), (1, torch.float32), (2, torch.float16)):
    for rows, V in ((1, 90000), (300, 900)):
        z = torch.ones(rows, V, device="cuda", dtype=t)
        for top in (0, 20):
            tl, ti, en = torch.empty(rows, top, device="cuda"), torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
            calls[f"logprobs {dt} {rows} {top}"] = lambda z=z, dt=dt, rows=rows, V=V, top=top, tl=tl, ti=ti, en=en: pb.prox_token_logprobs(
                z, dt, rows, V, V, 1.0, None, 0, None, en, top, tl, ti)
wd, y1 = torch.ones(F, D, device="cuda", dtype=torch.bfloat16), torch.empty(1, D, device="cuda")
calls["noalloc"] = lambda: pb.prox_stage2_ffn_noalloc(x, wb, wb, wd, D, F, sel, k2, y1, 1)

torch.cuda.synchronize()
if sys.argv[1] == "create":
    wdown = torch.ones(D, F, device="cuda", dtype=torch.bfloat16)
    h = pb.prox_ffn_create(D, F, 1, 1, wb, wb, wdown)
else:
    t0 = time.perf_counter()
    pb.prox_load_kernels()
    print("load ms", 1e3 * (time.perf_counter() - t0), file=sys.stderr)
    pb.prox_load_kernels()
torch.cuda.synchronize()
taken, free = {}, torch.cuda.mem_get_info()[0]
for name, call in calls.items():
    call()
    torch.cuda.synchronize()
    now = torch.cuda.mem_get_info()[0]
    if now != free:
        taken[name] = free - now
    free = now
print(json.dumps({"calls": len(calls), "taken": taken}))
"""


@pytest.mark.parametrize("how", ["load", "create"])
def test_no_call_takes_device_memory_once_its_code_is_loaded(how):
    import __graft_entry__ as entry
    entry.build()
    res = subprocess.run([sys.executable, "-c", SCRIPT, how], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]
    out = json.loads(res.stdout.splitlines()[-1])
    print(res.stderr)
    assert out["calls"] > 80 and out["taken"] == {}, out
