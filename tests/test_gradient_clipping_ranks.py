"""Clipping over ranks: each rank's own parts and what all hold alike, on two gloo ranks on the CPU (plain torch stands in for the kernels)."""
import json
import os
import socket
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WORKER = r'''
import os, sys, json
sys.path.insert(0, os.environ["REPO_ROOT"])
import torch, torch.distributed as dist
from paper_2506_08027_b200 import binding as B
from paper_2506_08027_b200 import dp
rank, world = int(os.environ["RANK"]), int(os.environ["WORLD_SIZE"])
dist.init_process_group("gloo", rank=rank, world_size=world)
calls = []
B.make_grad_items = lambda grads, results=None: list(grads)
B.mxfp8_grad_ws_bytes = lambda items: 64
def sumsq(items, out, ws):
    calls.append("sumsq")
    out[0] = sum(float(t.double().square().sum()) for t in items)
def scale(items, total, max_norm, norm):
    calls.append("scale")
    norm[0] = float(total) ** 0.5
    norm[1] = min(1.0, max_norm / (float(norm[0]) + 1e-6))
    for t in items:
        t.mul_(norm[1])
B.mxfp8_grad_sumsq, B.mxfp8_grad_scale = sumsq, scale
owned = [torch.full((3 + rank,), 1.0 + rank), torch.full((2,), 2.0)]        # 3 * 1 + 2 * 4 and 4 * 4 + 2 * 4
shared = torch.full((5,), 3.0)                                              # 45, once
clipping = dp.GradientClipping(owned, [shared])
norm = clipping.clip(4.0)
print(json.dumps({"norm": float(norm[0]), "factor": float(norm[1]), "owned": float(owned[0][0]) / (1 + rank), "shared": float(shared[0]) / 3, "calls": calls}), flush=True)
dist.destroy_process_group()
'''


def test_two_ranks_share_one_norm():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    procs = []
    for r in range(2):
        env = dict(os.environ, RANK=str(r), WORLD_SIZE="2", MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), REPO_ROOT=ROOT)
        procs.append(subprocess.Popen([sys.executable, "-c", WORKER], env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, cwd=ROOT))
    want = (3 * 1 + 2 * 4 + 4 * 4 + 2 * 4 + 45) ** 0.5
    for p in procs:
        out, err = p.communicate(timeout=300)
        assert p.returncode == 0, err[-3000:]
        got = json.loads(out.strip().splitlines()[-1])
        factor = 4.0 / (want + 1e-6)
        assert abs(got["norm"] - want) <= 1e-6 * want and abs(got["factor"] - factor) <= 1e-6
        assert abs(got["owned"] - factor) <= 1e-6 and abs(got["shared"] - factor) <= 1e-6       # FP32: a few 2^-24
        assert got["calls"] == ["sumsq", "scale"]
