"""Two gloo ranks (CPU): the power sums of a norm over both ranks' tensors, joined in rank order."""
import json
import math
import os
import socket
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WORKER = r"""
import sys, json
sys.path.insert(0, %(root)r)
import torch
from paper_2412_21124_b200 import dist as adist
rank, world, _ = adist.init_from_env(backend="gloo")
mine = torch.tensor([[0.1, 1e300, float("nan")], [0.2, 3.0, 7.0]][rank], dtype=torch.float64)
out = {}
for name, norm in (("sum", 2), ("sum1", 1), ("max", float("inf"))):
    out[name] = [repr(float(adist.join_power_sums(x, norm))) for x in mine]
adist.barrier()
print(json.dumps(out))
"""


def test_power_sums_are_joined_in_rank_order():
    s = socket.socket()
    s.bind(("127.0.0.1", 0))
    port = s.getsockname()[1]
    s.close()
    procs = []
    for rank in range(2):
        env = dict(os.environ, RANK=str(rank), WORLD_SIZE="2", LOCAL_RANK=str(rank),
                   MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), OMP_NUM_THREADS="2")
        procs.append(subprocess.Popen([sys.executable, "-c", WORKER % {"root": ROOT}], env=env,
                                      stdout=subprocess.PIPE, stderr=subprocess.PIPE))
    outs = []
    for p in procs:
        so, se = p.communicate(timeout=300)
        assert p.returncode == 0, se.decode()[-2000:]
        outs.append(json.loads(so.decode().strip().splitlines()[-1]))
    assert outs[0] == outs[1]
    for name in ("sum", "sum1"):
        got = [float(x) for x in outs[0][name]]
        assert got[:2] == [0.1 + 0.2, 1e300 + 3.0] and math.isnan(got[2])
    got = [float(x) for x in outs[0]["max"]]
    assert got[:2] == [0.2, 1e300] and math.isnan(got[2])


def test_one_rank_gets_a_copy():
    import torch
    from paper_2412_21124_b200 import dist as adist
    x = torch.tensor([4.0, 9.0], dtype=torch.float64)
    y = adist.join_power_sums(x[1])
    assert y.tolist() == [9.0] and y.data_ptr() != x[1:].data_ptr()
