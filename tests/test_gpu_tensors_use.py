"""The calls over a list of tensors as they are used: the training example, two ranks that hold
different tensors, and a C program."""
import importlib.util
import json
import os
import shutil
import socket
import subprocess
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2412_21124_b200")
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")


def test_training_example():
    spec = importlib.util.spec_from_file_location("clipped_training",
                                                  os.path.join(ROOT, "examples", "clipped_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms, coefs = example.run(steps=60, quiet=True)
    assert sum(losses[-10:]) < 0.6 * sum(losses[:10])
    for norm, coef in zip(norms, coefs):
        assert abs(coef - min(1.0, 1.0 / (norm + 1e-6))) <= 1e-6
    assert min(coefs) < 1.0


WORKER = r"""
import sys, json, datetime
sys.path.insert(0, %(root)r)
import torch, torch.distributed as tdist
import paper_2412_21124_b200 as absnt
from paper_2412_21124_b200 import dist as adist
tdist.init_process_group("gloo", timeout=datetime.timedelta(seconds=120))
rank, dev = tdist.get_rank(), "cuda:0"
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
def tensors(seed):
    g = torch.Generator(device=dev).manual_seed(seed)
    return [torch.randn(s, device=dev, generator=g) for s in ((300, 40), (777,), (50_001,), (3,))]
grads, p = tensors(1), tensors(2)
m, v = [x * 0.1 for x in tensors(3)], [x.square() * 0.1 for x in tensors(4)]
mine = lambda xs: [x.clone() for x in xs[rank::2]]
out = {}
for norm in (2, 1, float("inf")):
    # both ranks' lists as one, against each rank with its own part
    whole = absnt.GradTensors(grads, out=[torch.empty_like(x) for x in grads],
                              params=[x.clone() for x in p], m=[x.clone() for x in m], v=[x.clone() for x in v])
    part = absnt.GradTensors(mine(grads), params=mine(p), m=mine(m), v=mine(v))
    max_norm = 0.25 * float(absnt.abs_grad_norm(whole, norm_type=norm))
    absnt.abs_grad_clip(whole, max_norm, norm_type=norm)
    absnt.abs_grad_adamw(whole, HP, 3, max_norm, norm_type=norm)
    adist.sharded_grad_adamw(part, HP, 3, max_norm, norm_type=norm)
    a = [float(part.norm), float(part.coef)]
    adist.sharded_grad_clip(part, max_norm, norm_type=norm)
    for role in ("params", "m", "v"):
        for x, y in zip(part._keep[1][role], whole._keep[1][role][rank::2]):
            torch.testing.assert_close(x, y, rtol=2e-6, atol=1e-9)
    for x, y in zip(part._keep[0], whole._keep[1]["out"][rank::2]):
        torch.testing.assert_close(x, y, rtol=2e-6, atol=1e-9)
    assert abs(a[0] - float(whole.norm)) <= 1e-6 * a[0] and abs(a[1] - float(whole.coef)) <= 2e-6 * a[1]
    out[str(norm)] = [repr(x) for x in a]
tdist.barrier()
print(json.dumps(out))
"""


def test_two_ranks_with_different_tensors():
    """Two processes share the GPU; their kernels are independent launches and the sums go over gloo."""
    s = socket.socket()
    s.bind(("127.0.0.1", 0))
    port = s.getsockname()[1]
    s.close()
    procs = [subprocess.Popen([sys.executable, "-c", WORKER % {"root": ROOT}],
                              env=dict(os.environ, RANK=str(r), WORLD_SIZE="2", LOCAL_RANK="0",
                                       MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port)),
                              stdout=subprocess.PIPE, stderr=subprocess.PIPE) for r in range(2)]
    outs = []
    for p in procs:
        so, se = p.communicate(timeout=300)
        assert p.returncode == 0, se.decode()[-3000:]
        outs.append(json.loads(so.decode().strip().splitlines()[-1]))
    assert outs[0] == outs[1]  # the same bits on both ranks


C_SOURCE = r"""
#include <stdio.h>
#include <stdlib.h>
#include <cuda_runtime_api.h>
#include "abs_normtest.h"
#define CHECK(x) do { if (!(x)) { fprintf(stderr, "failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)

/* argv[1]: 3 tensors of 1000, 1 and 4097 floats, one after the other; writes 5 norms and the scaled
 * tensors to argv[2] */
int main(int argc, char** argv) {
  const long long sizes[3] = {1000, 1, 4097};
  const size_t total = 5098;
  float host[5098 + 5];
  CHECK(argc == 3);
  FILE* f = fopen(argv[1], "rb");
  CHECK(f && fread(host, 4, total, f) == total);
  fclose(f);
  float *dev, *norms;
  void *work, *plan;
  cudaStream_t st;
  CHECK(cudaMalloc((void**)&dev, 4 * total) == cudaSuccess);
  CHECK(cudaMalloc((void**)&norms, 4 * 5) == cudaSuccess);
  CHECK(cudaStreamCreate(&st) == cudaSuccess);
  CHECK(cudaMemcpyAsync(dev, host, 4 * total, cudaMemcpyHostToDevice, st) == cudaSuccess);
  abs_tensor t[3] = {{0}};
  size_t at = 0;
  for (int i = 0; i < 3; ++i) {
    t[i].data = dev + at;
    t[i].numel = sizes[i];
    t[i].dtype = ABS_F32;
    at += (size_t)sizes[i];
  }
  const size_t bytes = abs_tensors_plan_bytes(t, 3);
  plan = malloc(bytes);
  CHECK(plan && abs_tensors_plan(t, NULL, NULL, NULL, NULL, NULL, 3, plan, bytes) == ABS_OK);
  CHECK(cudaMalloc(&work, abs_tensors_work_bytes(plan)) == cudaSuccess);
  CHECK(abs_tensors_upload(plan, work, st) == ABS_OK);
  CHECK(abs_grad_clip(plan, work, ABS_NORM_2, 0.5, 3.0, NULL, norms, st) == ABS_OK);
  CHECK(cudaMemcpyAsync(host + 5, dev, 4 * total, cudaMemcpyDeviceToHost, st) == cudaSuccess);
  CHECK(cudaMemcpyAsync(host, norms, 4 * 5, cudaMemcpyDeviceToHost, st) == cudaSuccess);
  CHECK(cudaStreamSynchronize(st) == cudaSuccess);
  f = fopen(argv[2], "wb");
  CHECK(f && fwrite(host, 4, total + 5, f) == total + 5);
  fclose(f);
  return 0;
}
"""


def test_from_c(tmp_path):
    assert torch.cuda.is_available()
    src, exe = tmp_path / "clip.c", tmp_path / "clip"
    src.write_text(C_SOURCE)
    subprocess.check_call([shutil.which("gcc"), "-std=c99", "-Wall", "-Werror", "-I",
                           os.path.join(ROOT, "include"), "-I", os.path.join(CUDA, "include"), str(src),
                           "-o", str(exe), "-L", PKG, "-labs_normtest", "-L", os.path.join(CUDA, "lib64"),
                           "-lcudart", "-Wl,-rpath," + PKG + ":" + os.path.join(CUDA, "lib64")])
    x = np.random.default_rng(3).standard_normal(5098).astype(np.float32)
    x.tofile(tmp_path / "in")
    subprocess.check_call([str(exe), str(tmp_path / "in"), str(tmp_path / "out")])
    got = np.fromfile(tmp_path / "out", dtype=np.float32)
    parts = np.split(x.astype(np.float64), [1000, 1001])
    each = np.array([0.5 * np.sqrt((p * p).sum()) for p in parts])
    total = np.sqrt((each ** 2).sum())
    coef = 3.0 / (total + 1e-6)
    np.testing.assert_allclose(got[0], total, rtol=6e-7)
    np.testing.assert_allclose(got[1], coef, rtol=7e-7)
    np.testing.assert_allclose(got[2:5], each, rtol=6e-7)
    np.testing.assert_allclose(got[5:], 0.5 * coef * x, rtol=8e-7)


def test_built_on_a_side_stream(monkeypatch):
    """Calls on the default stream after an upload on another one: it is the default stream that waits
    for the upload, and the results are those of the list."""
    import paper_2412_21124_b200 as absnt
    gen = torch.Generator(device="cuda").manual_seed(21)
    grads = [torch.randn(n, device="cuda", generator=gen) for n in (5000, 33, 1_000_003)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ts = absnt.GradTensors(grads)
    waits = []
    wait_event = torch.cuda.Stream.wait_event
    monkeypatch.setattr(torch.cuda.Stream, "wait_event",
                        lambda self, event: (waits.append(self.cuda_stream), wait_event(self, event))[1])
    expected = torch.cat(grads).double().norm()
    for stream in (None, torch.cuda.default_stream(), 0):
        norm = absnt.abs_grad_norm(ts, stream=stream)
        assert waits.pop() == torch.cuda.default_stream().cuda_stream == 0 and not waits
        assert abs(float(norm) - float(expected)) <= 6e-7 * float(expected)


def test_capture_of_a_given_stream():
    """A call with `stream` on a stream under capture, while another one is current."""
    import paper_2412_21124_b200 as absnt
    grads = [torch.full((n,), 2.0, device="cuda") for n in (50, 9)]
    ts = absnt.GradTensors(grads)
    absnt.abs_grad_norm(ts)  # the first call on a device is made outside of captures
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin(capture_error_mode="thread_local")
    absnt.abs_grad_norm(ts, norm_type=1, stream=side)
    with torch.cuda.stream(side):
        graph.capture_end()
    assert float(ts.norm) == pytest.approx(2 * 59 ** 0.5)  # captured, not run
    graph.replay()
    torch.cuda.synchronize()
    assert float(ts.norm) == 118.0
