"""Logits that the kernel in front of a call writes at its very end, after it has let the call's kernel be placed beside it and has read the old
ones on every SM: the call sees the new ones, whatever lies in the SMs' first-level caches."""
import ctypes
import os
import shutil
import subprocess

import pytest

pytestmark = pytest.mark.gpu

SOURCE = r"""
#include <cuda_runtime.h>
// Every CTA reads all of x a number of times, the first one then writes it; nothing waits for anything but time.
__global__ void k_late(uint4* x, const uint4* next, int n, int times, int let_in) {
    for (int t = 0; t < times; t++) {
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            unsigned a, b, c, d;
            asm volatile("ld.global.ca.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "l"(x + i) : "memory");
        }
        if (t == let_in) cudaTriggerProgrammaticLaunchCompletion();
        __nanosleep(1000);
    }
    if (blockIdx.x != 0) return;
    for (int i = 0; i < 20; i++) __nanosleep(1000);
    for (int i = threadIdx.x; i < n; i += blockDim.x) x[i] = next[i];
}
extern "C" int late(void* x, const void* next, int n, int ctas, int times, int let_in, void* stream) {
    k_late<<<ctas, 128, 0, (cudaStream_t)stream>>>((uint4*)x, (const uint4*)next, n, times, let_in);
    return (int)cudaGetLastError();
}
"""
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


@pytest.fixture(scope="module")
def late(tmp_path_factory):
    if not shutil.which(NVCC):
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("late")
    (d / "late.cu").write_text(SOURCE)
    subprocess.check_call([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-o", str(d / "late.so"), str(d / "late.cu")])
    f = ctypes.CDLL(str(d / "late.so")).late
    f.argtypes = [ctypes.c_void_p, ctypes.c_void_p] + 4 * [ctypes.c_int] + [ctypes.c_void_p]
    return f


@pytest.mark.parametrize("let_in", [0, 19])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_scores_and_gradient_of_logits_written_late(late, kind, let_in):
    import torch
    import paper_2607_29678_b200 as tt
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[kind]
    g = torch.Generator(device="cuda").manual_seed(5)
    rows, n = 8, 65_536 // 8 // (4 if kind == "fp32" else 2)                # 64 KB: they fit into a first-level cache
    old, new = (torch.randn((rows, n), generator=g, device="cuda").to(dtype) for _ in range(2))
    ids = torch.randint(0, n, (rows,), generator=g, dtype=torch.int32, device="cuda")
    gl, ge = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    want, dx = tt.alloc_logprobs(rows, 5), torch.zeros_like(new)
    tt.logprobs(new, ids, want)
    tt.logprobs_grad(new, ids, want, gl, dx, grad_entropy=ge)
    torch.cuda.synchronize()
    ctas = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    x, got, dgot = old.clone(), tt.alloc_logprobs(rows, 5), torch.zeros_like(new)
    stream = torch.cuda.current_stream().cuda_stream
    for _ in range(5):
        for call in (lambda: tt.logprobs(x, ids, got), lambda: tt.logprobs_grad(x, ids, {**want, "status": got["status"]}, gl, dgot, grad_entropy=ge)):
            x.copy_(old)
            torch.cuda.synchronize()
            assert late(x.data_ptr(), new.data_ptr(), rows * n * x.element_size() // 16, ctas, 20, let_in, stream) == 0
            call()
            torch.cuda.synchronize()
        assert torch.equal(x, new) and torch.equal(dgot, dx)
        for k in want:
            assert torch.equal(got[k], want[k]), k
