"""What a kernel needs before its first launch is done once on every device (no GPU needed: the runtime's answer is faked)."""
import os
import subprocess

import pytest

from conftest import ROOT

PROGRAM = r"""
#include <cstdio>
#include "once.h"
static int device = 0;
static cudaError_t answer = cudaSuccess;
extern "C" cudaError_t CUDARTAPI cudaGetDevice(int *d) { *d = device; return answer; }
int main()
{
    static ris::Once once;
    int calls = 0;
    cudaError_t result = cudaSuccess;
    auto call = [&](int d) { device = d; return once([&] { ++calls; return result; }); };
    auto expect = [&](cudaError_t got, cudaError_t want, int n) {
        if (got != want || calls != n) std::printf("status %d, %d calls; not %d, %d\n", (int)got, calls, (int)want, n);
        return got == want && calls == n;
    };
    bool ok = expect(call(0), cudaSuccess, 1) && expect(call(0), cudaSuccess, 1);
    ok = ok && expect(call(1), cudaSuccess, 2) && expect(call(1), cudaSuccess, 2) && expect(call(0), cudaSuccess, 2);
    result = cudaErrorInvalidValue;  // tried again where it failed
    ok = ok && expect(call(63), cudaErrorInvalidValue, 3) && expect(call(63), cudaErrorInvalidValue, 4);
    result = cudaSuccess;
    ok = ok && expect(call(63), cudaSuccess, 5) && expect(call(63), cudaSuccess, 5);
    ok = ok && expect(call(64), cudaSuccess, 6) && expect(call(64), cudaSuccess, 7);  // past the table: every time
    answer = cudaErrorNoDevice;
    ok = ok && expect(call(0), cudaErrorNoDevice, 7);
    return ok ? 0 : 1;
}
"""


def test_done_once_on_each_device(tmp_path):
    from paper_2607_21927_gb300 import build

    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.nvcc()))), "include")
    if not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
        cuda = "/usr/local/cuda/include"
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", cuda, "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_shared_memory_limits_are_set_per_device():
    """Every kernel of the serving operators that asks for more shared memory than the default does so through it."""
    for name in ("attn_packed.cu", "attn_packed_f32.cu", "cache4.cu", "cache4_evict.cu"):
        text = open(os.path.join(ROOT, "paper_2607_21927_gb300", "csrc", name)).read()
        assert "std::call_once" not in text.replace("std::call_once(once, [] {\n        void *p = nullptr;", "")  # (a driver symbol: the same on all)
        uses = text.count("static Once once;")
        assert uses >= 1 and uses == text.count("= once([")


@pytest.mark.gpu
def test_calls_on_two_devices():
    """One call of each kind on both (skipped where there is one)."""
    import torch

    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    from paper_2607_21927_gb300 import ris

    for dev in ("cuda:0", "cuda:1"):
        with torch.cuda.device(dev):
            for dtype, D in ((torch.float32, 128), (torch.bfloat16, 128), (torch.bfloat16, 64)):
                q, k, v = (torch.randn(40, h, D, device=dev).to(dtype) for h in (4, 2, 2))
                cache = ris.Cache4.empty(2, 2, D, 8192, device=dev)
                with ris.ris_pack_create([30, 10]) as pack:
                    ris.ris_attention_packed(pack, q, k, v, weight_rows=4)
                    ris.ris_cache4_append(cache, pack, k, v, torch.arange(40, dtype=torch.int32, device=dev))
                ris.ris_cache4_attend(cache, q[:2].contiguous())
                ris.ris_cache4_evict(cache, cache, 16, 4)
            ris.ris_device_status()


def test_tile_kernel_is_prepared_per_device():
    text = open(os.path.join(ROOT, "paper_2607_21927_gb300", "csrc", "attn_tile.cu")).read()
    assert text.count("cudaFuncSetAttribute(") == 1 and "static bool" not in text
    assert text.index("static Once once;") < text.index("= once([") < text.index("cudaFuncSetAttribute(")
