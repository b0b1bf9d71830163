"""The dynamic shared-memory limit of a kernel whose calls need different sizes: raised, never lowered, whatever two threads' first calls do."""
import os
import subprocess
import sys

import pytest

from paper_2506_05413_b200 import build

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>

#include "common.cuh"

// the runtime, faked: the limit of the one kernel on either of two devices
static std::atomic<int> g_limit[2], g_sets{0}, g_first{0}, g_second{0};
static thread_local int t_dev = 0;
extern "C" cudaError_t cudaGetDevice(int* dev) { *dev = t_dev; return cudaSuccess; }
extern "C" cudaError_t cudaGetLastError() { return cudaSuccess; }
extern "C" cudaError_t cudaDeviceGetAttribute(int*, cudaDeviceAttr, int) { return cudaErrorUnknown; }
extern "C" cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int bytes) {
  if (bytes > 1000) return cudaErrorInvalidValue;
  if (bytes == 100 && t_dev == 0) {      // held up until the other thread's call is over, or half a second
    g_first = 1;
    for (int i = 0; i < 500 && g_second == 0; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
  }
  g_limit[t_dev] = bytes;
  ++g_sets;
  return cudaSuccess;
}

int main() {
  static const char kern = 0;
  std::thread small([] { smoothrot::allow_dynamic_smem(&kern, 100); });
  while (g_first == 0) std::this_thread::yield();
  std::thread large([] {
    smoothrot::allow_dynamic_smem(&kern, 200);
    g_second = 1;
  });
  small.join();
  large.join();
  const bool again = smoothrot::allow_dynamic_smem(&kern, 200);
  std::printf("limit %d %d\n", int(again), g_limit[0].load());
  const int sets = g_sets;
  for (int bytes : {50, 100, 150, 200})
    if (!smoothrot::allow_dynamic_smem(&kern, bytes)) return 1;
  std::printf("known %d\n", int(g_sets == sets && g_limit[0] == 200));
  const bool refused = !smoothrot::allow_dynamic_smem(&kern, 2000), more = smoothrot::allow_dynamic_smem(&kern, 300);
  std::printf("raised %d %d %d\n", int(refused), int(more), g_limit[0].load());
  t_dev = 1;
  const bool there = smoothrot::allow_dynamic_smem(&kern, 100);
  std::printf("other device %d %d %d\n", int(there), g_limit[1].load(), g_limit[0].load());
}
"""


def test_two_threads_with_a_faked_runtime(tmp_path):
    source, program = tmp_path / "limit.cpp", str(tmp_path / "limit")
    source.write_text(PROGRAM)
    cuda = os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-x", "c++", str(source), "-o", program, "-I" + build.CSRC, "-I" + os.path.join(build.ROOT, "include"),
                    "-isystem" + cuda], check=True)
    out = subprocess.run([program], capture_output=True, text=True, timeout=60, check=True).stdout
    assert out.splitlines() == ["limit 1 200", "known 1", "raised 1 1 300", "other device 1 100 300"]


CALLS = """
import ctypes, threading, torch
from paper_2506_05413_b200 import binding
lib = binding.load()
D, M = "cuda:0", 4096
ptr = lambda t: ctypes.c_void_p(t.data_ptr())
work = {}
for k in (4096, 8192):
    torch.manual_seed(k)
    y, h = (torch.randn(M, k, device=D).half() for _ in range(2))
    work[k] = (y, h, torch.empty_like(y), torch.empty(M, k // 2, dtype=torch.uint8, device=D), torch.zeros(M * k // 32, dtype=torch.uint8, device=D))
def call(k, stream):
    y, h, out, q, s = work[k]
    return lib.smoothrot_add_norm(ptr(y), k, ptr(h), k, M, k, 1, None, None, 0.5, 1.0, None, 1e-5, ptr(out), k, None, k, 32, 0.9, ptr(q), ptr(s), None,
                                  ctypes.c_void_p(stream.cuda_stream))
streams = {k: torch.cuda.Stream() for k in work}
torch.cuda.synchronize()
gate, got = threading.Barrier(2), []
def first(k):
    gate.wait()
    got.append(call(k, streams[k]))
threads = [threading.Thread(target=first, args=(k,)) for k in work]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
for k, (y, h, out, q, s) in work.items():
    once = out.clone(), q.clone(), s.clone()
    got.append(call(k, streams[k]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(once, (out, q, s)))
    z = y.double()
    want = h.double() + 0.5 * z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-5)
    # half a step of fp16, and six roundings to fp32 of numbers below 16
    assert bool(((out.double() - want).abs() <= 2.0 ** -11 * want.abs() + 6 * 2.0 ** -20).all())
assert got == [0] * 4, got
print("both")
"""


@pytest.mark.gpu
def test_two_widths_from_two_threads_in_a_fresh_process():
    build.build()
    for _ in range(3):
        done = subprocess.run([sys.executable, "-c", CALLS], capture_output=True, text=True, timeout=300, cwd=build.ROOT)
        assert done.returncode == 0 and "both" in done.stdout, done.stderr[-2000:]
