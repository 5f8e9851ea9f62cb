"""A kernel's shared-memory limit, raised by two host threads at once: the bookkeeping of launch_util.cuh, compiled for the CPU against a stand-in
for the runtime's two calls."""
import ctypes as C
import os
import subprocess
import threading
import time

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "launch_util.cuh"
#include <atomic>
#include <chrono>
#include <thread>

static std::atomic<int> limit{0}, calls{0}, device{0}, slow_from{1 << 30};

extern "C" {
cudaError_t cudaGetDevice(int* d) { *d = device; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int bytes) {
  ++calls;
  limit = bytes;
  if (bytes >= slow_from) std::this_thread::sleep_for(std::chrono::milliseconds(300));
  return cudaSuccess;
}
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes* a, const void*) { a->maxDynamicSharedSizeBytes = limit; return cudaSuccess; }

static uint32_t table[marl::SMEM_OPTIN_DEVICES];
int ensure(uint32_t bytes) { return (int)marl::ensure_dynamic_smem(nullptr, bytes, table); }
void start(int dev, int slow) { device = dev; slow_from = slow; limit = 0; calls = 0; for (auto& t : table) t = 0; }
int now(void) { return limit; }
int count(void) { return calls; }
int noted(int dev) { return (int)table[dev]; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("smem_limit")
    (d / "limit.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2205_05248_b200", "csrc"),
                           "-I", "/usr/local/cuda/include", "-Wl,-Bsymbolic", "-o", str(d / "limit.so"), str(d / "limit.cpp"), "-lpthread"])  # (its own calls, not a loaded runtime's)
    return C.CDLL(str(d / "limit.so"))


def test_the_largest_size_stays_set(lib):
    lib.start(0, 1 << 30)
    for size, limit, calls in ((1000, 1000, 1), (500, 1000, 1), (1000, 1000, 1), (4000, 4000, 2), (1000, 4000, 2)):
        assert lib.ensure(size) == 0 and lib.now() == limit and lib.count() == calls and lib.noted(0) == limit


@pytest.mark.parametrize("device", [0, 63, 64, 200])
def test_a_small_size_beside_a_large_one(lib, device):
    """The large size is being set when another thread asks for a small one: the limit must not end below what is noted or was asked for."""
    lib.start(device, 98304)
    large = threading.Thread(target=lib.ensure, args=(98304,))
    large.start()
    time.sleep(0.1)
    assert lib.ensure(32768) == 0
    large.join()
    assert lib.now() == 98304
    if device < 64:
        assert lib.noted(device) == 98304


@pytest.mark.parametrize("device", [0, 200])
def test_a_large_size_beside_a_small_one(lib, device):
    lib.start(device, 32768)
    small = threading.Thread(target=lib.ensure, args=(32768,))
    small.start()
    time.sleep(0.1)
    assert lib.ensure(98304) == 0
    small.join()
    assert lib.now() == 98304
