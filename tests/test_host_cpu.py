"""Host code of the library on its own, compiled with the host's compiler against fakes of CUDA's calls."""

import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc")))


def compile_and_run(tmp_path, source):
    (tmp_path / "t.cpp").write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", os.path.join(CUDA, "include"), "-I",
                    os.path.join(ROOT, "paper_2609_31568_gb300", "csrc"), str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")],
                   check=True)
    return subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, timeout=60, check=True).stdout.strip()


def test_first_tensor_maps_of_two_threads(tmp_path):
    """Threads whose first calls need the tensor map encoder at the same time all get it, and it is looked up once."""
    got = compile_and_run(tmp_path, r'''
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>
#include "tma_host.h"

std::atomic<int> calls{0};

extern "C" cudaError_t CUDARTAPI cudaGetDriverEntryPointByVersion(const char*, void** fn, unsigned int, unsigned long long,
                                                                  cudaDriverEntryPointQueryResult* status)
{
    ++calls;
    std::this_thread::sleep_for(std::chrono::milliseconds(300));  // the other threads' calls fall into this
    *fn = reinterpret_cast<void*>(&calls);
    *status = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

int main()
{
    std::atomic<int> found{0};
    std::vector<std::thread> threads;
    for (int i = 0; i < 4; ++i) threads.emplace_back([&] { found += scale_host::tensor_map_encoder() != nullptr; });
    for (auto& t : threads) t.join();
    std::printf("%d %d\n", found.load(), calls.load());
}
''')
    assert got == "4 1"
