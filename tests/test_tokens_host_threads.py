"""Host threads that make a kernel's first calls at the same time, against a fake of the CUDA calls (no GPU)."""
import os
import subprocess

import pytest

from paper_2608_01653_gb300 import build

SOURCE = r"""
#include <stdio.h>
#include <thread>
#include <unistd.h>
#include "hatq_tokens.h"

// one kernel's limit, as CUDA keeps it: a call sets it, to less than it was if so asked
static std::atomic<int> limit(0), asked(0);
extern "C" cudaError_t fake_get_device(int *d) { *d = 0; return cudaSuccess; }
extern "C" cudaError_t fake_set(const void *, cudaFuncAttribute, int bytes) {
    asked.fetch_add(1);
    usleep(bytes < 100000 ? 50000 : 1000);           // the smaller request takes effect after the larger one
    limit.store(bytes);
    usleep(bytes < 100000 ? 0 : 100000);             // and is known to have before that one returns
    return cudaSuccess;
}

int main() {
    static std::atomic<int> allowed[64];
    int kernel = 0, failed = 0;
    auto call = [&](int bytes) {
        if (hatq::allow_shared(&kernel, bytes, allowed) != cudaSuccess || limit.load() < bytes) ++failed;
    };
    std::thread small(call, 64 * 1024), large(call, 128 * 1024);
    small.join();
    large.join();
    call(128 * 1024);                                // and every later one
    call(64 * 1024);
    printf("%d %d %d", failed, limit.load(), asked.load());
}
"""


def test_threads_never_lower_a_kernels_shared_memory(tmp_path):
    cc = build.nvcc()
    toolkit = os.path.dirname(os.path.dirname(os.path.realpath(cc)))
    (tmp_path / "t.cpp").write_text(SOURCE)
    cmd = ["g++", "-std=c++17", "-O1", "-pthread", "-I", os.path.join(toolkit, "include"), "-I", build.INCLUDE, "-I", build.CSRC,
           "-DcudaGetDevice=fake_get_device", "-DcudaFuncSetAttribute=fake_set", str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    for _ in range(5):
        failed, limit, asked = map(int, subprocess.run([tmp_path / "t"], capture_output=True, text=True, check=True).stdout.split())
        assert failed == 0 and limit == 128 * 1024 and asked <= 2
