"""What a launcher sets once (a kernel's limit of dynamic shared memory) is set once
on every device: the helper with a fake of the runtime's current device, on the CPU."""
import os
import shutil
import subprocess

import pytest

from paper_2608_29539_gb300 import build

PROGRAM = r"""
#include <cstdio>
#include "host_common.h"

static int device = 0;
static cudaError_t answer = cudaSuccess;
extern "C" cudaError_t cudaGetDevice(int* d) { *d = device; return answer; }

int main()
{
    static logo::OncePerDevice once, other;
    int calls = 0;
    auto set = [&] { ++calls; return cudaSuccess; };
    auto fail = [&] { ++calls; return cudaErrorInvalidValue; };
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
    for (int i = 0; i < 3; ++i) CHECK(once(set) == cudaSuccess && calls == 1);
    device = 1;  // a second device has its own limit
    CHECK(once(fail) == cudaErrorInvalidValue && calls == 2);  // and a failure is not taken for done
    for (int i = 0; i < 3; ++i) CHECK(once(set) == cudaSuccess && calls == 3);
    device = 0;
    CHECK(once(set) == cudaSuccess && calls == 3);
    CHECK(other(set) == cudaSuccess && calls == 4);
    device = 63;
    for (int i = 0; i < 3; ++i) CHECK(once(set) == cudaSuccess && calls == 5);
    device = 64;  // past the word: each time
    CHECK(once(set) == cudaSuccess && once(set) == cudaSuccess && calls == 7);
    answer = cudaErrorNoDevice;
    CHECK(once(set) == cudaErrorNoDevice && calls == 7);
    return 0;
}
"""


def test_each_device_gets_it_once(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.nvcc()))), "include")
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", build.CSRC, "-I", cuda, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
