"""The limit of dynamic LDS (csrc/lds_limit.h) on several devices and from several threads, with stand-ins for the two runtime calls that it makes."""
import os
import subprocess

from conftest import ROOT

PROGRAM = r"""
#include "lds_limit.h"
#include <stdio.h>
#include <string.h>
#include <thread>
#include <vector>
thread_local int current = 0;
std::atomic<int> raised[80];
bool fails = false;
extern "C" hipError_t hipGetDevice(int* d) { *d = current; return hipSuccess; }
extern "C" hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute a, int bytes)
{
    if (f != (const void*)&fails || a != hipFuncAttributeMaxDynamicSharedMemorySize || bytes != 131072) return hipErrorInvalidValue;
    if (fails) return hipErrorUnknown;
    ++raised[current];
    return hipSuccess;
}
int main()
{
    std::atomic<uint64_t> done{ 0 };
    auto ask = [&](int device) { current = device; return drf::allow_lds(&fails, 131072, done); };
    fails = true;
    if (ask(0) == hipSuccess) return 1;                 // an error is not taken for done
    fails = false;
    for (int round = 0; round < 3; ++round)
        for (int device : { 0, 1, 7, 63 })
            if (ask(device) != hipSuccess) return 2;
    for (int device : { 0, 1, 7, 63 })
        if (raised[device] != 1) return 3;              // on each of them, once
    for (int i = 0; i < 2; ++i) ask(70);
    if (raised[70] != 2) return 4;
    std::vector<std::thread> threads;
    std::atomic<int> bad{ 0 };
    for (int t = 0; t < 8; ++t) threads.emplace_back([&, t] { for (int i = 0; i < 1000; ++i) { bad += ask(8 + t % 4) != hipSuccess; bad += raised[8 + t % 4] == 0; } });
    for (auto& t : threads) t.join();
    return bad ? 5 : 0;
}
"""


def test_every_device_has_its_limit_raised(tmp_path):
    src, exe = tmp_path / "limit.cpp", tmp_path / "limit"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "paper_2603_25872_amd", "csrc"),
                    str(src), "-o", str(exe), "-pthread"], check=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0
