"""One-time set-up per device under threads, on the host alone: cudaGetDevice is a stand-in, no CUDA library is linked."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
PROGRAM = r"""
#include "common.cuh"
#include <atomic>
#include <chrono>
#include <thread>
#include <vector>

static thread_local int current = 0;
extern "C" cudaError_t cudaGetDevice(int* device) {
    *device = current;
    return current < 0 ? cudaErrorNoDevice : cudaSuccess;
}

int main() {
    // threads that come while another is at the set-up: none goes on before a set-up of its device has ended
    for (int round = 0; round < 20; ++round) {
        zq::DeviceOnce once;
        std::atomic<int> ready[2] = {{0}, {0}}, early{0};
        std::vector<std::thread> threads;
        for (int t = 0; t < 8; ++t)
            threads.emplace_back([&, t] {
                current = t & 1;
                const bool ok = once.done([&] {
                    std::this_thread::sleep_for(std::chrono::milliseconds(t < 2 ? 5 : 1));
                    ready[current] = 1;
                    return true;
                });
                if (!ok || !ready[current]) ++early;
            });
        for (std::thread& t : threads) t.join();
        if (early) return 1;
        int again = 0;                                   // and no second set-up afterwards
        for (current = 0; current < 2; ++current) once.done([&] { ++again; return true; });
        if (again) return 2;
    }
    // a set-up that failed is tried again; devices without a bit of their own, or unknown ones, repeat it
    zq::DeviceOnce once;
    int calls = 0;
    current = 5;
    if (once.done([&] { ++calls; return false; }) || !once.done([&] { ++calls; return true; }) || !once.done([&] { ++calls; return false; }) || calls != 2) return 3;
    for (int device : {64, -1}) {
        current = device;
        calls = 0;
        for (int i = 0; i < 2; ++i)
            if (!once.done([&] { ++calls; return true; })) return 4;
        if (calls != 2) return 5;
    }
    return 0;
}
"""


def test_no_thread_goes_on_before_a_set_up_has_ended(tmp_path):
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", os.path.join(HERE, "..", "paper_2509_00031_b200", "csrc"), "-I", os.path.join(cuda, "include"),
                    str(src), "-o", str(exe)], check=True, capture_output=True, text=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0
