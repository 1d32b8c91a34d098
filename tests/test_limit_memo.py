"""The memo of kernels' LDS limits, compiled for the host: every kernel of the library on every device of a node is remembered."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r'''
#include <cstdio>
#include "limit_memo.hpp"
static moe::LimitMemo memo;
int main() {
    // 200 kernels (functions lie on 16 bytes) on 8 devices, and on as many devices as there can be places for
    for (int dev = 0; dev < 8; ++dev)
        for (int k = 0; k < 200; ++k) {
            size_t *limit = memo.of(dev, (const void *)(0x7f0000001000 + 16 * k));
            if (!limit || *limit) return 1;
            *limit = 1000 * dev + k + 1;
        }
    for (int dev = 0; dev < 8; ++dev)
        for (int k = 0; k < 200; ++k)
            if (*memo.of(dev, (const void *)(0x7f0000001000 + 16 * k)) != (size_t)(1000 * dev + k + 1)) return 2;
    int kept = 1600;
    for (int k = 1000; k < 10000; ++k) kept += memo.of(0, (const void *)(0x7f0000001000 + 16 * k)) != nullptr;
    if (kept != (int)moe::LimitMemo::kPlaces) return 3;  // (full: told, and nothing is lost)
    for (int dev = 0; dev < 8; ++dev)
        for (int k = 0; k < 200; ++k)
            if (*memo.of(dev, (const void *)(0x7f0000001000 + 16 * k)) != (size_t)(1000 * dev + k + 1)) return 4;
    puts("ok");
}
'''


def test_every_kernel_on_every_device(tmp_path):
    (tmp_path / "memo.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "paper_2605_00686_amd", "csrc"), str(tmp_path / "memo.cpp"),
                    "-o", str(tmp_path / "memo")], check=True)
    assert subprocess.run([str(tmp_path / "memo")], capture_output=True, text=True, check=True).stdout == "ok\n"
