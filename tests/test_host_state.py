"""What the library's host side keeps between calls, under several threads and many kernels (a host program; no GPU needed)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(tmp_path, body):
    from paper_2503_00245_b200 import build
    src, exe = tmp_path / "host.cu", tmp_path / "host"
    src.write_text('#include <cstdio>\n#include <thread>\n#include <vector>\n#include "common.cuh"\n'
                   "int main() {\n" + body + "\n}\n")
    flags = [f for f in build.FLAGS if f != "-O3"]
    made = subprocess.run([build.NVCC, *flags, "-I", build.CSRC, str(src), "-o", str(exe)], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=60).stdout.split()


@pytest.mark.skipif(not os.path.exists(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")), reason="needs nvcc")
def test_launches_of_overlapping_calls_are_all_counted(tmp_path):
    out = run(tmp_path, """
  static moe_ctx ctx{};
  std::vector<std::thread> pool;
  for (int i = 0; i < 4; ++i) pool.emplace_back([] { for (int j = 0; j < 1000000; ++j) ctx.launches++; });
  for (auto& t : pool) t.join();
  printf("%llu", (unsigned long long)ctx.launches);""")
    assert out == ["4000000"]


@pytest.mark.skipif(not os.path.exists(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")), reason="needs nvcc")
def test_kernels_beyond_the_mask_of_shared_memory_limits_have_no_bit(tmp_path):
    """(allow_full_smem asks the driver again for each of their launches; with another kernel's bit it would never ask.)"""
    bits = [int(v) for v in run(tmp_path, '  for (int i = 0; i < 70; ++i) printf("%llu ", cosmoe::next_smem_bit());')]
    assert bits[:64] == [1 << i for i in range(64)] and bits[64:] == [0] * 6
