"""Host state that the calls of several threads share (no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

SOURCE = r"""
#include <thread>
#include <vector>
#include "cu_count.hpp"
static hipError_t get(int *v, int to) { *v = to; return hipSuccess; }
extern "C" hipError_t hipGetDevice(int *dev) { return get(dev, 0); }
extern "C" hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { return get(v, 112); }
int main() {
  std::vector<std::thread> ts;
  std::vector<int> n(8);
  for (int i = 0; i < 8; ++i) ts.emplace_back([&n, i] { n[i] = tr::cu_count(); });
  for (auto &t : ts) t.join();
  for (int v : n)
    if (v != 112) return 2;
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="needs g++")
def test_first_calls_of_several_threads(tmp_path):
    """The number of CUs, asked for once, by threads whose first calls come together."""
    src, exe = tmp_path / "threads.cpp", tmp_path / "threads"
    src.write_text(SOURCE)
    base = ["g++", "-std=c++17", "-g", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include",
            f"-I{ROOT}/paper_2607_06601_amd/csrc", str(src), "-o", str(exe), "-lpthread"]
    built = subprocess.run(base + ["-fsanitize=thread"], capture_output=True, text=True)
    if built.returncode != 0 and "tsan" in built.stderr:
        pytest.skip("no thread sanitizer")
    assert built.returncode == 0, built.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    if "unexpected memory mapping" in r.stderr:
        pytest.skip("the thread sanitizer does not run here")
    assert r.returncode == 0 and "data race" not in r.stderr, r.stderr[-3000:]
