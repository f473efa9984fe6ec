"""What the library keeps of the process (not of a call) may be asked for by several threads at once."""
import glob
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_27258_gb300", "csrc")
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")

# the driver's entry point, looked up by threads that start together
PROGRAM = r"""
#include <thread>
#include <vector>
#include "tensor_map.h"

static CUresult found(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                      const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill) { return CUDA_SUCCESS; }

extern "C" cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **f, unsigned int, unsigned long long,
                                                        cudaDriverEntryPointQueryResult *qr) {
    *f = reinterpret_cast<void *>(found);
    *qr = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

int main() {
    std::vector<std::thread> threads;
    std::vector<int> wrong(8, 0);
    for (int i = 0; i < 8; ++i)
        threads.emplace_back([&wrong, i] {
            for (int k = 0; k < 1000; ++k) wrong[i] += hla::encode_fn() != found;
        });
    for (auto &t : threads) t.join();
    int sum = 0;
    for (int w : wrong) sum += w;
    return sum ? 1 : 0;
}
"""


def test_one_definition_of_the_entry_point():
    """No file keeps a copy of its own, and nothing unguarded is kept in a function's static variable."""
    for path in glob.glob(os.path.join(CSRC, "*")):
        text = open(path).read()
        assert ("cudaGetDriverEntryPointByVersion" in text) == (os.path.basename(path) == "tensor_map.h"), path
        kept = re.findall(r"^\s+static (?!constexpr|__device__|std::atomic|const |thread_local)[\w: *<>]+ = .*;", text, re.M)
        assert not kept, (path, kept)


def test_entry_point_by_threads(tmp_path):
    if not shutil.which("g++") or not os.path.exists(os.path.join(CUDA, "include", "cuda.h")):
        pytest.skip("no host compiler or CUDA headers")
    (tmp_path / "t.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "t")
    built = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=thread", "-I", CSRC, "-I",
                            os.path.join(CUDA, "include"), str(tmp_path / "t.cpp"), "-o", exe, "-pthread"],
                           capture_output=True, text=True)
    if built.returncode and "tsan" in built.stderr:
        pytest.skip("no thread sanitizer")
    assert built.returncode == 0, built.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    if "unexpected memory mapping" in run.stderr:
        pytest.skip("the thread sanitizer does not run here")
    assert run.returncode == 0 and "data race" not in run.stderr, run.stderr[:2000]
