"""Packed tensors of an AdamW launch: every word that a kernel reads of a record, the last one's
included, lies in the launch's words, and a launch takes what the header says."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")

PROGRAM = """
#include <cstdio>
#include "hilore_internal.hpp"
int main() {
  std::printf("%d %d\\n", hilore::kAdamwWords, hilore::kAdamwRecord);
  for (int stride : {9, 11, 12, 14}) std::printf("%d %d\\n", stride, hilore::adamw_capacity(stride));
}
"""


def test_records_lie_in_the_words(tmp_path):
    src, exe = tmp_path / "records.cpp", tmp_path / "records"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2609_33570_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True, timeout=60).stdout
    (words, record), *plans = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert record == max(stride for stride, _ in plans)
    for stride, cap in plans:  # [cap] first chunks, then the records
        last = cap + (cap - 1) * stride
        assert last + record <= words, (stride, cap)
        assert last + record + stride + 1 > words, (stride, cap)  # one more would not fit
    assert min(c for _, c in plans) == 67 and max(c for _, c in plans) == 100
