"""Answers of the runtime that the 4-bit step keeps: per kernel, per device and size, and only where there was one."""
import os
import re
import subprocess

from tests.test_dependent_launches_cpu import CSRC, _code

PROGRAM = r"""
#include <cassert>
#include "known_counts.h"
int main() {
  static vatp::KnownCounts<2, 4> a, b;
  int asked = 0;
  auto says = [&](int n) { return [&asked, n] { ++asked; return n; }; };
  assert(a.get(0, 1, says(-1)) == 0 && asked == 1);      // no answer
  assert(a.get(0, 1, says(7)) == 7 && asked == 2);       // is asked for again
  assert(a.get(0, 1, says(9)) == 7 && asked == 2);
  assert(b.get(0, 1, says(9)) == 9 && asked == 3);       // another kernel's
  assert(a.get(1, 1, says(3)) == 3 && a.get(0, 2, says(0)) == 0 && asked == 5);
  assert(a.get(0, 2, says(4)) == 0 && asked == 5);       // none fits: that is an answer
  assert(a.get(2, 1, says(5)) == 5 && a.get(-1, 1, says(6)) == 6 && a.get(0, 4, says(8)) == 8 && asked == 8);      // beyond the table
  assert(a.get(2, 1, says(6)) == 6);
}
"""


def test_only_answers_are_kept(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)


def test_every_kernel_has_a_table_of_its_own():
    code = _code("decode_q4.cu")
    launch = code[code.index("cudaError_t launch_gt("):]
    assert "template <typename T, int HD, int GT>" in code[:code.index("cudaError_t launch_gt(")].splitlines()[-1]
    assert "static ClusterCounts known[2];" in launch and re.search(r"kern16 = win \? ", launch)
    assert set(re.findall(r"clusters_at_once\(([^,]*),", launch)) == {"known[win]"}
    assert "static" not in code[code.index("int clusters_at_once("):code.index("cudaError_t launch_gt(")].replace("static_cast", "")
    assert os.path.exists(os.path.join(CSRC, "known_counts.h"))
