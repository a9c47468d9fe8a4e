"""Layer norm, 8-bit checkpoints and output layers: what the host decides at the edges.  Needs no GPU."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_04930_b200", "csrc")


def _compiled(tmp_path, body):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text(body)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + CSRC, "-o", str(exe), str(src)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()


def test_register_shares_are_held_against_what_the_compiler_gave(tmp_path):
    """The shares of a kernel of 1 + 2 + 2 + 2 warpgroups, launched with 72 registers a thread: with fewer than a `dec` names or
    more than an `inc` names it must not run, nor with a total above the launch's."""
    out = _compiled(tmp_path, """
#include <cstdio>
#include <initializer_list>
#include "register_split.h"
using gcnsa::RegisterShare;
int main() {
  const RegisterShare kernel[4] = {{1, 32, false}, {2, 72, false}, {2, 64, false}, {2, 96, true}};
  for (int launched : {40, 64, 65, 71, 72, 80, 104}) std::printf("%d ", gcnsa::registers_hold(launched, kernel));
  const RegisterShare greedy[2] = {{1, 40, false}, {2, 96, true}}, odd[2] = {{1, 44, false}, {1, 96, true}}, low[2] = {{1, 16, false}, {1, 96, true}};
  std::printf("%d %d %d", gcnsa::registers_hold(72, greedy), gcnsa::registers_hold(72, odd), gcnsa::registers_hold(72, low));
}
""")
    assert out == ["0", "0", "1", "1", "1", "1", "0"] + ["0", "0", "0"]
