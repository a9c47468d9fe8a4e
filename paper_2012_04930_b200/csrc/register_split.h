// Registers of a kernel whose warps take a share each with setmaxnreg.  The shares are constants, and what they are taken from is
// what the compiler gave every thread of the launch: a `dec` to more than that is an illegal instruction, and an `inc`
// beyond the launch's total waits for good.  So the host asks the compiled kernel before its first launch.
#pragma once

namespace gcnsa {

struct RegisterShare {
  int groups, registers;  // warpgroups of the role, registers of each of its threads
  bool inc;               // setmaxnreg.inc or .dec
};

template <int N>
constexpr bool registers_hold(int launched, const RegisterShare (&shares)[N]) {
  launched = (launched + 7) / 8 * 8;  // (given out in units of 8)
  int want = 0, have = 0;
  for (int i = 0; i < N; ++i) {
    const RegisterShare& s = shares[i];
    if (s.registers % 8 != 0 || s.registers < 24 || s.registers > 256) return false;
    if (s.inc ? s.registers < launched : s.registers > launched) return false;
    want += s.groups * s.registers;
    have += s.groups * launched;
  }
  return want <= have;
}

}  // namespace gcnsa
