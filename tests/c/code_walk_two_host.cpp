// What an 8-bit operand asks for that is two steps ahead, walked on the host (tests/test_code_walk_two.py).
#include "../../paper_2102_10485_amd/csrc/code_walk.h"

extern "C" void code_walk_two(int k0, int k_end, int writes, int* asked) {
  gan::CodeWalkTwo w;
  w.start(k0, k_end);
  for (int i = 0; i < 2 + writes; ++i) {               // two before the first step is written, and one for each that is
    *asked++ = w.k;
    w.asked();
  }
}
