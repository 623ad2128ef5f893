// Which codes of its rows an 8-bit operand of a grouped product asks for (group_product.h): a step's when the step before it is written to LDS, so that the loads
// have a step's time.  Plain arithmetic, which the host can walk too.
#pragma once

#include "k_order.h"

namespace gan {

constexpr int CODE_STEP = 64;                                     // sum indices a step

// Sum indices k0 .. k_end - 1 of a row, at least one step of them.  Behind the last step it asks for the first again, which is not used: nothing outside the
// row's own codes is read, also where a set of waves has a single step.
struct CodeWalk {
  int k, first;                                                   // of the step that is asked for next, and of the first

  GAN_DEVICE_INLINE void start(int k0) { k = first = k0; }
  // the first step has been asked for
  GAN_DEVICE_INLINE void started(int k_end) { k = k_end - first > CODE_STEP ? first + CODE_STEP : first; }
  // the step that `left` sum indices begin with has been written, and k asked for
  GAN_DEVICE_INLINE void asked(int left) { k = left > 2 * CODE_STEP ? k + CODE_STEP : first; }
};

// The same for loads that have two steps' time: two steps are asked for before the first is written, and each write asks for the step two behind it.  Behind the last
// step it goes on from the first.
struct CodeWalkTwo {
  int k, first, end;                                              // k: of the step that is asked for next

  GAN_DEVICE_INLINE void start(int k0, int k_end) { k = first = k0, end = k_end; }
  // k has been asked for
  GAN_DEVICE_INLINE void asked() { k = k + CODE_STEP < end ? k + CODE_STEP : first; }
};

}  // namespace gan
