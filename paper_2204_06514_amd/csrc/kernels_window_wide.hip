// dQ of the window attention at head widths above 128, in a file of its own: here the compiler may keep the accumulators in the upper half of the
// registers, where the products' factors of two tiles, dQ and the rows' own operands fit all 512 (in the lower half alone 512 bytes a lane go to scratch).
// Backward pass, us, with them in the lower half | here: 2 x 4096 positions, 16 heads on 4 of 256, window 1024  938 | 657; 4 x 1000, 8 heads of 192, window
// 300  132 | 93.  (The forward pass fits either way, and loses a tenth to moving scores between the halves: 178 | 200.)
#include "window_dq_mfma.h"

namespace fax {

int window_dq_wide(const WindowArgs& a, int waves, int splits, float* part_dq, float* part_ds, hipStream_t s) {
  return dq_launch<256, true>(a, waves, 1, splits, part_dq, part_ds, s);
}

}  // namespace fax
