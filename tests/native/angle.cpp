// The half turns that a position's angle comes to, for the host tests.
#include "mst_angle.h"

extern "C" {
uint64_t turn_a_position(float inv_freq) { return mst_rot::step_of(inv_freq); }
float half_turns(float inv_freq, int pos) { return mst_rot::half_turns(mst_rot::step_of(inv_freq), pos); }
}
