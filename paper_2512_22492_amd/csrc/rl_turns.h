// rl_turns.h -- how a work-group's wavefronts learn which piece of work comes next.
// For the host and the device.
#pragma once

#include <stdint.h>

#if defined(__HIP__)
#define RL_TURNS_HD __host__ __device__
#else
#define RL_TURNS_HD
#endif

namespace rl_da {

// One thread writes the place that its work-group takes in turn t, all wavefronts pass a
// barrier and read it.  A turn's work need not hold a barrier, so the writer can reach
// its next write while another wavefront has yet to read: the turns alternate between
// two words, and a word is written again only behind the barrier of the turn between,
// which every wavefront passes after its read.
struct NextPlace {
    int32_t words[2];
    RL_TURNS_HD int32_t& of(int turn) { return words[turn & 1]; }
};

}  // namespace rl_da
