// A wait on the barriers of a ring of shared-memory slots that bulk copies fill: its rule alone, without the hardware.
// np_pipe.cuh puts mbarriers under it, tests/test_ring_replay.py a model that replays it on the host.  At the end of the file the same for a
// ring that one warp fills and reads (np_attn_decode.cu; tests/test_warp_ring_replay.py).
//
// A slot has two barriers: `full` (the lane that fills the ring arms it, the copies complete it) and `empty` (its readers).  A
// barrier's parity tells the phase before the current one from the current one and nothing older, so a wait means what it says only
// while the ring keeps step: no slot is armed while copies are on their way into it.  Else `full` loses count of its phases, and
// with it the last means to tell when the block's shared memory is its own again; the block could leave before its copies.
//
// So a wait on these two barriers is not skipped once another wait of the block has run out, as all others are.  (If readers passed
// slots that they have not waited for, they would give them back ahead of the ring, and the filler's wait for a free slot would be
// over at once, on the parity of another use.)  Nor need it be: what it waits for are copies, and warps of this block that wait for
// nothing else then.  After kLimit polls it lowers the block's flag itself; the warps it waits for may then be at the start of a
// wait as long as that, so it goes on for 2 kLimit and pauses in between.  If that does not end it either, copies are lost;
// then the block gives up its ring.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define NP_RING_FN __device__ __forceinline__
#else
#define NP_RING_FN inline
#endif

namespace npp {

// The step behind a poll that has found the phase not complete; `polls` counts these.  True: the wait is given up.
// Block: stands() tells whether its flag does and lower() lowers it, pause(), given_up() tells whether the ring was given up, give_up().
template <uint32_t kLimit, class Block>
NP_RING_FN bool ring_wait_step(uint32_t& polls, Block& b) {
  if (!b.stands()) {
    if (b.given_up()) return true;
    b.pause();
    if (polls > 3 * kLimit) b.give_up();
  }
  if (++polls == kLimit) b.lower();
  return false;
}

// A ring of kSlots slots of one warp, use u in slot u % kSlots.  One lane asks for copies, all lanes wait for them and read; there is no
// barrier for free slots: a slot is asked for again by the lane that has waited for its last use, behind a barrier of the warp.  So the
// lane asks for nothing more once a wait of its own was given up: the copies of that use may still be on their way.  The warp goes on with
// what lies there (its results are reported as incomplete), no later wait is longer than a poll, and at its end the lane waits for the
// copies that it has asked for.
template <int kSlots>
struct WarpRing {
  uint32_t asked = 0, used = 0;  // uses so far; `asked` is the lane's that asks
  bool lost = false;             // a wait of this lane was given up
  static NP_RING_FN uint32_t slot(uint32_t use) { return use % kSlots; }
  static NP_RING_FN uint32_t parity(uint32_t use) { return use / kSlots & 1u; }
  NP_RING_FN bool may_ask() const { return !lost; }
};

// The step behind a poll that has found a use not complete.  True: the wait is given up.  Warp: lost() tells whether any lane's wait was
// given up, lose() says so and reports it.
template <uint32_t kLimit, class Warp>
NP_RING_FN bool warp_ring_wait_step(uint32_t& polls, Warp& w) {
  if (w.lost()) return true;
  if (++polls < kLimit) return false;
  w.lose();
  return true;
}

}  // namespace npp
