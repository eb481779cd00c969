"""A ring of slots that one warp fills and reads, replayed on the host: the rule of csrc/np_ring.h over a model of its barriers, copies that
land in any order, one of them later than any wait lasts."""
import ctypes as C
import subprocess

import pytest

from paper_2608_22643_b200 import build as nbuild

_SOURCE = r"""
#include <random>
#include <utility>
#include <vector>
#include "np_ring.h"

namespace {
// An mbarrier of one arrival: a phase completes when it is in and no bytes are on their way.
struct Barrier {
  int pending = 1, bytes = 0;
  uint32_t phase = 0;
  bool overrun = false;
  void look() {
    if (pending == 0 && bytes == 0) pending = 1, ++phase;
  }
  void arm(int n) {
    if (pending == 0) overrun = true;
    else --pending;
    bytes += n;
  }
  void land() {
    bytes -= 1;
    look();
  }
  bool complete(uint32_t parity) const { return (phase & 1u) != parity; }
};

constexpr int kLanes = 4;  // lane 0 asks
constexpr uint32_t kLimit = 2000;

template <int kSlots>
struct Warp {
  std::mt19937 rng;
  int late;           // the use whose copies land only after `hold` steps
  long hold, steps = 0;
  bool word = false;
  int reports = 0;
  Barrier full[kSlots];
  int holds[kSlots];
  std::vector<std::pair<int, int>> under_way;  // (slot, use)
  npp::WarpRing<kSlots> lane[kLanes];
  int armed_over_copies = 0, read_wrong = 0, waits_after = 0;

  bool lost() { return word; }
  void lose() { word = true, ++reports; }

  void others() {
    ++steps;
    if (under_way.empty() || rng() % 3 == 0) return;
    const size_t i = rng() % under_way.size();
    const std::pair<int, int> c = under_way[i];
    if (c.second == late && steps < hold) return;
    under_way.erase(under_way.begin() + i);
    holds[c.first] = c.second;
    full[c.first].land();
  }
  void ask() {
    if (!lane[0].may_ask()) return;
    const int use = (int)lane[0].asked, s = (int)lane[0].slot(lane[0].asked++);
    for (const std::pair<int, int>& c : under_way) armed_over_copies += c.first == s;
    full[s].arm(3);
    for (int k = 0; k < 3; ++k) under_way.push_back({s, use});
  }
  void run(unsigned seed, int uses) {
    rng.seed(seed);
    for (int& h : holds) h = -1;
    for (int u = 0; u < kSlots && u < uses; ++u) ask();
    for (int u = 0; u < uses; ++u) {
      bool through[kLanes] = {};
      uint32_t polls[kLanes] = {};
      const bool before = word;
      const long t0 = steps;
      for (int left = kLanes; left > 0;) {  // lanes poll at any pace
        others();
        const int l = (int)(rng() % kLanes);
        npp::WarpRing<kSlots>& r = lane[l];
        if (through[l]) continue;
        if (!full[r.slot(r.used)].complete(r.parity(r.used))) {
          if (!npp::warp_ring_wait_step<kLimit>(polls[l], *this)) continue;
          r.lost = true;
        } else if (!r.lost && holds[r.slot(r.used)] != u) {
          ++read_wrong;
        }
        through[l] = true, --left;
        ++r.used;
      }
      if (before && steps - t0 > 1000) ++waits_after;  // a wait behind the first that was given up
      if (u + kSlots < uses) ask();
    }
    if (lane[0].lost) {  // as npp::drain_ring
      const uint32_t next = lane[0].slot(lane[0].asked), par = lane[0].parity(lane[0].asked);
      for (uint32_t s = 0; s < kSlots; ++s)
        for (long k = 0; k < 1000000 && !full[s].complete(s < next ? par : par ^ 1u); ++k) others();
    }
  }
};

template <int kSlots>
void replay(int seeds, int uses, int late, long hold, int* out) {
  for (int i = 0; i < 6; ++i) out[i] = 0;
  for (int seed = 0; seed < seeds; ++seed) {
    Warp<kSlots> w{};
    w.late = late, w.hold = hold;
    w.run((unsigned)seed, uses);
    out[0] += w.armed_over_copies;
    for (const Barrier& b : w.full) out[0] += b.overrun;
    out[1] += !w.under_way.empty();
    out[2] += w.read_wrong;
    out[3] += w.reports > 0;
    out[4] += w.waits_after;
    out[5] += (int)w.lane[0].asked;
  }
}
}  // namespace

// out: slots armed over copies or barriers out of step, blocks left with copies under way, slots read before they were there, rings that
// reported a wait, long waits behind one that was given up, uses asked for
extern "C" void t_replay(int slots, int seeds, int uses, int late, long hold, int* out) {
  if (slots == 2) replay<2>(seeds, uses, late, hold, out);
  else if (slots == 3) replay<3>(seeds, uses, late, hold, out);
  else replay<4>(seeds, uses, late, hold, out);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("warp_ring")
    src, so = str(out / "t.cpp"), str(out / "t.so")
    with open(src, "w") as f:
        f.write(_SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", nbuild.CSRC, src, "-o", so], check=True)
    lib = C.CDLL(so)
    lib.t_replay.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_long, C.POINTER(C.c_int)]
    return lib


@pytest.mark.parametrize("slots", [2, 3, 4])
@pytest.mark.parametrize("uses", [1, 2, 7, 40])
def test_a_ring_that_is_served_reads_everything(lib, slots, uses):
    out = (C.c_int * 6)()
    lib.t_replay(slots, 200, uses, -1, 0, out)
    assert list(out) == [0, 0, 0, 0, 0, 200 * uses]


@pytest.mark.parametrize("slots", [2, 3, 4])
@pytest.mark.parametrize("late", [0, 1, 2, 5, 38, 39])
@pytest.mark.parametrize("hold", [30000, 60000, 300000])
def test_a_copy_that_comes_after_the_wait_for_it(lib, slots, late, hold):
    """The wait ends and is reported once, nothing is asked for over copies, the warp is soon through and leaves when all have landed."""
    out = (C.c_int * 6)()
    lib.t_replay(slots, 100, 40, late, hold, out)
    assert list(out[:5]) == [0, 0, 0, 100, 0]
    assert out[5] <= 100 * min(40, late + 2 * slots)
