// Host model of the rings of the tile kernel: producer, asynchronous copies that land in any order, four converter warps
// (two pairs) and two issuers, stepped in random order.  Barriers count phases and answer waits by parity, as mbarriers do.
// Prints "ok", or what went wrong first.  Build with -DOWNER(load)=... to run another assignment of loads to pairs.
#include <cstdio>
#include <cstdlib>
#include <deque>
#include <random>
#include <vector>

#include "cache_ring.h"

using namespace crisp;
#ifndef OWNER
#define OWNER(load) pair_of_slot((load) % kRaw)
#endif

struct Bar {
  int count, left, phases = 0;
  explicit Bar(int n) : count(n), left(n) {}
  void arrive() {
    if (--left == 0) {
      left = count;
      ++phases;
    }
  }
  bool done(unsigned parity) const { return (phases & 1u) != (parity & 1u); }
};

struct Converter {
  unsigned load = 0;
  bool landed = false, reading = false;  // passed the wait for the copy; passed both waits
};

static const char* run(unsigned seed, unsigned n_loads) {
  std::mt19937 rng(seed);
  std::vector<Bar> raw_full(kRaw, Bar(1)), raw_empty(kRaw, Bar(2)), conv_full(kConv, Bar(2)), conv_empty(kConv, Bar(2));
  std::vector<int> raw(kRaw, -1), conv(kConv, -1);
  std::vector<int> written(kConv, 0);
  std::vector<unsigned> flight;              // loads whose bytes are on their way
  unsigned issued = 0;
  Converter warp[4];
  unsigned used[2] = {0, 0};                 // loads that an issuer has started on
  std::deque<unsigned> busy[2];              // products under way, which complete in order
  unsigned freed[2] = {0, 0};
  const int late = static_cast<int>(rng() % 3) * 40;   // how unwilling copies are to land
  for (long step = 0; freed[0] < n_loads || freed[1] < n_loads; ++step) {
    if (step > 2000000) return "no progress";
    const int who = static_cast<int>(rng() % 12);
    if (who < 3) {
      if (issued < n_loads) {
        const unsigned s = issued % kRaw;
        if (issued < static_cast<unsigned>(kRaw) || raw_empty[s].done(issued / kRaw - 1)) {
          for (const Converter& w : warp)
            if (w.reading && w.load % kRaw == s) return "a slot is filled while it is read";
          raw[s] = -1;
          flight.push_back(issued++);
        }
      }
    } else if (who < 5) {
      if (!flight.empty() && static_cast<int>(rng() % 100) >= late) {
        const size_t i = rng() % flight.size();
        raw[flight[i] % kRaw] = static_cast<int>(flight[i]);
        raw_full[flight[i] % kRaw].arrive();
        flight.erase(flight.begin() + static_cast<long>(i));
      }
    } else if (who < 9) {
      Converter& w = warp[who - 5];
      const unsigned pair = static_cast<unsigned>(who - 5) / 2;
      while (w.load < n_loads && OWNER(w.load) != pair) ++w.load;
      if (w.load >= n_loads) continue;
      const unsigned r = w.load % kRaw, c = w.load % kConv;
      if (!w.reading) {
        if (!w.landed) {  // the waits come one after the other
          w.landed = raw_full[r].done(w.load / kRaw);
          continue;
        }
        if (w.load >= static_cast<unsigned>(kConv) && !conv_empty[c].done(w.load / kConv - 1)) continue;
        for (int i = 0; i < 2; ++i)
          for (unsigned x : busy[i])
            if (x % kConv == c) return "a slot is converted into while products read it";
        w.reading = true;
      } else {
        if (raw[r] != static_cast<int>(w.load)) return "codes of another load are converted";
        conv[c] = static_cast<int>(w.load);
        raw_empty[r].arrive();
        conv_full[c].arrive();
        w.landed = w.reading = false;
        ++w.load;
      }
    } else {
      const int i = who & 1;
      if (rng() % 2 && used[i] < n_loads) {
        const unsigned c = used[i] % kConv;
        if (conv_full[c].done(used[i] / kConv)) {
          if (conv[c] != static_cast<int>(used[i])) return "another load's operands are multiplied";
          busy[i].push_back(used[i]++);
        }
      } else if (!busy[i].empty()) {
        conv_empty[busy[i].front() % kConv].arrive();
        busy[i].pop_front();
        ++freed[i];
      }
    }
  }
  return nullptr;
}

int main() {
  for (unsigned seed = 0; seed < 3000; ++seed)
    if (const char* what = run(seed, 1 + seed % 90)) {
      std::printf("%s (seed %u)\n", what, seed);
      return 0;
    }
  std::printf("ok\n");
}
