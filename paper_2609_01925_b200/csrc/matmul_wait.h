// How long the product's warps that write a tile wait for it (plain C++: a test compares it with the product's own estimates).
#pragma once

namespace crisp {

// 0.4 s, as elsewhere, and as much again for every 2^14 blocks of 128 columns: 24 us for a block, which takes a CTA 0.1 to 0.5 us
// (four times that where CTAs crowd an SM, see plan_split).  Up to 2^21 columns it is 0.4 s.
constexpr unsigned long long tile_wait_ns(int blocks) {
  return 400ull * 1000ull * 1000ull * (1ull + (static_cast<unsigned>(blocks) >> 14));
}

}  // namespace crisp
