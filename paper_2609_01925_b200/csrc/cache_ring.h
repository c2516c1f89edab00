// The two rings between the loads and the products of the tile kernel (cache_prefill.cu), in plain C++ so that a test can run
// their protocol on the host: halves of pages as codes (raw), and as 16-bit operands (conv).
//
// Two pairs of converter warps share the loads.  A wait on an mbarrier names only the parity of the phase it waits for, so it
// is sound only for a waiter that has seen every earlier phase of that barrier: before the first phase has completed, the
// other parity reads as done.  Therefore a slot belongs to one pair for good, in both rings (they are equally long, so one
// slot number serves both), and that pair alone waits for the slot's copies and for its consumers.
#pragma once

namespace crisp {

constexpr int kRaw = 6;   // ring of halves as codes (8 KB)
constexpr int kConv = 6;  // ring of converted halves (16 KB)
static_assert(kRaw == kConv, "a load has the same slot in both rings");
// Bit s: the pair of slot s.  Loads alternate between K and V, so three slots each hold two of one kind and one of the other;
// single turns alternate with double ones to keep the loads' order.  (Turns of three measure the same, 1122 us; one kind per
// pair, 1197: V takes longer.)
constexpr unsigned kPairOfSlot = 0b100110;
constexpr unsigned pair_of_slot(unsigned slot) { return kPairOfSlot >> slot & 1u; }

}  // namespace crisp
