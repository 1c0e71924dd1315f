// The fault-injection hook of the bounded waits (actkv_debug_inject_stall), read at every launch.
#pragma once

#include <atomic>

#include "tc_ptx.cuh"

namespace actkv {
namespace tc {

// Fault-injection hook of the bounded waits (actkv_debug_inject_stall): while stall_tile >= 0 the K-tile
// producers of every tensor-core score launch, and the loaders of K and V of every tensor-core attend launch, issue no tile from that one
// on (attend: of each stretch), and every wait gives up after `wait_cycles`.  Process-wide, read at launch.
struct StallHook {
  std::atomic<int32_t> stall_tile{-1};
  std::atomic<long long> wait_cycles{WAIT_LIMIT_CYCLES};
};
inline StallHook& stall_hook() { static StallHook h; return h; }

}  // namespace tc
}  // namespace actkv
