// What one launch can number
#pragma once
#include <cstdint>

namespace sig {

// The hardware numbers the threads of a launch in 32 bits
inline bool launchable(int64_t workgroups, int64_t threads) { return workgroups <= 0xffffffffll / threads; }

}  // namespace sig
