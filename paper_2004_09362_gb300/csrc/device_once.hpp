// State that belongs to a device rather than to the process.
#pragma once

#include <atomic>
#include <cstdint>

namespace gar {

// The devices for which something has succeeded.
using DeviceSet = std::atomic<uint64_t>;

// f's error (0: none) for a device that is not in the set, which it joins if there was none; 0 for one that is.  (Devices
// from 64 on are never in the set: f is called each time, as by two threads that come at once.)
template <typename F> int once_for_device(DeviceSet &set, int device, F f) {
  const uint64_t bit = device >= 0 && device < 64 ? uint64_t(1) << device : 0;
  if (set.load(std::memory_order_acquire) & bit) return 0;
  const int error = f();
  if (error == 0) set.fetch_or(bit, std::memory_order_release);
  return error;
}

}  // namespace gar
