// Work that has to be done once on each device (host side, plain C++).
#pragma once

#include <atomic>
#include <cstdint>

namespace jagg {

// Remembers the devices on which a call has succeeded.  Safe with several threads: run() returns
// success only after the call has succeeded on that device, by this thread or by another; two
// threads may both make it.  Devices past the 64th make it every time.
class OncePerDevice {
 public:
  // f() returns its status, whose zero value is success.
  template <class F>
  auto run(int device, F&& f) -> decltype(f()) {
    using Status = decltype(f());
    const uint64_t bit = device >= 0 && device < 64 ? uint64_t(1) << device : 0;
    if (done_.load(std::memory_order_acquire) & bit) return Status{};
    const Status st = f();
    if (st == Status{}) done_.fetch_or(bit, std::memory_order_release);
    return st;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

// Keeps a positive number that a call has found for each device.  Safe with several threads (two may
// both make the call).  Devices past the 64th make it every time.
class NumberPerDevice {
 public:
  // f(&number) returns its status, whose zero value is success; *number is written on success.
  template <class F>
  auto get(int device, int* number, F&& f) -> decltype(f(number)) {
    using Status = decltype(f(number));
    std::atomic<int>* at = device >= 0 && device < 64 ? &known_[device] : nullptr;
    const int known = at ? at->load(std::memory_order_relaxed) : 0;
    if (known > 0) {
      *number = known;
      return Status{};
    }
    int found = 0;
    const Status st = f(&found);
    if (st == Status{}) {
      *number = found;
      if (at) at->store(found, std::memory_order_relaxed);
    }
    return st;
  }

 private:
  std::atomic<int> known_[64] = {};
};

}  // namespace jagg
