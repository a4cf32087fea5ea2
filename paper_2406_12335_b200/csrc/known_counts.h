// Answers of the runtime that hold for a device and a number, asked for once.  Host code only.
#pragma once
#include <atomic>

namespace vatp {

// One table per kernel: what runs at once depends on its registers and shared memory.
template <int DEVICES, int NUMBERS> class KnownCounts {
 public:
  // ask() tells how many, or a negative number where that could not be told: then 0, and the next call asks again
  template <typename Ask> int get(int dev, int number, Ask ask) {
    std::atomic<int>* entry = dev >= 0 && dev < DEVICES && number >= 0 && number < NUMBERS ? &known_[dev][number] : nullptr;
    const int before = entry ? entry->load(std::memory_order_relaxed) : 0;
    if (before) return before - 1;
    const int n = ask();
    if (n < 0) return 0;
    if (entry) entry->store(n + 1, std::memory_order_relaxed);
    return n;
  }

 private:
  std::atomic<int> known_[DEVICES][NUMBERS] = {};      // the answer and one; 0: not asked
};

}  // namespace vatp
