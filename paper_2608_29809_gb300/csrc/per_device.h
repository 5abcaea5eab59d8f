// Facts of the devices that a launch asks for (host code).
#pragma once
#include <atomic>

namespace rc {

// Answers (0 or more) to KINDS questions, kept for each device that gave them.  A
// question that fails (below 0) is asked again by the next call.  Threads may ask
// at once: the same answer is then found twice.
template <int KINDS>
class PerDevice {
 public:
  // What `ask()` answers for the device of this number, -1 where it fails.
  template <class Ask>
  int get(int device, int kind, Ask ask) {
    if (device < 0 || device >= DEVICES || kind < 0 || kind >= KINDS) return ask();
    std::atomic<int>& kept = known_[device][kind];
    int n = kept.load(std::memory_order_relaxed) - 1;
    if (n >= 0) return n;
    n = ask();
    if (n >= 0) kept.store(n + 1, std::memory_order_relaxed);
    return n < 0 ? -1 : n;
  }

 private:
  static constexpr int DEVICES = 64;
  std::atomic<int> known_[DEVICES][KINDS] = {};  // the answer and 1, or 0
};

}  // namespace rc
