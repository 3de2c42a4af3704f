// Answers of the device, asked for once a device.  (No CUDA in here: the host compiler can take it by itself.)
#pragma once
#include <atomic>

// How many clusters of `ranks` CTAs run at once, by device and ranks.  ask() answers that, or a number below 0 where it could not be
// told; that is passed on, and asked again at the next call.
template <int MAX_RANKS>
struct SmatRoom {
  static constexpr int DEVICES = 64;
  std::atomic<int> known[DEVICES][MAX_RANKS + 1];      // clusters + 1

  template <typename Ask>
  int operator()(int device, unsigned ranks, Ask ask) {
    if (device < 0 || device >= DEVICES) return ask();
    int n = known[device][ranks].load(std::memory_order_relaxed) - 1;
    if (n >= 0) return n;
    n = ask();
    if (n >= 0) known[device][ranks].store(n + 1, std::memory_order_relaxed);
    return n;
  }
};
