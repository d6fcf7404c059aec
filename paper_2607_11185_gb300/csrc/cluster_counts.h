// cluster_counts.h - how many clusters of a kernel run at a time, kept by device and shared memory (distill.cu).
// Plain C++, so that it can be checked without a GPU.
#pragma once

#include <atomic>
#include <cstdint>

namespace vcs {

// Answers of one kernel at one cluster size.  They depend on the device, whose parts may differ, and on a block's share of
// shared memory, a multiple of 16 bytes below 256 KB.  An answer takes one word, so that calls at once are safe, at a place
// that its share and device give; another one with the same place takes it over, and the question is asked again.
class ClusterCounts {
 public:
  static constexpr int kPlaces = 32;
  int find(int device, uint32_t share) const {   // 0: not known
    const uint64_t w = words_[place(device, share)].load(std::memory_order_relaxed);
    return w >> 16 == key(device, share) ? (int)(w & 0xffff) : 0;
  }
  void keep(int device, uint32_t share, int count) {
    if (count > 0 && count < 0x10000)
      words_[place(device, share)].store(key(device, share) << 16 | (uint64_t)count, std::memory_order_relaxed);
  }

 private:
  // (the lowest bit is set: no answer's word is 0)
  static uint64_t key(int device, uint32_t share) { return (uint64_t)(uint32_t)device << 15 | (share >> 4) << 1 | 1; }
  static int place(int device, uint32_t share) { return (int)(((share >> 4) + 5u * (uint32_t)device) % kPlaces); }
  std::atomic<uint64_t> words_[kPlaces] = {};
};

}  // namespace vcs
