// What a thread remembers of (kernel, device) pairs (host only).
#pragma once
#include <cstddef>
#include <cstdint>

namespace rt {

// A hash table of fixed size: the library has some two hundred kernels with dynamic shared memory, most of them the shapes of a rotation's pass, and a process may meet
// them all.  What does not fit any more is not remembered.
struct KnownKernels {
  struct Entry { const void* fn; int dev, bytes; };
  static constexpr unsigned kSlots = 1024, kMost = kSlots - kSlots / 4;
  Entry tab[kSlots] = {};
  unsigned used = 0;

  // the pair's entry, or the free one where it belongs (fn is null there)
  Entry* at(const void* fn, int dev) {
    uint64_t h = ((uint64_t)reinterpret_cast<uintptr_t>(fn) >> 3) * 64 + (unsigned)dev;
    h *= 0x9e3779b97f4a7c15ull;
    unsigned i = (unsigned)(h >> 54);
    while (tab[i].fn && (tab[i].fn != fn || tab[i].dev != dev)) i = (i + 1) % kSlots;
    return &tab[i];
  }
  void put(Entry* e, const void* fn, int dev, int bytes) {
    if (used >= kMost) return;                                       // (so that a search always meets a free entry)
    *e = {fn, dev, bytes};
    ++used;
  }
};

}  // namespace rt
