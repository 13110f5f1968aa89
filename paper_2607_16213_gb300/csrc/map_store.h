// What was made for a buffer's rows, kept by what it depends on: plain C++, so that it can be tested without a device.
#pragma once

#include <cstdint>

namespace selkv {

// An item a key (base, rows, d, box).  Up to kMost keys that come back are always found: none takes another one's place.  The
// next one empties the store, and what is still in use is made once more (programs hold two to seven maps a layer).  Open
// addressing in twice as many places: a search looks at 1.5 of them on the average when it finds the key, 2.5 when it does not.
template <typename Item, int kMost>
class MapStore {
  static constexpr uint32_t kPlaces = 2 * kMost;
  static_assert((kMost & (kMost - 1)) == 0, "places by a mask");
  struct Entry {
    const void* base;
    uint64_t rows;
    int32_t d, box;
    uint64_t filling;  // in which it was put in
    Item item;
  };
  Entry entries_[kPlaces];
  uint64_t filling_ = 1;  // since the store was emptied for the last time (entries start at 0: not in use)
  uint32_t used_ = 0;

  // The key's place, or the one where it belongs (there is always one).
  Entry& place(const void* base, uint64_t rows, int d, int box) {
    uint64_t h = reinterpret_cast<uintptr_t>(base) >> 4;
    h = (h ^ rows * 31u ^ (uint64_t)(d * 257 + box) * 7919u) * 0x9E3779B97F4A7C15ull;
    uint32_t i = (uint32_t)(h >> 40) & (kPlaces - 1);
    for (;; i = (i + 1) & (kPlaces - 1)) {
      Entry& e = entries_[i];
      if (e.filling != filling_ || (e.base == base && e.rows == rows && e.d == d && e.box == box)) return e;
    }
  }

 public:
  // The item of a key, or nullptr.
  const Item* find(const void* base, uint64_t rows, int d, int box) {
    const Entry& e = place(base, rows, d, box);
    return e.filling == filling_ ? &e.item : nullptr;
  }
  void put(const void* base, uint64_t rows, int d, int box, const Item& item) {
    Entry* e = &place(base, rows, d, box);
    if (e->filling != filling_) {
      if (used_ == kMost) {
        ++filling_;
        used_ = 0;
        e = &place(base, rows, d, box);
      }
      ++used_;
    }
    e->base = base;
    e->rows = rows;
    e->d = d;
    e->box = box;
    e->filling = filling_;
    e->item = item;
  }
};

}  // namespace selkv
