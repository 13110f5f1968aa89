// The store of what is made for a buffer: keys that come back are found, whatever the buffers' distances.
#include <cstdio>
#include <initializer_list>

#include "map_store.h"

#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #x); \
      return 1;                                   \
    }                                             \
  } while (0)

static const void* at(uint64_t a) { return reinterpret_cast<const void*>((uintptr_t)a); }

int main() {
  constexpr int kMost = 2048;
  static selkv::MapStore<uint64_t, kMost> s;  // (items: the number of the key)
  uint64_t name = 1;
  // programs of L layers: caches of K and V with two box sizes, q, k and v, at the distances that allocators give
  for (uint64_t stride : {512ull, 4096ull, 1ull << 20, 2ull << 20, 51ull << 20, 1ull << 31})
    for (int layers : {1, 32, 60, 128}) {
      const uint64_t start = name;
      for (int pass = 0; pass < 3; ++pass) {
        int made = 0;
        uint64_t n = start;
        for (int l = 0; l < layers; ++l)
          for (int t = 0; t < 7; ++t, ++n) {
            const void* base = at(0x7f0000000000ull + (l * 5ull + (t < 4 ? t / 2 : t - 2)) * stride);
            const int box = t < 4 && t % 2 == 0 ? 64 : 32;
            const uint64_t rows = 8 * (t < 4 ? 25000 : 32) + name * 64;  // (another program's keys are others)
            const uint64_t* found = s.find(base, rows - start % 2, 128, box);
            if (found != nullptr) {
              CHECK(*found == n);
            } else {
              ++made;
              s.put(base, rows - start % 2, 128, box, n);
            }
          }
        // only the first pass makes them, and one more where the store was emptied within the program
        CHECK(pass == 0 ? made == 7 * layers : pass == 1 ? made <= 7 * layers : made == 0);
      }
      name += 7 * (uint64_t)layers;
    }
  // as many keys as it holds, one more, and those that differ in one number alone
  static selkv::MapStore<uint64_t, 64> t;
  for (int round = 0; round < 1000; ++round) {
    for (uint64_t i = 0; i < 64; ++i) t.put(at(round + 1), i, 64, 32, round * 64 + i);
    int left = 0;
    for (uint64_t i = 0; i < 64; ++i) {
      const uint64_t* f = t.find(at(round + 1), i, 64, 32);
      CHECK(f == nullptr || *f == round * 64 + i);
      left += f != nullptr;
    }
    CHECK(left == 64);
  }
  CHECK(t.find(at(1000), 0, 64, 32) != nullptr);
  CHECK(t.find(at(1000), 0, 128, 32) == nullptr && t.find(at(1000), 0, 64, 64) == nullptr && t.find(at(1000), 64, 64, 32) == nullptr);
  CHECK(t.find(nullptr, 0, 64, 32) == nullptr);
  t.put(at(1000), 0, 64, 32, 7);  // a key that is there takes its own place
  CHECK(*t.find(at(1000), 0, 64, 32) == 7 && t.find(at(1000), 63, 64, 32) != nullptr);
  std::printf("done\n");
  return 0;
}
