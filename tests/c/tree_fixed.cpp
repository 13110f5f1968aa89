// A probability in fixed point against its value, and what is none.  (Built with the compiler's check for undefined shifts.)
#include <cmath>
#include <cstdio>
#include <initializer_list>
#include <limits>

#include "tree_fixed.h"

#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #x); \
      return 1;                                   \
    }                                             \
  } while (0)

int main() {
  bool bad = false;
  // every exponent below 2, a few mantissas: the value's whole units of 2^-62 (exact in an 80-bit or wider sense: at most 2^63)
  for (uint32_t e = 1; e < 128; ++e)
    for (uint32_t m : {0u, 1u, 0x2aaaaau, 0x7fffffu}) {
      const uint32_t bits = e << 23 | m;
      float p;
      std::memcpy(&p, &bits, sizeof(p));
      CHECK(selkv::to_fix(p, bad) == (unsigned long long)std::floor(std::ldexp((double)p, 62)));
    }
  CHECK(selkv::to_fix(0.f, bad) == 0);
  CHECK(selkv::to_fix(std::numeric_limits<float>::denorm_min(), bad) == 0);
  CHECK(selkv::to_fix(-0.f, bad) == 0);  // a zero like any other
  CHECK(!bad);
  for (float p : {2.f, -1e-30f, -1.f, INFINITY, -INFINITY, NAN}) {
    bad = false;
    CHECK(selkv::to_fix(p, bad) == 0 && bad);
  }
  std::printf("done\n");
  return 0;
}
