// Host-only check of the order that the sampling kernel searches in.  Compiled and run by tests/test_sample_host.py.
#include <cstdio>
#include <cstring>
#include <vector>

#include "mq_sample_order.h"

#define CHECK(cond)                                                  \
  do {                                                               \
    if (!(cond)) {                                                   \
      std::printf("FAILED line %d: %s\n", __LINE__, #cond);          \
      return 1;                                                      \
    }                                                                \
  } while (0)

using namespace mq;

static uint32_t order(float x) {
  uint32_t b;
  std::memcpy(&b, &x, 4);
  return order_of_bits(b);
}
static float value(uint32_t k) {
  const uint32_t b = bits_of_order(k);
  float x;
  std::memcpy(&x, &b, 4);
  return x;
}

struct Some { float x; long n; };
// The place of the value at which `goal` elements are reached, by the bounds that the kernel keeps; how many steps that takes
static int narrow(const std::vector<Some>& row, long goal, uint32_t* place) {
  uint32_t lo = order(-3.402823466e38f), hi = 0;
  for (const Some& s : row) hi = order(s.x) + 1 > hi ? order(s.x) + 1 : hi;
  for (int step = 0; step < 1000; ++step) {
    if (hi - lo <= 1) { *place = lo; return step; }
    const uint32_t from_lo = lo, from_hi = hi;
    for (int k = 0; k < 2; ++k) {
      const float at = value(order_between(from_lo, from_hi, k, 2));
      long count = 0;
      for (const Some& s : row) count += s.x >= at ? s.n : 0;
      if (count < goal) { hi = order(at); continue; }
      lo = order(at);
      break;
    }
  }
  return 1000;
}

int main() {
  const float most = 3.402823466e38f, tiny = 1.401298464e-45f;
  CHECK(order(0.0f) == order(-0.0f) && value(order(-0.0f)) == 0.0f);
  CHECK(order(tiny) == order(0.0f) + 1 && order(-tiny) == order(0.0f) - 1);
  CHECK(value(order(0.0f) - 1) == -tiny && value(order(0.0f) - 1) < 0.0f);
  // every place between the infinities is a number's, and in their order (every 97th, and all around zero)
  const uint32_t first = order(-most), last = order(most);
  CHECK(last - first == 2u * 0x7f7fffffu);
  for (uint64_t k = first; k < last; k += 97) CHECK(order(value((uint32_t)k)) == (uint32_t)k && value((uint32_t)k) < value((uint32_t)k + 1));
  for (uint32_t k = order(0.0f) - 70000; k != order(0.0f) + 70000; ++k) CHECK(order(value(k)) == k && value(k) < value(k + 1));
  // bf16 numbers: 16 bits say their place, without gaps
  uint32_t before = 0;
  for (uint32_t h = 0x7f80; h-- > 0;) {   // from the largest down to 0, then the negative ones
    const uint32_t k = order_of_bits(h << 16);
    CHECK((k & 0xffffu) == 0 && (before == 0 || k == before - 0x10000u));
    before = k;
  }
  for (uint32_t h = 0x8001; h <= 0xff80; ++h) {
    const uint32_t k = order_of_bits(h << 16);
    CHECK((k & 0xffffu) == 0 && k == before - 0x10000u);
    before = k;
  }
  // an interval of two places or more always shrinks, to a third of its places rounded up at most
  for (uint64_t n = 2; n < 1ull << 32; n = n * 5 / 4 + 1) {
    const uint32_t a = order_between(7, 7 + (uint32_t)n, 1, 2) - 7, b = order_between(7, 7 + (uint32_t)n, 0, 2) - 7;
    const uint64_t third = (n + 2) / 3;
    CHECK(a <= b && b > 0 && b < n && a <= third && b - a <= third && n - b <= third);
  }
  // rows of thousands of equal values, where a search goes down to a single place
  for (float equal : {-tiny, tiny, 0.0f, -0.0f, -1.5f, 1.5f, -most, -1.17549435e-38f, 5.0e-39f}) {
    uint32_t place = 0;
    const int steps = narrow({{2.0f, 1}, {equal, 5000}, {-most, 1}}, 50, &place);
    CHECK(steps <= 21 && place == order(equal));
  }
  std::printf("ok\n");
  return 0;
}
