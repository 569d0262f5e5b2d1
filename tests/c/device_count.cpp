// CountPerDevice: once a device, again after a failure, together from many threads.
#include <cstdio>
#include <thread>
#include <vector>

#include "device_once.h"

#define EXPECT(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main() {
  sky::CountPerDevice count, other;
  int calls[70] = {};
  auto at = [&](sky::CountPerDevice& c, int d, int n) { return c(d, [&] { ++calls[d]; return n; }); };
  for (int d = 0; d < 8; ++d)
    for (int r = 0; r < 3; ++r) EXPECT(at(count, d, 70 + d + r) == 70 + d);  // each device its own, the first answer
  for (int d = 0; d < 8; ++d) EXPECT(calls[d] == 1);
  EXPECT(at(other, 0, 5) == 5 && calls[0] == 2);  // nor one kernel for another
  EXPECT(at(count, 63, 0) == 0 && at(count, 63, -1) == -1);  // a failure is not kept
  EXPECT(at(count, 63, 9) == 9 && at(count, 63, 8) == 9 && calls[63] == 3);
  EXPECT(at(count, 64, 1) == 1 && at(count, 64, 2) == 2 && calls[64] == 2);
  sky::CountPerDevice shared;
  std::atomic<int> wrong{0};
  std::vector<std::thread> ts;
  for (int t = 0; t < 8; ++t)
    ts.emplace_back([&, t] { for (int i = 0; i < 1000; ++i) wrong += shared(t & 1, [&] { return 10 + (t & 1); }) != 10 + (t & 1); });
  for (auto& t : ts) t.join();
  EXPECT(wrong == 0);
  return 0;
}
