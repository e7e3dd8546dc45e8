// Host check of csrc/wf_per_device.h; prints the number of violations.
#include <cstdio>
#include <thread>
#include <vector>

#include "wf_per_device.h"

static int violations = 0;
static void want(bool ok, const char *what) {
  if (!ok) ++violations, std::printf("violated: %s\n", what);
}

int main() {
  {
    wf::PerDevice p;
    int calls = 0;
    for (int round = 0; round < 3; ++round)
      for (int dev = 0; dev < 8; ++dev) want(p.get(dev, [&] { return ++calls, 100 + dev; }) == 100 + dev, "each device has its own value");
    want(calls == 8, "set up once for each device");
  }
  {
    wf::PerDevice p;
    int calls = 0;
    want(p.get(1, [&] { return ++calls, 0; }) == 0, "a failure is told");
    want(p.get(1, [&] { return ++calls, 0; }) == 0 && calls == 2, "and not kept");
    want(p.get(1, [&] { return ++calls, 7; }) == 7, "a later call may succeed");
    want(p.get(1, [&] { return ++calls, 9; }) == 7 && calls == 3, "which is kept");
    want(p.get(0, [&] { return 0; }) == 0, "whatever another device has");
  }
  {
    wf::PerDevice p;
    for (int dev : {-1, 64, 1000})
      for (int k = 1; k < 3; ++k) want(p.get(dev, [&] { return k; }) == k, "a device past the table is set up each time");
  }
  {
    wf::PerDevice p;
    std::atomic<int> calls{0}, wrong{0};
    std::vector<std::thread> all;
    for (int t = 0; t < 8; ++t)
      all.emplace_back([&] {
        for (int i = 0; i < 1000; ++i)
          if (p.get(i % 4, [&] { return ++calls, 1 + i % 4; }) != 1 + i % 4) ++wrong;
      });
    for (auto &t : all) t.join();
    want(calls == 4 && wrong == 0, "threads set up once");
  }
  std::printf("%d violations\n", violations);
  return violations != 0;
}
