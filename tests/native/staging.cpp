// Uploads of one thread to two devices in any order: each arrives whole, whatever the buffers' sizes
// and the copies still in flight.  Exit status 0 when every check passed.
#include "staging.h"

#include <cstdio>
#include <random>

int main() {
  std::mt19937 rng(5);
  wisp::Staging stage;
  FakeStream streams[2][2] = {{{0, {}}, {0, {}}}, {{1, {}}, {1, {}}}};
  std::vector<std::vector<int>> sent, got;
  sent.reserve(400);
  got.reserve(400);
  for (int k = 0; k < 400; ++k) {
    fake_device = k < 2 ? k : (int)(rng() % 2);
    std::vector<int> x(1 + rng() % (k % 7 == 6 ? 60000 : 300));
    for (int &v : x) v = (int)rng();
    sent.push_back(x);
    got.emplace_back(x.size(), 0);
    const char *what = stage.upload(x.data(), x.size() * sizeof(int), got.back().data(), &streams[fake_device][rng() % 2]);
    if (what) {
      std::fprintf(stderr, "upload %d to device %d: %s\n", k, fake_device, what);
      return 1;
    }
    std::fill(x.begin(), x.end(), -1);   // the caller's copy may go
    if (k == 1 && fake_waits != 0) {
      std::fprintf(stderr, "the second device's upload waited for the first's\n");
      return 1;
    }
  }
  for (auto &d : streams)
    for (auto &s : d) fake_finish(&s);
  if (sent != got) {
    std::fprintf(stderr, "an upload was lost or overwritten\n");
    return 1;
  }
  std::puts("staging ok");
  return 0;
}
