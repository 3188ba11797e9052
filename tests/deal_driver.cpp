// Drives csrc/deal.h on the host: what few rows over a cache are cut into, for sequences of all kinds.  Prints the first thing that is wrong.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2509_11628_amd/csrc/deal.h"

using namespace speca;

struct Sequence {
  int64_t tiles;
  int pages;
};
struct Dealt {
  int split_pages;
  int64_t units, split_units, cost;
  int longest;
};

static void count_of(const std::vector<Sequence>& s, int heads, int split_pages, Dealt* d) {
  *d = {split_pages, 0, 0, 0, 0};
  for (const Sequence& q : s) {
    const int64_t splits = splits_of(q.pages, split_pages), n = q.tiles * splits * heads;
    d->units += n;
    if (splits > 1) d->split_units += n;
    if (q.tiles) d->longest = std::max<int>(d->longest, static_cast<int>((q.pages + splits - 1) / splits));
  }
}

static Dealt deal(const std::vector<Sequence>& s, int heads, int resident, int least, int most) {
  int64_t work = 0, whole = 0;
  for (const Sequence& q : s) { work += q.tiles * q.pages * heads; whole += q.tiles * heads; }
  const Cut cut = cut_few_rows(work, whole, resident, least, most, [&](int split_pages, int64_t* units, int* longest) {
    if (split_pages < 1) { std::printf("splits of %d pages\n", split_pages); std::exit(1); }
    Dealt d;
    count_of(s, heads, split_pages, &d);
    *units = d.units;
    if (longest) *longest = d.longest;
  });
  Dealt d;
  count_of(s, heads, cut.split_pages, &d);
  if (d.units != cut.units) { std::printf("units\n"); std::exit(1); }
  d.cost = (d.units + resident - 1) / resident * (d.longest + 4);
  return d;
}

int main() {
  const int resident = 512;
  // one long sequence among short ones, up to and past four rounds of whole units: never much more than with any other number of short ones
  for (int heads : {1, 8, 24}) {
    int64_t last = -1;
    for (int n = 2; n * heads <= 5 * resident; ++n) {
      std::vector<Sequence> s(n, {1, 8});
      s[n / 2].pages = 1024;
      const Dealt d = deal(s, heads, resident, 8, 1024);
      if (last >= 0 && d.cost > last + last / 4 + 64) { std::printf("%d sequences, %d heads: cost %lld behind %lld\n", n, heads, (long long)d.cost, (long long)last); return 1; }
      last = d.cost;
    }
  }
  // any sequences: what is cut has room in the workspace, and no split is longer than twice the ranges of all blocks would make it
  std::mt19937 rng(1);
  for (int turn = 0; turn < 20000; ++turn) {
    const int heads = 1 + rng() % 32, n = 1 + rng() % (turn % 3 ? 40 : 700), kind = rng() % 3;
    std::vector<Sequence> s(n);
    int64_t work = 0;
    int most = 0;
    for (Sequence& q : s) {
      q.tiles = rng() % 8 ? 1 + rng() % (kind == 2 ? 40 : 2) : 0;
      q.pages = rng() % (kind ? 64 : 8) ? rng() % 200 : rng() % 20000;
      work += q.tiles * q.pages * heads;
      most = std::max(most, q.pages);
    }
    const Dealt d = deal(s, heads, resident, 8, most);
    if (d.split_units > 4 * resident) { std::printf("%lld units of ranges that are cut\n", (long long)d.split_units); return 1; }
    Dealt even;
    count_of(s, heads, static_cast<int>(std::min<int64_t>(std::max<int64_t>(8, (work + 2 * resident - 1) / (2 * resident)), 1 << 30)), &even);
    even.cost = (even.units + resident - 1) / resident * (even.longest + 4);
    int64_t whole = 0;
    for (const Sequence& q : s) whole += q.tiles * heads;
    if (2 * whole >= resident * 4 && d.cost > even.cost) { std::printf("cost %lld, %lld with ranges for two rounds\n", (long long)d.cost, (long long)even.cost); return 1; }
  }
  // pages of every tile together beyond 32 bits, with room for one range or a few
  for (int n : {2047, 2046, 2000, 1000, 511, 128, 1}) {
    const Dealt d = deal(std::vector<Sequence>(n, {1, 1 << 24}), 1, resident, 8, 1 << 24);
    if (d.split_units > 4 * resident || d.longest < 1) { std::printf("%d sequences of 2^24 pages\n", n); return 1; }
  }
  for (int64_t even : {int64_t{1}, int64_t{1} << 31, int64_t{1} << 32, (int64_t{1} << 32) + 5, int64_t{511} << 24, int64_t{1} << 60})
    for (int most : {0, 5, 1000, 1 << 24}) {
      const int p = pages_of_split(even, 16, most);
      if (p < 16 || p > std::max(16, most) || splits_of(most, p) < 1) { std::printf("%lld pages: splits of %d\n", (long long)even, p); return 1; }
    }
  std::printf("dealing is right\n");
  return 0;
}
