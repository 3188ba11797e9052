// The arithmetic by which attention over a cache is cut into splits (attn_cached.h), apart from the lists that it is worked out from: for the
// device, and for the host as it stands.
#pragma once

#include <stdint.h>

namespace speca {

constexpr int splits_of(int pages, int split_pages) { return pages > split_pages ? (pages + split_pages - 1) / split_pages : 1; }

// What a split can have where `even` pages would make them even: not fewer than `least`, and not more than any sequence has, `most`, from where on
// nothing is cut.  (`even` may pass 32 bits: the pages of every tile together, where there is room for one range.)
constexpr int pages_of_split(int64_t even, int least, int most) { return even <= least ? least : even < most ? static_cast<int>(even) : most > least ? most : least; }

// Few rows: `whole` units if nothing is cut, `work` pages to visit in all.  Splits of work / E pages make at most min(E + whole, 2 E) units of ranges
// that are cut, and
//   whole <= resident / 4:  E = resident - whole: one round of the blocks that fit on the chip
//   otherwise:              the E of R resident - whole, R = 1 to 4, and of 2 resident where that is more than the last of them, whose rounds x
//                           (longest unit + 4 pages that it takes to begin and end one) are fewest
// which is never more than 4 resident units: what the workspace has room for.  (Close to whole = 4 resident the first four leave room for next to
// no range, and a long sequence among short ones whole.  One token of 255 sequences, 8 heads of 128, 254 of 512 tokens and one of 65 536: 413 us
// with the four alone, 99 with the last; of 224 121 and 94; of 200 of up to 1000, where nothing is gained, 47 and 49.)
// count(split_pages, &units, &longest): units of all sequences, and pages of the longest of them (not asked for: nullptr).
struct Cut {
  int split_pages;
  int64_t units;
};
template <typename Count>
constexpr Cut cut_few_rows(int64_t work, int64_t whole, int64_t resident, int least, int most, Count&& count) {
  Cut best{};
  if (4 * whole <= resident) {
    const int64_t ranges = resident - whole;
    best.split_pages = pages_of_split((work + ranges - 1) / ranges, least, most);
    count(best.split_pages, &best.units, static_cast<int*>(nullptr));
    return best;
  }
  int64_t lowest = -1;
  for (int rounds = 1; rounds <= 5; ++rounds) {
    const int64_t ranges = rounds <= 4 ? rounds * resident - whole : 2 * resident;
    if (ranges <= 0 || (rounds == 5 && 4 * resident - whole >= ranges)) continue;
    Cut cut{pages_of_split((work + ranges - 1) / ranges, least, most), 0};
    int longest = 0;
    count(cut.split_pages, &cut.units, &longest);
    const int64_t cost = (cut.units + resident - 1) / resident * (longest + 4);
    if (lowest >= 0 && cost >= lowest) continue;
    lowest = cost;
    best = cut;
  }
  return best;
}

}  // namespace speca
