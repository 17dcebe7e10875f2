// How the attention of many new tokens over a paged cache is cut over CTAs.  Plain integer arithmetic, shared with the
// host's tests.
//
// An item is one block of query rows of a sequence, layer and key head: `per` new tokens (fewer in a sequence's last item)
// with all query heads of the key head.  Item i of a sequence at position pos sees its first pos + min((i + 1) per, rows)
// tokens, tile by tile; it takes that many places on a line, and `extra` more for its start and end.  Sums over the
// items of a sequence have a closed form, so a place is found without a list.  The line runs over layers and key heads,
// in each over the sequences, and is cut evenly, or every item is: a part owns the tiles that stand in it.
#pragma once
#include <math.h>

#include "paged_split.h"

namespace think {

// n / parts and n % parts for parts <= 2^15, 16 bits at a time (a 64-bit division is a routine of a hundred instructions, which
// a kernel fetches to run it once)
struct PromptShare {
  int64_t each;
  int rest, parts;
  THINK_HD PromptShare(int64_t n, int parts_) : each(0), rest(0), parts(parts_) {
#ifdef __CUDACC__
#pragma unroll 1
#endif
    for (int i = 48; i >= 0; i -= 16) {
      const uint32_t x = (uint32_t)rest << 16 | (uint32_t)(n >> i & 0xffff), q = x / (uint32_t)parts;
      each = each << 16 | q;
      rest = (int)(x - q * (uint32_t)parts);
    }
  }
  THINK_HD int64_t begin(int i) const { return i * each + (uint32_t)(i * rest) / (uint32_t)parts; }      // floor(i n / parts), i <= parts
};
// place / length for 0 <= place, where the quotient fits 31 bits
THINK_HD int prompt_quotient(int64_t place, int64_t length) {
  int64_t q = (int64_t)((float)place / (float)length);
  while (q * length > place) --q;
  while ((q + 1) * length <= place) ++q;
  return (int)q;
}

// The softmax scale in base 2 as a power of two on the queries, which bf16 ones above 2^-126 / scale take exactly (2^-126 at the least:
// a scale below that leaves all weights alike anyway), and what is left of it on the logits, 1 to 2 for scales up to 1.  A logit then passes fp32 only where
// the formula's does, not the product of a query and a key.  Never 0, so that a masked logit, -infinity, stays what it is.
struct PromptScale {
  int queries;                // exponent
  float logits;
  explicit PromptScale(double scale_log2) {
    int e;
    frexp(scale_log2, &e);
    queries = e - 1 < -126 ? -126 : e - 1 > 0 ? 0 : e - 1;
    logits = (float)ldexp(scale_log2, -queries);
    if (!(logits >= 1.17549435e-38f)) logits = 1.17549435e-38f;
  }
};

struct PromptCut {
  int extra;                  // places of an item besides its tokens
  static constexpr int tile = 64;       // tokens; tile j stands at slot(j) of its item
  THINK_HD int64_t slot(int64_t j) const { return j == 0 ? 0 : extra + tile * j; }
  THINK_HD int64_t first_tile(int64_t x) const {        // that stands at x or behind
    if (x <= 0) return 0;
    const uint64_t y = (uint64_t)(x - extra + tile - 1 > 0 ? x - extra + tile - 1 : 0);
    const int64_t j = (int64_t)(y >> 6);
    return j < 1 ? 1 : j;
  }
  // Pieces of each item, or 0: the line is cut evenly, in one part for each CTA.  Where there are fewer items than CTAs and none is
  // much longer than others, an item has CTAs of its own, so that none starts and ends two (64 rows over 8192 tokens, 8 items: 36
  // instead of 40 us).  A piece may be without a tile.
  THINK_HD int pieces(int64_t total, int64_t items, int64_t largest, int most) const {
    if (items < 1 || items > most) return 0;
    const int k = most / (int)items;
    if ((largest - extra) * most > total * k) return 0;
    const uint32_t places = (uint32_t)((uint64_t)largest >> 6) + 1, each = (places + k - 1) / k;
    return (int)((places + each - 1) / each);         // no more than shorten the longest piece by a tile
  }
};

struct PromptLine {           // a sequence's items
  int64_t base;               // places of an item besides its tokens of this call: extra + max(pos, 0)
  int rows, per;
  THINK_HD int items() const { return (int)(((int64_t)rows + per - 1) / per); }
  THINK_HD int64_t begin(int64_t i) const { return i * base + per * (i * (i + 1) / 2); }       // of item i < items()
  THINK_HD int64_t cost(int64_t i) const { return base + ((i + 1) * per < rows ? (i + 1) * per : rows); }
  THINK_HD int64_t total() const { return rows > 0 ? begin(items() - 1) + base + rows : 0; }
  THINK_HD int find(int64_t place) const {              // the item that holds a place, 0 <= place < total()
    int lo = 0, hi = items() - 1;
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (begin(mid) <= place) lo = mid; else hi = mid - 1;
    }
    return lo;
  }
};

// Of a CTA: the item that it begins and another ends, if there is one; and what it does with the one that it is in the middle
// of when it begins.
struct PromptDesc {
  int lh, b, item;
  int16_t begins, carries;    // carries: 0 none, 1 ends it, 2 hands it on
  // Whether the item that it begins is one of a call of B sequences and `heads` layers and key heads; its number is looked at
  // with the sequence's rows.  (A CTA whose waits ran out leaves an empty one behind; nothing else may become an address.)
  THINK_HD bool names_item(int B, int heads) const {
    return (begins != 0) & ((uint32_t)b < (uint32_t)B) & ((uint32_t)lh < (uint32_t)heads) & (item >= 0);
  }
};

}  // namespace think
