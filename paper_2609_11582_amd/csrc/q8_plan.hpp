// Launch plan of the 8-bit cache's attention: which kernel, how many work-groups share a sequence, and where their
// records lie. Host arithmetic over the call's counts alone.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cstddef>

namespace okvq {

constexpr int kQ8MaxBatch = 1024;    // slots: one thread each in the page kernels
constexpr int kQ8Cols = 16;          // query columns of a tile of the split kernel
constexpr int kQ8WideCols = 64;      // of the wide kernel (a window's or a tree's rows)
constexpr int kQ8PromptCols = 256;   // and of the prompt kernel at most
constexpr int kQ8MaxSplits = 128;
constexpr int kQ8Groups = 512;       // work-groups that a call of few rows is split into
constexpr int kQ8PromptGroups = 256; // and a call of many: one for each compute unit
constexpr int kQ8Record = 128 + 4;   // floats of a column's record: its sums, and (M, m, l, 0)

// Launch order of the slots: first those whose sequence is split (a record takes a split, a tile and a head, and there are
// kQ8Groups at most: 256 slots), then the others with new rows, then those without.
struct Q8Order {
  int split_slots, active_slots, slots;
  int flags;  // kQ8Reordered: places are not the slots themselves; kQ8Uneven: some slot has fewer tiles than the launch
  int most;   // splits of the sequence that has most
};
constexpr int kQ8Reordered = 1, kQ8Uneven = 2;
struct Q8Splits {
  Q8Order order;
  uint32_t part[kQ8Groups / 2 + 2];  // of each split slot: splits << 16 | records of one head in the slots before it
  uint32_t slot[kQ8MaxBatch / 2];    // of each place in the order, two 16-bit numbers a dword; read where kQ8Reordered
};
struct Q8Plan {
  int cols;    // query columns of a tile: rows of a KV head's group, G to a position
  int ntile;   // tiles of the slot that has most rows
  int rows;    // columns that rows have in the first tile
  Q8Splits splits;
};

// What a work-group has to do with a tile of the slot at a place of the order, x its index among the splits; w, next: part[] of
// the place and the one after it, of any others where they are none (constexpr: for the host and the device)
struct Q8Part {
  bool none = true;             // nothing
  int split = 0, nsplit = 1;
  int records = 0;              // records of the slot and head, 0: the one split writes the output rows itself
  int first = 0;                // records of one head in the slots before it
};
constexpr int q8_part_index(int place) { return place < kQ8Groups / 2 ? place : kQ8Groups / 2; }
constexpr Q8Part q8_part(const Q8Order& o, uint32_t w, uint32_t next, int place, int x, int tile) {
  Q8Part p;
  const int first = w & 0xffffu, n = w >> 16, records = (int)(next & 0xffffu) - first;
  const bool shared = place < o.split_slots;
  if (shared && tile * n < records) {  // not the rows that the plan did not count: those have one split without a record
    p.nsplit = n;
    p.records = records;
    p.first = first;
  }
  p.split = shared ? x : 0;
  p.none = place >= o.slots || p.split >= p.nsplit;
  return p;
}
constexpr int q8_slot_at(const Q8Splits& s, int place) { return (s.slot[place >> 1] >> (16 * (place & 1))) & 0xffffu; }

// Split kernel, launched as (splits, heads and tiles, layers): a layer for each split slot; the others share the axis of splits
constexpr int q8_place(const Q8Order& o, int layer, int x) {
  return layer < o.split_slots ? layer : o.split_slots + (layer - o.split_slots) * o.most + x;
}
// Prompt kernel, launched as (width, splits). Slots and heads vary fastest: work-groups go round the 8 XCDs, so a head's tiles
// meet in few L2s; the last tiles, which see most, start first; slots that are split come before the others with rows, and
// these before idle ones, so that all XCDs have work.
struct Q8Tile {
  int place = -1, h = 0, tile = 0;  // place < 0: nothing
};
constexpr Q8Tile q8_tile(const Q8Order& o, int H, int ntile, int width, int w, int x) {
  const int per = H * ntile, shared = o.split_slots * per;
  int from = 0, slots = o.split_slots, at = w;
  if (w >= shared) {
    const int active = (o.active_slots - o.split_slots) * per;
    at = w - shared + x * (width - shared);
    const bool idle = at >= active;
    from = idle ? o.active_slots : o.split_slots;
    slots = (idle ? o.slots : o.active_slots) - from;
    at -= idle ? active : 0;
  }
  Q8Tile t;
  if (at >= slots * per) return t;
  const int units = slots * H, unit = at % units;
  t.tile = ntile - 1 - at / units;
  t.place = from + unit / H;
  t.h = unit % H;
  return t;
}

inline int q8_layers(const Q8Plan& p) {
  const Q8Order& o = p.splits.order;
  return o.split_slots + (o.slots - o.split_slots + o.most - 1) / o.most;
}

// Wide kernel, launched as one row of work-groups: the splits of the plan, dealt to the 8 XCDs (which take work-groups in turn) in
// even shares whose neighbours are tiles of one split, then the tiles that have one split: of all slots, or, where every split
// slot has all tiles split, of the others
struct Q8Units {
  int split, per;      // work-groups that are splits, and of an XCD
  int64_t singles;     // work-groups behind them
  int first_single;    // place of the first slot that may have such tiles
};
struct Q8Unit {
  int place = -1, h = 0, tile = 0;  // place < 0: nothing
  int split = 0, nsplit = 1, records = 0, first = 0;  // as in Q8Part
};
inline Q8Units q8_units(const Q8Plan& p, int H) {
  const Q8Order& o = p.splits.order;
  Q8Units u;
  u.split = (int)(p.splits.part[o.split_slots] & 0xffffu) * H;
  u.per = (u.split + 7) / 8;
  u.first_single = o.split_slots;
  for (int i = 0; i < o.split_slots; ++i)
    if ((int)((p.splits.part[i + 1] & 0xffffu) - (p.splits.part[i] & 0xffffu)) < (int)(p.splits.part[i] >> 16) * p.ntile) u.first_single = 0;
  u.singles = (int64_t)(o.slots - u.first_single) * H * p.ntile;
  return u;
}
inline int64_t q8_wide_groups(const Q8Plan& p, int H) {
  const Q8Units u = q8_units(p, H);
  return 8 * (int64_t)u.per + u.singles;
}
constexpr Q8Unit q8_unit(const Q8Splits& s, const Q8Units& units, int H, int ntile, int64_t id) {
  Q8Unit u;
  if (id < 8 * (int64_t)units.per) {
    const int at = (int)(id & 7) * units.per + (int)(id >> 3);
    if (at >= units.split) return u;
    int lo = 0, hi = s.order.split_slots;  // the last slot whose splits begin at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if ((int)(s.part[mid] & 0xffffu) * H <= at) lo = mid;
      else hi = mid;
    }
    u.place = lo;
    u.first = (int)(s.part[lo] & 0xffffu);
    u.nsplit = (int)(s.part[lo] >> 16);
    u.records = (int)(s.part[lo + 1] & 0xffffu) - u.first;
    const int tiles = u.records / u.nsplit, local = at - u.first * H, rest = local / tiles;
    u.tile = local - rest * tiles;
    u.h = rest / u.nsplit;
    u.split = rest - u.h * u.nsplit;
    return u;
  }
  const int64_t at = id - 8 * (int64_t)units.per, unit = at / ntile;
  const int tile = (int)(at - unit * ntile), place = units.first_single + (int)(unit / H);
  if (place < s.order.split_slots && tile * (int)(s.part[place] >> 16) < (int)((s.part[place + 1] & 0xffffu) - (s.part[place] & 0xffffu)))
    return u;  // split
  u.place = place;
  u.h = (int)(unit % H);
  u.tile = tile;
  return u;
}

constexpr int kFewRows = 32;  // rows of a head that always take the split kernel

// Where the wide kernel's tiles are more than compute units: microseconds of its rounds against those of the kernel that would take
// the call otherwise, from the starts and ends of a work-group and its time a token (256 work-groups at once, of the split
// kernel 512), as measured over the calls that the plan's comment names and six more. tokens: wide tiles x tokens
inline bool q8_wide_is_faster(int64_t rows, int64_t units16, int64_t units64, int64_t units256, double tokens) {
  const double wide = 15.5 * units64 / 256 + 0.0071 * tokens / 256, mean = tokens / units64;
  if (rows <= kFewRows) return wide < (4.0 + 0.0166 * mean) * units16 / 512;
  const double u256 = units256 / 256.0;
  return wide < 8.5 * std::max(1.0, u256) + u256 * mean / 64 * (0.8 + 1.24 * std::min<int64_t>(rows, 256) / 256);
}

// Every split takes the same number of tokens at most, the least that needs no more work-groups than fit the GPU at
// once: a ragged batch is shared evenly (16 sequences of 8704 to 16384 tokens: 46 -> 41 us against as many splits for each).
// Only the slots with new rows count, each with the tiles that its own rows take (one token at 32768 in a cache of 64 slots
// without other rows 71 -> 11.8 us, of 1024 178 -> 14.6; 512 rows in one of 16 slots 1820 -> 257; 512 rows beside 15 single tokens
// at 8192 914 -> 245).
// * The split kernel, 16 columns at a time, up to 32 rows of a head (0.47 to 1.0 of the prompt kernel's time in 97 of 105 calls,
//   1.12 at most, 64 sequences of 2000), and beyond where all its tiles find a place at once and tiles x tokens, its reads of
//   the cache, are few: in 390 calls of 113 to 8192 rows within both bounds it takes 0.36 to 0.84 of the prompt kernel's time
//   (16 positions x 7 heads at 1024 tokens 18.5 -> 9.4 us, a prompt of 100 x 28 heads 11 -> 5.9). With 640 work-groups it
//   takes up to 1.11, with 1152 1.57 (16 prompts of 40), at 2^18.6 tile tokens 1.16 (4 sequences of 2048, 8 heads, 84 rows), at
//   2^19.6 1.6 (16 sequences of 8192, 1 head, 84 rows: 38 us against 23.6). Tiles that only the largest slot has cost the
//   others a work-group each: up to 8192 of them it is faster all the same (100 rows beside 15 single tokens of 4 heads 14.5 us
//   against 25.9, 250 rows beside 63 of 1 head 16.7 against 26.0), with 11000 no longer (one prompt of 100 in 64 slots 16.1 against 10.9).
// * One split up to 4 rounds of a block for each wave, which saves the merge launch (on the device; the host has one launch
//   less to make too): 300 tokens 8.4 -> 6.2 us, 512 8.5 -> 7.0, 1024 8.6 -> 9.2. Windows, whose walk waits for the length: up to 7 (4 heads,
//   windows of 1024: 1 slot 12.3 -> 9.6 us, 16 slots 12.8 -> 9.8, 64 slots 20.5 -> 14.1; of 1500 12.0 -> 11.3; of 1900, 8 rounds, 12.0 ->
//   13.1), and more where many even tiles share the GPU's bandwidth anyway: as many times 7 as there are 64 tiles, and without a limit
//   from 160 tiles on (4 heads, windows of 2000: 24 slots 17.6 -> 16.6, 32 20.8 -> 16.8, 48 25.4 -> 19.3, 64 29.5 -> 24.8; of 4096:
//   32 28.1 and 27.8, 48 40.5 -> 32.8; of 8192: 32 47 and 55, 40 63 -> 62, 48 87 -> 72; 48 sequences of 3000 to 6000 46 -> 40).
//   Trees, which are merged in any case, up to 3: 300 tokens 13.6 -> 11.8, 1000 (4 rounds) 13.7 -> 14.0; and all from 160 tiles on that
//   are even (4 heads x 8192 tokens: 40 slots 66.8 and 67.6, 48 87.8 -> 77.2, 64 103 -> 100; not 96 of 1000 to 2000, 31 and 36).
// * At most 64 splits, as more cost the merge what they save (32768 tokens, 4 heads: 11.2 us, with 128 splits 13.1),
//   but 128 where 64 would leave compute units idle for more than 4 rounds (131072 tokens, 1 head: 18.3 -> 14.4 us).
// * Tiles of 128 columns where short sequences leave compute units idle: a tile of half the columns takes half the time
//   a token (prompts x 28 heads: 512 tokens 24.9 -> 20.9 us, 2048 68.8 -> 62.7; 1024 rows x 28 heads against 4096 tokens 79 -> 111,
//   as every work-group widens all codes). Up to 128 rows the second half of the waves only brings tiles, which is better (120 rows
//   x 8 heads of 16 sequences of 300: 13.4 us, in halves 15.7). Over 122 calls the rule is within 3 % of the better on average; it is wrong
//   by up to 19 % where 256 columns would split 2048 tokens (512 rows x 28 heads 37.3 us, in halves 43.3), and at 256 tiles exactly.
// * A prompt kernel's split has 256 tokens or more, or 512 in sequences below 1024, where a record weighs more than a split
//   saves (512 rows x 28 heads at 512 tokens 20.8 us, in splits of 256 24.4, 4 chunks of 75 at 300 15.8 and 18.8; at 1024 tokens 256
//   rows x 28 heads 26.3 -> 22.8, 2048 tokens 512 rows x 7 heads 25.6 -> 23.1, 8192 tokens 64 rows x 28 heads 34.3 -> 29.9).
// * Where the tiles alone are more than the GPU holds at once, one split each; but sequences of more than twice the mean work of
//   a place are split into such means, as far as there are records (4 heads, one token: 200 sequences of 300 tokens and one of
//   131072 627 -> 38.5 us, 200 spread over 64 to 16384 176 -> 132). From the mean itself on, 200 of 2000 and one of 4096
//   81.7 -> 85.7, 200 even up to 16000 354 -> 348.
// Where rows see a window or precede a tree (span), lens are the tokens that a tile walks (q8_span), and:
// * The wide kernel, 64 columns at a time, takes what the split kernel does not (which has up to 16 rows, and beyond what the second
//   rule above gives it) as long as its tiles find a place at once. Its time goes with the columns rounded up to 64, the
//   prompt kernel's with those rounded up to 256, at much the same rate: 28 rows 83 -> 50 us (16 slots of 16384 tokens x 4 heads, against
//   the split kernel), 112 rows 28 -> 23 (4 heads x 32768 tokens, against the prompt kernel), 280 rows 57 -> 37, 320 rows x 131072 tokens
//   158 -> 111, 448 rows 57 -> 48. Where the rows fill tiles of 256 and the sequence is long it is no faster: 512 rows x 131072 tokens 160 -> 165
//   with int8, 157 -> 153 with e4m3 (at 32768 58 -> 53 and 57 -> 50). With more tiles than compute units it takes more rounds,
//   each with a start and an end, and is taken where that pays (4 heads of 128 slots: 56 rows at 2000 tokens 113 -> 76 us, 28 rows 88 -> 62;
//   not for 112 rows, 134 and 148, nor for 28 rows at 300 tokens, 30 and 33; prompts with windows of 1024 171 and 240).
// * The prompt kernel's tiles of 128 columns where short windows leave compute units idle, or take more than one round of tiles of
//   256, whose last one is seldom full: two work-groups share a compute unit and end one by one (8192 rows x 28 heads, window 1024: 896
//   tiles 192 -> 175 us; 1024 tiles, 4 full rounds, 196 -> 194; 256 tiles, one round, 49 -> 55). Windows of 2000 and more: 5 % slower.
// most_new: the most new rows of a slot, 1 at least.
// Tiles of 256 columns x heads are below 2^23 a slot (checked before), so that no product here passes 64 bits.
inline void q8_plan(Q8Plan& p, int B, int H, int G, int most_new, const int32_t* lens, const int32_t* n_new, int span = 0) {
  const int64_t rows = (int64_t)most_new * G;
  const auto tiles = [&](int b, int cols) { return ((int64_t)n_new[b] * G + cols - 1) / cols; };
  int longest = 0, active = 0, fewest = most_new;
  int64_t units16 = 0, units64 = 0, units256 = 0, work16 = 0;  // tiles of all heads, and tiles x tokens
  double tokens64 = 0;
  for (int b = 0; b < B; ++b) {
    if (n_new[b] == 0) continue;
    ++active;
    longest = std::max(longest, lens[b]);
    const int64_t n = rows <= kQ8Cols ? H : tiles(b, kQ8Cols) * H;
    units16 += n;
    if (units16 <= kQ8Groups) work16 += n * lens[b];
    fewest = std::min(fewest, n_new[b]);
    if (rows > (span ? kQ8Cols : kFewRows)) {
      units64 += tiles(b, kQ8WideCols) * H;
      tokens64 += (double)(tiles(b, kQ8WideCols) * H) * lens[b];
      units256 += tiles(b, kQ8PromptCols) * H;
    }
  }
  const int64_t launched = (rows + kQ8Cols - 1) / kQ8Cols * H * B;
  bool few = rows <= (span ? kQ8Cols : kFewRows) || (units16 <= kQ8Groups && work16 <= 1 << 18 && launched <= 16 * kQ8Groups);
  const bool wide = span != 0 && !few && (units64 <= kQ8PromptGroups || q8_wide_is_faster(rows, units16, units64, units256, tokens64));
  few = few || (rows <= kFewRows && !wide);
  const bool half = rows > 128 && (span != 1        ? longest <= 2048 && units256 <= 256
                                   : units256 <= 128 ? longest <= 2048
                                                     : longest <= 1536 && units256 > 256);
  p.cols = few ? kQ8Cols : wide ? kQ8WideCols : half ? kQ8PromptCols / 2 : kQ8PromptCols;
  p.ntile = (int)((rows + p.cols - 1) / p.cols);
  p.rows = (int)std::min<int64_t>(rows, p.cols);
  const int64_t groups = few ? kQ8Groups : kQ8PromptGroups;
  const int64_t round = few || wide ? 256 : longest < 1024 ? 512 : 256;  // tokens of a round
  int64_t units = few ? units16 : wide ? units64 : units256;
  if (half && !wide) {
    units = 0;
    for (int b = 0; b < B; ++b) units += tiles(b, p.cols) * H;
  }
  const bool over = units > groups;
  const auto count = [&](int64_t rounds, bool all) {  // work-groups of splits of so many rounds, or those that have a record
    int64_t n = 0;
    for (int b = 0; b < B; ++b) {
      const int64_t s = n_new[b] > 0 ? std::max<int64_t>(1, (lens[b] + rounds * round - 1) / (rounds * round)) : 0;
      if (all || s > 1) n += s * tiles(b, p.cols) * H;
    }
    return n;
  };
  const auto fits = [&](int64_t rounds) { return count(rounds, !over) <= groups; };
  int64_t lo = 1, hi = std::max<int64_t>((longest + round - 1) / round, 1);  // hi rounds: one split each
  if (over) {
    const int64_t mean = (count(1, true) + groups - 1) / groups;
    lo = hi > 2 * mean ? mean : hi;
  }
  while (lo < hi) {  // the fewest rounds that fit
    const int64_t mid = (lo + hi) / 2;
    if (fits(mid)) hi = mid;
    else lo = mid + 1;
  }
  int64_t alone = span == 1 ? 7 : span == 2 ? 3 : 4;
  if (span && few && units16 <= kQ8Groups && longest * units16 * 4 <= work16 * (span == 1 ? 6 : 5))
    alone = units16 >= 160 ? (longest + round - 1) / round : span == 1 ? std::max(alone, alone * units16 / 64) : alone;
  if (few && longest <= alone * round) hi = alone;
  const bool idle = units * 64 < 256 && longest > 64 * 4 * round;
  const int64_t cap = idle ? kQ8MaxSplits : 64;
  Q8Splits& s = p.splits;
  Q8Order& o = s.order;
  o.most = 1;
  o.slots = B;
  o.active_slots = active;
  o.split_slots = 0;
  uint32_t records = 0;
  const bool one = hi * round >= longest;  // split each
  const auto splits = [&](int b) {
    return n_new[b] == 0 ? 0 : one ? 1 : (int)std::max<int64_t>(1, std::min((lens[b] + hi * round - 1) / (hi * round), cap));
  };
  for (int b = 0; b < B && !one; ++b) {
    const int n = splits(b);
    if (n < 2) continue;
    o.most = std::max(o.most, n);
    s.part[o.split_slots++] = (uint32_t)n << 16 | records;
    records += n * (uint32_t)tiles(b, p.cols);
  }
  s.part[o.split_slots] = records;
  o.flags = active < B || (o.split_slots > 0 && o.split_slots < B) ? kQ8Reordered : 0;
  if (active < B || ((int64_t)fewest * G + p.cols - 1) / p.cols < p.ntile) o.flags |= kQ8Uneven;
  if (!(o.flags & kQ8Reordered)) return;
  std::fill(s.slot, s.slot + (B + 1) / 2, 0u);
  int at[3] = {0, o.split_slots, active};
  for (int b = 0; b < B; ++b) {
    const int n = splits(b), place = at[n > 1 ? 0 : n == 1 ? 1 : 2]++;
    s.slot[place >> 1] |= (uint32_t)b << (16 * (place & 1));
  }
}

// The units (blocks or tiles of `size` tokens) that a tile of rows walks where they see the sinks, and the tokens from..end - 1:
// those of the sinks, then those from the one that holds `from` on
struct Q8Walk {
  int sinks, skip, count;  // units of the sinks, units left out behind them, units in all
  constexpr Q8Walk(int sink_tokens, int from, int end, int size) : sinks(0), skip(0), count((end + size - 1) / size) {
    const int s = (sink_tokens + size - 1) / size, gap = from / size;
    sinks = s < count ? s : count;
    skip = gap > sinks ? (gap < count ? gap : count) - sinks : 0;
    count -= skip;
  }
  constexpr int operator()(int i) const { return i < sinks ? i : i + skip; }
  constexpr int before(int end, int size) const {  // units of the walk with tokens before `end`
    const int n = (end + size - 1) / size;
    return n <= sinks ? n : n - skip > sinks ? n - skip : sinks;
  }
};

// Tokens that a tile of a slot's rows walks where they see the sinks and a window: what the plan counts in place of its length
inline int q8_span(int len, int n_new, int G, int window, int sinks) {
  const int64_t positions = std::min<int64_t>(n_new, kQ8PromptCols / G + 1);
  return (int)std::min<int64_t>(len, (int64_t)sinks + window + positions + 2 * 32);  // window and sinks may begin and end inside blocks
}

// Split records of every call of up to n_max rows. A call's splits fit into its groups, but for units (tiles of a sequence
// and head) that are more than the groups: those have one split and no record. Calls of few rows and of many count by themselves
inline size_t q8_workspace_bound(int G, int n_max) {
  const size_t few = (size_t)kQ8Groups * kQ8Cols, many = (size_t)kQ8PromptGroups * kQ8PromptCols;
  return ((int64_t)n_max * G > kFewRows ? std::max(few, many) : few) * kQ8Record * sizeof(float);
}
// the same where rows see a window or precede a tree: the wide kernel takes up calls of fewer rows
inline size_t q8_span_workspace_bound(int G, int n_max) {
  const size_t wide = (size_t)kQ8PromptGroups * kQ8WideCols * kQ8Record * sizeof(float);
  return (int64_t)n_max * G > kQ8Cols ? std::max(q8_workspace_bound(G, n_max), wide) : q8_workspace_bound(G, n_max);
}

// A tree's merge: groups of 32 lanes for a column, 8 splits each at most, and columns of a work-group
struct Q8TreeMerge {
  int groups, cols;
};
inline Q8TreeMerge q8_tree_merge(const Q8Plan& p) {
  const int most = p.splits.order.most;
  if (most > 64) return {16, 1};
  if (most > 32) return {8, 1};
  if (most > 16) return {4, 2};
  if (most > 8) return {2, 4};
  return {1, 8};
}
inline int64_t q8_tree_merge_groups(const Q8Plan& p, int H) {  // work-groups
  const int cols = q8_tree_merge(p).cols;
  return (int64_t)((p.rows + cols - 1) / cols) * H * p.ntile * p.splits.order.slots;
}

// A tree's records: those of the splits, then one for each tile of each slot and head that has one split
inline int64_t q8_split_records(const Q8Plan& p, int H) { return (int64_t)(p.splits.part[p.splits.order.split_slots] & 0xffffu) * H; }
inline size_t q8_tree_workspace(const Q8Plan& p, int H) {
  return (q8_split_records(p, H) + (int64_t)p.splits.order.slots * H * p.ntile) * p.cols * kQ8Record * sizeof(float);
}
// and of every call of up to n_max rows: the tiles have 16 columns, 64 at most from 17 rows and 256 at most from 33 rows on
inline size_t q8_tree_workspace_bound(int B, int H, int G, int n_max) {
  const int64_t rows = (int64_t)n_max * G, cols = rows > kFewRows ? kQ8PromptCols : rows > kQ8Cols ? kQ8WideCols : kQ8Cols;
  return q8_span_workspace_bound(G, n_max) + (size_t)B * H * ((rows + cols - 1) / cols * cols) * kQ8Record * sizeof(float);
}

}  // namespace okvq
