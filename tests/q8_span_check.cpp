// Host check of what a window and a tree add to the 8-bit attention's launch plan, with the mappings that its kernels use: a
// walk meets every unit that a row sees once and in order and no unit that none does; a tree's records lie apart and inside
// its workspace, which the stated bound covers. Prints "ok" or the first call that breaks a rule.
#include "q8_plan.hpp"

#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <set>
#include <vector>

using namespace okvq;

static std::mt19937 rng(11);
static int below(int n) { return (int)(rng() % (unsigned)n); }
static int spread(int most) { return (int)std::exp2(std::log2(most + 1.0) * (rng() / 4294967296.0)); }
static void fail(const char* what, long a, long b, long c, long d) {
  std::printf("%s: %ld %ld %ld %ld\n", what, a, b, c, d);
  std::exit(1);
}

int main() {
  for (int call = 0; call < 200000; ++call) {
    const int end = below(6) ? spread(3000) : 0, size = below(2) ? 32 : 64;
    const int sinks = below(3) ? below(200) : below(2) ? 0 : 1 << 27, from = below(5) ? below(end + 40) : 0;
    const Q8Walk w(sinks, from, end, size);
    if (w.count < 0 || w.sinks < 0 || w.skip < 0) fail("negative", sinks, from, end, size);
    int at = 0;
    for (int u = 0; u * size < end; ++u) {
      const int a = u * size, b = std::min(a + size, end);
      const bool seen = a < sinks || (from < b && from < end);
      if (seen && (at >= w.count || w(at) != u)) fail("unit", sinks, from, end, size);
      at += seen;
    }
    // from behind the end: the unit that holds it may be walked, and is masked
    if (at != w.count && !(from >= end && w.count <= at + 1)) fail("count", sinks, from, end, size);
    const int part = below(end + 1);
    int n = 0;
    while (n < w.count && w(n) * size < part) ++n;
    if (w.before(part, size) != n) fail("before", sinks, from, part, size);
    for (int i = 0; i < w.count; ++i)
      if (w(i) < 0 || w(i) * size >= end) fail("outside", sinks, from, end, size);
  }
  for (int call = 0; call < 4000; ++call) {
    const int B = call % 3 == 0 ? 1 : 1 + spread(call % 3 == 1 ? 40 : 1023), H = 1 + spread(15), G = 1 + below(16), n_max = 1 + spread(255);
    const int window = below(2) ? INT_MAX : 1 + spread(5000), sinks = below(2) ? 0 : spread(1 << 27);
    std::vector<int32_t> lens(B), n_new(B), spans(B);
    int most = 0;
    for (int b = 0; b < B; ++b) {
      lens[b] = below(8) ? spread(call % 5 ? 70000 : 1500) : 0;
      n_new[b] = below(4) ? 1 + below(n_max) : 0;
      most = std::max(most, n_new[b]);
      spans[b] = q8_span(lens[b], n_new[b], G, window, sinks);
      if (spans[b] < 0 || spans[b] > lens[b]) fail("span", lens[b], spans[b], window, sinks);
      if (window == INT_MAX && spans[b] != lens[b]) fail("whole span", lens[b], spans[b], window, sinks);
    }
    if (most == 0) continue;
    const int span = 1 + below(2);
    Q8Plan p;
    std::memset(&p, 0xff, sizeof(p));  // nothing may be read that the plan does not set
    q8_plan(p, B, H, G, most, spans.data(), n_new.data(), span);
    if (p.splits.order.split_slots + 1 > (int)(sizeof(p.splits.part) / 4)) fail("too many split slots", B, H, G, most);
    const int64_t single = q8_split_records(p, H), all = (int64_t)q8_tree_workspace(p, H) / sizeof(float) / ((int64_t)p.cols * kQ8Record);
    if (q8_span_workspace_bound(G, most) > q8_span_workspace_bound(G, n_max)) fail("window's bound", B, H, G, most);
    if (q8_tree_workspace(p, H) > q8_tree_workspace_bound(B, H, G, n_max)) fail("bound", B, H, G, most);
    if (single * p.cols > (int64_t)q8_span_workspace_bound(G, most) / 4 / kQ8Record) fail("split records", B, H, G, most);
    // every slot, head, tile and split is met by one work-group
    std::set<int64_t> met, done;
    const auto meet = [&](int place, int x, int h, int tile) {
      const Q8Part w = q8_part(p.splits.order, p.splits.part[q8_part_index(place)], p.splits.part[q8_part_index(place) + 1], place, x, tile);
      if (w.none) return;
      const int b = p.splits.order.flags & kQ8Reordered ? q8_slot_at(p.splits, place) : place;
      if (b >= B || w.split >= w.nsplit || w.nsplit > p.splits.order.most || h >= H || tile >= p.ntile) fail("range", B, H, G, most);
      if (!done.insert((((int64_t)b * H + h) * p.ntile + tile) * p.splits.order.most + w.split).second) fail("twice", B, H, G, most);
      int64_t at = w.first * H + h * w.records + tile * w.nsplit + w.split;
      if (w.records == 0) at = single + ((int64_t)b * H + h) * p.ntile + tile;
      if (at < 0 || at >= all || (w.records && at >= single) || !met.insert(at).second) fail("record", B, H, G, most);
    };
    const int width = q8_layers(p) * H * p.ntile;
    for (int x = 0; x < p.splits.order.most; ++x)
      if (p.cols == kQ8WideCols) {
        const Q8Units units = q8_units(p, H);
        for (int64_t id = 0; x == 0 && id < 8 * (int64_t)units.per + units.singles; ++id) {
          const Q8Unit u = q8_unit(p.splits, units, H, p.ntile, id);
          if (u.place < 0) continue;
          const Q8Part w = q8_part(p.splits.order, p.splits.part[q8_part_index(u.place)], p.splits.part[q8_part_index(u.place) + 1], u.place, u.split, u.tile);
          if (w.none || w.nsplit != u.nsplit || w.split != u.split || w.records != u.records || w.first != u.first) fail("unit", B, H, G, most);
          meet(u.place, u.split, u.h, u.tile);
        }
      } else if (p.cols == kQ8Cols) {
        for (int layer = 0; layer < q8_layers(p); ++layer)
          for (int y = 0; y < H * p.ntile; ++y) meet(q8_place(p.splits.order, layer, x), x, y / p.ntile, y % p.ntile);
      } else {
        for (int w = 0; w < width; ++w) {
          const Q8Tile t = q8_tile(p.splits.order, H, p.ntile, width, w, x);
          if (t.place >= 0) meet(t.place, x, t.h, t.tile);
        }
      }
    // and what the merge reads is what they wrote
    for (int place = 0; place < B; ++place)
      for (int tile = 0; tile < p.ntile; ++tile) {
        const Q8Part w = q8_part(p.splits.order, p.splits.part[q8_part_index(place)], p.splits.part[q8_part_index(place) + 1], place, 0, tile);
        const int b = p.splits.order.flags & kQ8Reordered ? q8_slot_at(p.splits, place) : place;
        if (w.nsplit > kQ8MaxSplits) fail("splits", B, H, G, most);
        for (int h = 0; h < H; ++h)
          for (int split = 0; split < w.nsplit; ++split) {
            int64_t at = w.first * H + h * w.records + tile * w.nsplit + split;
            if (w.records == 0) at = single + ((int64_t)b * H + h) * p.ntile + tile;
            if (!met.erase(at)) fail("merge", B, H, G, most);
          }
      }
    if (!met.empty()) fail("left over", B, H, G, most);
  }
  // the shapes that tests on the GPU mean for the wide kernel
  const auto cols = [&](std::vector<int32_t> lens, std::vector<int32_t> n, int H, int G, int window, int sinks, int span) {
    std::vector<int32_t> spans;
    for (size_t b = 0; b < lens.size(); ++b) spans.push_back(q8_span(lens[b], n[b], G, window, sinks));
    Q8Plan p;
    q8_plan(p, (int)lens.size(), H, G, *std::max_element(n.begin(), n.end()), spans.data(), n.data(), span);
    return p.cols;
  };
  std::vector<int32_t> lens, n, l16;
  for (int b = 0; b < 40; ++b) {
    const int32_t some[] = {0, 1, 31, 32, 33, 64, 65, 100, 500, 1003};
    lens.push_back(some[b * 7 % 10]);
    n.push_back(b % 5 == 0 ? b % 16 : 16);
  }
  for (int b = 0; b < 16; ++b) l16.push_back(4096 - 37 * b);
  if (cols({20011}, {16}, 1, 16, INT_MAX, 0, 2) != kQ8WideCols || cols({30000}, {16}, 1, 16, 17000, 33, 2) != kQ8WideCols ||
      cols({30000}, {16}, 1, 16, 16900, 0, 2) != kQ8WideCols || cols({20000}, {20}, 1, 16, 15000, 70, 1) != kQ8WideCols ||
      cols(lens, n, 2, 8, INT_MAX, 0, 2) != kQ8WideCols || cols(lens, n, 2, 8, 50, 3, 2) != kQ8WideCols || cols(lens, n, 2, 8, 90, 40, 1) != kQ8WideCols ||
      cols(std::vector<int32_t>(40, 300), std::vector<int32_t>(40, 16), 2, 8, INT_MAX, 0, 2) != kQ8WideCols ||
      cols(l16, std::vector<int32_t>(16, 3), 4, 7, INT_MAX, 0, 2) != kQ8WideCols || cols({20000}, {128}, 1, 2, INT_MAX, 0, 2) != kQ8WideCols)
    fail("not wide", 0, 0, 0, 0);
  // and for the prompt kernel's tiles of 128 and 256 columns
  if (cols({900}, {600}, 4, 7, 130, 40, 1) != 128 || cols({1200}, {1200}, 4, 7, 333, 5, 1) != 256 || cols({2500}, {2500}, 4, 7, 100, 65, 1) != 128 ||
      cols({3000}, {1200}, 4, 7, 1, 0, 1) != 256 || cols({700}, {600}, 4, 7, 1 << 30, 0, 1) != 128)
    fail("prompt", 0, 0, 0, 0);
  std::vector<int32_t> l64, n64;
  for (int b = 0; b < 16; ++b) l64.push_back(1500 - 90 * b), n64.push_back(b == 5 ? 0 : 64 - b);
  if (cols(l64, n64, 4, 7, INT_MAX, 0, 2) < 128 || cols(l64, n64, 4, 7, 300, 33, 2) < 128) fail("prompt of a tree", cols(l64, n64, 4, 7, INT_MAX, 0, 2), 0, 0, 0);
  std::printf("ok\n");
}
