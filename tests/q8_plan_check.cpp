// Host check of the 8-bit attention's launch plan, with the mapping that its kernels use: over random calls, every slot, tile and
// split is met by exactly one work-group, records lie apart and inside the workspace, no merge has more splits than
// its kernel holds, and slots without new rows take no splits from the others. Prints "ok" or the first call that breaks a rule.
#include "q8_plan.hpp"

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <set>
#include <utility>
#include <vector>

using namespace okvq;

static std::mt19937 rng(7);
static int below(int n) { return (int)(rng() % (unsigned)n); }
static int spread(int most) { return (int)std::exp2(std::log2(most + 1.0) * (rng() / 4294967296.0)); }

static void fail(const char* what, int B, int H, int G, const std::vector<int32_t>& lens, const std::vector<int32_t>& n_new) {
  std::printf("%s: B %d H %d G %d\n", what, B, H, G);
  for (int b = 0; b < B; ++b) std::printf(" %d/%d", lens[b], n_new[b]);
  std::printf("\n");
  std::exit(1);
}

int main() {
  for (int call = 0; call < 6000; ++call) {
    const int kind = call % 4, B = kind == 0 ? 1 : 1 + spread(kind == 3 ? 1023 : 40), H = 1 + spread(15), G = 1 + below(16);
    const int most_new = kind == 1 ? 1 : 1 + spread(700), idle = below(3);  // idle: none, some, most of the slots
    std::vector<int32_t> lens(B), n_new(B);
    for (int b = 0; b < B; ++b) {
      lens[b] = below(8) ? spread(call % 5 ? 70000 : 1500) : 0;
      n_new[b] = (idle == 1 && below(2)) || (idle == 2 && below(16)) ? 0 : 1 + below(most_new);
    }
    const int most = *std::max_element(n_new.begin(), n_new.end());
    if (most == 0) continue;
    Q8Plan p;
    std::memset(&p, 0xff, sizeof(p));  // nothing may be read that the plan does not set
    q8_plan(p, B, H, G, most, lens.data(), n_new.data());
    if (p.splits.order.split_slots + 1 > (int)(sizeof(p.splits.part) / 4)) fail("too many split slots", B, H, G, lens, n_new);
    const size_t bound = q8_workspace_bound(G, most) / sizeof(float) / ((size_t)p.cols * kQ8Record);
    std::vector<char> met((size_t)B * H * p.ntile * p.splits.order.most, 0);
    std::vector<int> nsplit((size_t)B * p.ntile, 0);
    std::set<int> records;
    const auto meet = [&](int place, int x, int h, int tile) {
      const Q8Part w = q8_part(p.splits.order, p.splits.part[q8_part_index(place)], p.splits.part[q8_part_index(place) + 1], place, x, tile);
      if (w.none) return;
      const int b = p.splits.order.flags & kQ8Reordered ? q8_slot_at(p.splits, place) : place;
      if (b >= B || w.split >= w.nsplit || w.nsplit > p.splits.order.most || h >= H || tile >= p.ntile) fail("range", B, H, G, lens, n_new);
      char& m = met[(((size_t)b * H + h) * p.ntile + tile) * p.splits.order.most + w.split];
      if (m) fail("twice", B, H, G, lens, n_new);
      m = 1;
      nsplit[(size_t)b * p.ntile + tile] = w.nsplit;
      if ((place >= p.splits.order.active_slots) != (n_new[b] == 0)) fail("idle", B, H, G, lens, n_new);
      const bool needed = (int64_t)tile * p.cols < (int64_t)n_new[b] * G;
      if (!needed && !(p.splits.order.flags & kQ8Uneven)) fail("even tiles", B, H, G, lens, n_new);
      if ((w.records > 0) != (w.nsplit > 1)) fail("records of one split", B, H, G, lens, n_new);
      if (w.records == 0) return;
      if (place >= p.splits.order.split_slots) fail("no merge", B, H, G, lens, n_new);
      const int at = w.first * H + h * w.records + tile * w.nsplit + w.split;
      if (at < 0 || (size_t)at >= bound || !records.insert(at).second) fail("record", B, H, G, lens, n_new);
    };
    const int width = q8_layers(p) * H * p.ntile;
    for (int x = 0; x < p.splits.order.most; ++x)
      if (p.cols == kQ8Cols) {
        for (int layer = 0; layer < q8_layers(p); ++layer)
          for (int y = 0; y < H * p.ntile; ++y) meet(q8_place(p.splits.order, layer, x), x, y / p.ntile, y % p.ntile);
      } else {
        for (int w = 0; w < width; ++w) {
          const Q8Tile t = q8_tile(p.splits.order, H, p.ntile, width, w, x);
          if (t.place >= 0) meet(t.place, x, t.h, t.tile);
        }
      }
    for (int b = 0; b < B; ++b)
      for (int tile = 0; tile < p.ntile; ++tile) {
        const int n = nsplit[(size_t)b * p.ntile + tile];
        if (n < 1 || n > kQ8MaxSplits) fail("tile missed", B, H, G, lens, n_new);
        for (int i = 0; i < H * n; ++i)
          if (!met[(((size_t)b * H + i / n) * p.ntile + tile) * p.splits.order.most + i % n]) fail("split missed", B, H, G, lens, n_new);
      }
    // the same call without the slots that have no rows: the same splits, where as many work-groups without work (a slot's, or a
    // tile's that it lacks) leave the kernel the same
    std::vector<int32_t> l2, n2;
    for (int b = 0; b < B; ++b)
      if (n_new[b]) l2.push_back(lens[b]), n2.push_back(n_new[b]);
    Q8Plan q;
    q8_plan(q, (int)l2.size(), H, G, most, l2.data(), n2.data());
    if (q.cols != p.cols && (q.cols != kQ8Cols || (int64_t)q.ntile * H * B <= 16 * kQ8Groups)) fail("idle slots change the kernel", B, H, G, lens, n_new);
    if (q.cols == p.cols && (q.splits.order.most != p.splits.order.most || q.splits.order.split_slots != p.splits.order.split_slots ||
        std::memcmp(q.splits.part, p.splits.part, 4 * (p.splits.order.split_slots + 1)) != 0))
      fail("idle slots change the plan", B, H, G, lens, n_new);
  }
  // a long sequence among more short ones than the GPU holds at once
  for (const int B : {200, 1000})
    for (const int rows : {1, 30}) {
      std::vector<int32_t> lens(B, 300), n_new(B, rows);
      lens[B / 3] = 131072;
      Q8Plan p;
      q8_plan(p, B, 4, 7, rows, lens.data(), n_new.data());
      if (p.splits.order.split_slots != 1 || p.splits.order.most < 10) fail("a long sequence is not split", B, 4, 7, lens, n_new);
    }
  std::printf("ok\n");
}
