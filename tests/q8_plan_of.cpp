// Prints the kernel that the launch plan gives to attention calls with a window or a tree of drafts: reads lines of
// "span H G window sinks B, B lengths, B counts of new rows" and prints "columns of a tile, most splits, tiles" for each.
#include "q8_plan.hpp"

#include <climits>
#include <cstdio>
#include <vector>

int main() {
  int span, H, G, window, sinks, B;
  while (std::scanf("%d %d %d %d %d %d", &span, &H, &G, &window, &sinks, &B) == 6) {
    std::vector<int32_t> lens(B), n(B);
    for (auto* v : {&lens, &n})
      for (auto& x : *v)
        if (std::scanf("%d", &x) != 1) return 1;
    for (int b = 0; b < B; ++b) lens[b] = okvq::q8_span(lens[b], n[b], G, window > 0 ? window : INT_MAX, sinks);
    okvq::Q8Plan p;
    okvq::q8_plan(p, B, H, G, *std::max_element(n.begin(), n.end()), lens.data(), n.data(), span);
    std::printf("%d %d %d\n", p.cols, p.splits.order.most, p.ntile);
  }
}
