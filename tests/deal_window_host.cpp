// As deal_host.cpp, with a window: each block of a tile from the one that holds
// the first slot its first row sees (rounded down to a unit) to its last has to
// be dealt exactly once. Prints the cases that fail.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <map>
#include <random>
#include <tuple>
#include <vector>

#include "../paper_2609_22335_amd/csrc/deal.h"

using namespace vla::pg;

struct Case {
  std::vector<Entry> ent;
  int nkv, group, wgs, window;
  bool causal, fixed;
};

template <int BM>
struct Lanes {
  const Case& c;
  Entry x[64];
  Geo<BM, true> g[64];
  int persum[64];
  long long all[64], incl[64];

  explicit Lanes(const Case& k) : c(k) {}
  static float root(float v) { return sqrtf(v); }
  void load(int c0) {
    for (int l = 0; l < 64; ++l) x[l] = c0 + l < (int)c.ent.size() ? c.ent[c0 + l] : Entry{-1, 0, 0, 0, 0};
  }
  long long count(bool causal, int unit) {
    long long sum = 0;
    for (int l = 0; l < 64; ++l) {
      g[l].set(c.group, causal, x[l], unit);
      g[l].slide(c.window, c.fixed);
      persum[l] = g[l].sum();
      all[l] = (long long)persum[l] * c.nkv;
      incl[l] = sum += all[l];
    }
    return sum;
  }
  long long tiles() const {
    long long t = 0;
    for (auto& k : g) t += k.tiles;
    return t;
  }
  int at(long long u) const {
    for (int l = 0; l < 64; ++l)
      if (incl[l] > u) return l;
    throw 2;
  }
  Entry entry(int l) const { return x[l]; }
  int units(int l) const { return persum[l]; }
  long long before(int l) const { return incl[l] - all[l]; }
};

struct Piece {
  int b0, b1, run, parts;
  bool whole, first;
};

template <int BM, int BN, int LONG>
static const char* check(const Case& c) {
  std::map<std::tuple<int, int, int>, std::vector<Piece>> got;  // first row, head, tile
  std::vector<int> slots(2 * c.wgs, 0);
  Batch b{(int)c.ent.size(), c.nkv, c.group, c.wgs, c.causal};
  b.back = c.window;
  b.fixed = c.fixed;
  int per = 1;
  try {
    for (int wg = 0; wg < c.wgs; ++wg) {
      Run r;
      Lanes<BM> lanes(c);
      Tile t = deal<BM, BN, LONG, true>(r, true, b, wg, lanes);
      while (t.b1 > t.b0) {
        per = r.per;
        got[{t.row0, t.head, t.rt}].push_back({t.b0, t.b1, r.w, t.parts, t.whole, t.first});
        if (!t.whole && slots.at(2 * r.w + (t.first ? 1 : 0))++) return "two parts in one slot";
        if (r.u >= r.u_end) break;
        if (!more<BM, BN, true>(r, t, c.nkv)) t = deal<BM, BN, LONG, true>(r, false, b, wg, lanes);
      }
    }
  } catch (int) {
    return "no lane holds the unit";
  }
  size_t want = 0;
  for (const Entry& e : c.ent) {
    const int M = e.n * c.group;
    for (int h = 0; h < c.nkv; ++h)
      for (int rt = 0; rt * BM < M; ++rt, ++want) {
        const int last = std::min((rt + 1) * BM, M) - 1;
        const bool fit = e.len + e.n <= e.cap;
        const int end = std::min(e.cap, e.len + e.n);
        const int keys = c.causal && fit ? e.len + last / c.group + 1 : end;
        const int nb = std::max(1, (keys + BN - 1) / BN);
        // by the definition: the first slot that the tile's first row sees
        const long long low = (long long)e.len + (c.fixed ? 0 : rt * BM / c.group) - c.window + 1;
        const int b0 = fit && low > 0 ? (int)(low / BN) / per * per : 0;
        auto it = got.find({e.row0, h, rt});
        if (it == got.end()) return "a tile that nobody works on";
        auto& p = it->second;
        std::sort(p.begin(), p.end(), [](const Piece& x, const Piece& y) { return x.b0 < y.b0; });
        int at = b0;
        for (size_t i = 0; i < p.size(); ++i) {
          if (p[i].b0 != at) return "blocks left out or dealt twice";
          at = p[i].b1;
          if (p[i].first != (i == 0)) return "a later part that passes for the first, or the reverse";
          if (p[i].whole != (p.size() == 1)) return "a part that passes for a whole tile, or the reverse";
          if (p[i].parts != (i == 0 && p.size() > 1 ? (int)p.size() : 0)) return "a wrong number of parts";
          if (p[i].run != p[0].run + (int)i) return "parts that are not in consecutive runs";
        }
        if (at != nb) return "blocks left out behind the last part";
      }
  }
  return got.size() == want ? "" : "a tile that does not exist";
}

int main(int argc, char** argv) {
  std::mt19937 rng(atoi(argv[1]));
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (uint32_t)(hi - lo + 1)); };
  auto log_pick = [&](int hi) { return (int)exp(log(hi + 1.0) * (rng() / 4294967296.0)) - 1; };
  int bad = 0;
  for (int i = 0; i < atoi(argv[2]); ++i) {
    Case c;
    c.nkv = 1 << pick(0, 3), c.group = pick(1, 9);
    c.window = 1 + log_pick(pick(0, 1) ? 30000 : 200);
    const int n = pick(1, pick(0, 3) ? 12 : 150), longest = log_pick(20000), most = log_pick(pick(0, 1) ? 4 : 600);
    int row0 = 0;
    for (int e = 0; e < n; ++e) {
      const bool live = pick(0, 9) > 0;
      const int rows = live ? pick(0, most) : 0, slots = live ? log_pick(longest) : 0;
      c.ent.push_back({live ? e : -1, row0, rows, slots, live ? slots + (pick(0, 9) ? rows : pick(0, rows)) : 0});
      row0 += rows;
    }
    for (int k = 0; k < 4; ++k) {
      c.causal = k & 1, c.fixed = k >> 1;
      c.wgs = 512;
      const char* w[4] = {check<32, 128, 1>(c), check<128, 32, 2>(c), (c.wgs = 256, check<128, 64, 1>(c)),
                          (c.wgs = 8, check<32, 128, 1>(c))};
      for (const char* x : w)
        if (*x) printf("case %d window %d form %d: %s\n", i, c.window, k, x), ++bad;
    }
  }
  printf("%d wrong\n", bad);
  return bad != 0;
}
