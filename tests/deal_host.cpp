// Every workgroup's share of the attention over pages, worked out on the host
// from the source that the kernels run: each block of every tile has to be dealt
// exactly once, each part of a shared tile to a slot of its own, and every
// search has to end inside the batch. Prints the cases that fail.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <map>
#include <random>
#include <string>
#include <tuple>
#include <vector>

#include "../paper_2609_22335_amd/csrc/deal.h"

using namespace vla::pg;

static bool strayed;  // entries were asked for behind the last one

struct Case {
  std::string name;
  std::vector<Entry> ent;
  int nkv = 1, group = 1, wgs = 256;
  bool causal = true;
};

template <int BM>
struct Lanes {
  const Case& c;
  Entry x[64];
  Geo<BM> g[64];
  int persum[64];
  long long all[64], incl[64];

  explicit Lanes(const Case& k) : c(k) {
    for (auto& e : x) e = Entry{-1, -1000, 1 << 20, 1 << 20, 1 << 20};  // (not looked at before a load)
  }
  static float root(float v) { return sqrtf(v); }
  void load(int c0) {
    if (c0 > 0 && c0 >= (int)c.ent.size()) {
      strayed = true;
      throw 1;
    }
    for (int l = 0; l < 64; ++l) x[l] = c0 + l < (int)c.ent.size() ? c.ent[c0 + l] : Entry{-1, 0, 0, 0, 0};
  }
  long long count(bool causal, int unit) {
    long long sum = 0;
    for (int l = 0; l < 64; ++l) {
      g[l].set(c.group, causal, x[l], unit);
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
  bool whole;
};

// "" where the case is dealt right, else what is wrong.
template <int BM, int BN, int LONG>
static std::string check(const Case& c) {
  std::map<std::tuple<int, int, int>, std::vector<Piece>> got;  // first row, head, tile
  std::vector<int> slots(2 * c.wgs, 0);
  const Batch b{(int)c.ent.size(), c.nkv, c.group, c.wgs, c.causal};
  try {
    for (int wg = 0; wg < c.wgs; ++wg) {
      Run r;
      Lanes<BM> lanes(c);
      Tile t = deal<BM, BN, LONG>(r, true, b, wg, lanes);
      int shared = 0;
      while (t.b1 > t.b0) {
        got[{t.row0, t.head, t.rt}].push_back({t.b0, t.b1, r.w, t.parts, t.whole});
        if (!t.whole && slots.at(2 * r.w + (t.b0 == 0 ? 1 : 0))++) return "two parts in one slot";
        if (t.parts && shared++) return "a run begins two shared tiles";
        if (r.u >= r.u_end) break;
        if (!more<BM, BN>(r, t, c.nkv)) t = deal<BM, BN, LONG>(r, false, b, wg, lanes);
      }
    }
  } catch (int) {
    return strayed ? "a search behind the last entry" : "no lane holds the unit";
  }
  size_t want = 0;
  for (const Entry& e : c.ent) {
    const int M = e.n * c.group;
    for (int h = 0; h < c.nkv; ++h)
      for (int rt = 0; rt * BM < M; ++rt, ++want) {
        // by the definition, one row at a time: what the tile's last row sees
        const int last = std::min((rt + 1) * BM, M) - 1;
        const int end = std::min(e.cap, e.len + e.n);
        const int keys = c.causal && e.len + e.n <= e.cap ? e.len + last / c.group + 1 : end;
        const int nb = std::max(1, (keys + BN - 1) / BN);
        auto it = got.find({e.row0, h, rt});
        if (it == got.end()) return "a tile that nobody works on";
        auto& p = it->second;
        std::sort(p.begin(), p.end(), [](const Piece& x, const Piece& y) { return x.b0 < y.b0; });
        int at = 0;
        for (size_t i = 0; i < p.size(); ++i) {
          if (p[i].b0 != at) return "blocks left out or dealt twice";
          at = p[i].b1;
          if (p[i].whole != (p.size() == 1)) return "a part that passes for a whole tile, or the reverse";
          if (p[i].parts != (i == 0 && p.size() > 1 ? (int)p.size() : 0)) return "a wrong number of parts";
          if (p[i].run != p[0].run + (int)i) return "parts that are not in consecutive runs";
        }
        if (at != nb) return "blocks left out behind the last part";
      }
  }
  return got.size() == want ? "" : "a tile that does not exist";
}

static std::string check_all(Case c) {
  const struct {
    std::string (*f)(const Case&);
    const char* what;
    int wgs;
  } forms[] = {{check<32, 128, 1>, "32 rows, two workgroups a CU", 512},
               {check<32, 128, 1>, "32 rows", 256},
               {check<128, 32, 2>, "128 rows, two workgroups a CU", 512},
               {check<128, 32, 1>, "128 rows", 256},
               {check<128, 64, 1>, "128 rows, blocks of 64", 512},
               {check<32, 128, 1>, "32 rows, eight workgroups", 8}};
  for (auto& f : forms) {
    c.wgs = f.wgs;
    for (int causal = 0; causal < 2; ++causal) {
      c.causal = causal;
      const std::string bad = f.f(c);
      if (!bad.empty()) return std::string(f.what) + (causal ? ", causal: " : ", masked: ") + bad;
    }
  }
  return "";
}

static void add(Case& c, int n, int rows, int slots, bool live = true, int room = -1) {
  static int row0;
  if (c.ent.empty()) row0 = 0;
  for (int i = 0; i < n; ++i) {
    Entry e{live ? (int)c.ent.size() : -1, row0, live ? rows : 0, live ? slots : 0, 0};
    e.cap = !live ? 0 : room < 0 ? slots + rows : std::max(slots, room);
    c.ent.push_back(e);
    row0 += rows;
  }
}

int main(int argc, char** argv) {
  std::vector<Case> cases;
  auto fresh = [&](const char* name, int nkv, int group) -> Case& {
    cases.push_back(Case{name, {}, nkv, group});
    return cases.back();
  };
  {
    add(fresh("80 tokens behind 4,000 slots", 1, 8), 80, 1, 4000);
    Case& a = fresh("20 live entries of 128", 1, 8);
    add(a, 20, 1, 3000), add(a, 108, 1, 0, false);
    Case& b = fresh("live entries at the end of 128", 1, 8);
    add(b, 120, 1, 0, false), add(b, 8, 1, 4000);
    Case& c = fresh("64 short sequences, then 36 long ones", 1, 8);
    add(c, 64, 1, 200), add(c, 36, 1, 6000);
    Case& d = fresh("64 long sequences, then 36 short ones", 1, 8);
    add(d, 64, 1, 6000), add(d, 36, 1, 200);
    add(fresh("96 trees of 40 rows", 1, 4), 96, 40, 2000);
    add(fresh("100 trees on two heads", 2, 4), 100, 20, 9000);
    Case& e = fresh("300 entries, one of them long", 1, 1);
    add(e, 200, 1, 0), add(e, 1, 1, 100000), add(e, 99, 1, 3);
    add(fresh("no entry", 1, 1), 0, 0, 0);
    add(fresh("200 empty entries", 4, 2), 200, 0, 50);
    add(fresh("a chunk of 2,000 rows behind 6,000", 8, 4), 2, 2000, 6000);
    Case& f = fresh("a prompt beside single tokens and padding", 2, 4);
    add(f, 1, 2000, 0), add(f, 60, 1, 700), add(f, 67, 1, 0, false);
    add(fresh("a token behind 2^26 slots", 1, 8), 1, 1, (1 << 26) - 1);
    add(fresh("32,768 rows behind 2^22 slots", 1, 8), 1, 1 << 15, 1 << 22);
    add(fresh("drafts without pages", 2, 3), 70, 50, 900, true, 900);
  }
  std::mt19937 rng(atoi(argv[1]));
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (uint32_t)(hi - lo + 1)); };
  auto log_pick = [&](int hi) { return (int)exp(log(hi + 1.0) * (rng() / 4294967296.0)) - 1; };
  for (int i = 0; i < atoi(argv[2]); ++i) {
    Case& c = fresh("drawn", 1 << pick(0, 3), pick(1, 9));
    const int n = pick(0, 300), longest = log_pick(20000), most = log_pick(pick(0, 3) ? 4 : 400), kind = pick(0, 3);
    for (int e = 0; e < n; ++e) {
      const int rows = pick(0, most), slots = kind == 0 ? longest : log_pick(longest);
      const bool live = kind < 2 || (kind == 2 ? e < 30 : pick(0, 9) > 6);
      add(c, 1, rows, slots, live, pick(0, 7) ? -1 : slots + pick(0, rows));
    }
    c.name = "drawn " + std::to_string(i) + ": " + std::to_string(n) + " entries, " + std::to_string(c.nkv) + " heads";
  }
  int bad = 0;
  for (auto& c : cases) {
    strayed = false;
    const std::string what = check_all(c);
    if (!what.empty()) printf("%s: %s\n", c.name.c_str(), what.c_str()), ++bad;
  }
  printf("%zu cases, %d wrong\n", cases.size(), bad);
  return bad != 0;
}
