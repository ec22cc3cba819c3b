// Who works on what in the attention over pages: the tiles of a batch's
// entries, and each workgroup's share of their blocks of keys. Plain arithmetic
// on lengths, for the device (tree_dev.h) and, where a test goes through every
// workgroup's share, for the host.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace vla {
namespace pg {

// What an entry of a batch is: its sequence (-1: none), first row, rows,
// committed slots and the slots that its pages hold. Rows and slots are
// clamped so that whatever the arrays hold, rows lie in [0, n_rows) and slots
// in the table.
struct Entry {
  int seq, row0, n, len, cap;
};

// sum over i < n of floor((a i + b) / m), by Euclid's steps
__host__ __device__ __forceinline__ uint32_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  uint32_t sum = 0;
  while (n > 0) {
    if (a >= m) {
      sum += (uint32_t)((unsigned long long)(n - 1) * n / 2) * (a / m);
      a %= m;
    }
    if (b >= m) {
      sum += n * (b / m);
      b %= m;
    }
    const uint32_t y = a * n + b;
    if (y < m) break;
    n = y / m;
    b = y % m;
    const uint32_t t = m;
    m = a;
    a = t;
  }
  return sum;
}

// The tiles of an entry and one KV head: BM rows by units of `unit` keys. A
// causal tile ends with its last row's own slot, so tile rt has
// ceil((len + 1 + floor((BM (rt + 1) - 1) / group)) / unit) units, which is
// floor((BM rt + BM - 1 + group (len + unit)) / (group unit)).
//
// With a window (WIN, slide()) a tile begins with the unit of the first slot
// that its first row sees, floor((max(0, len - back + 1 + floor(BM rt / group)))
// / unit), which from the tile on whose window begins inside the slots is
// floor((BM rt + group (len - back + 1)) / (group unit)).
template <int BM, bool WIN = false>
struct Geo {
  int tiles, M, group, len, end, unit;
  bool flat;  // every tile reads all keys
  int back;    // slots of the window (0: none)
  bool fixed;  // rows' places are not their order: every tile begins with the entry's first
  __host__ __device__ __forceinline__ void set(int group_, bool causal, const Entry& x, int unit_) {
    group = group_;
    unit = unit_;
    M = x.n * group;
    tiles = (M + BM - 1) / BM;
    len = x.len;
    const long long e = (long long)x.len + x.n;
    end = e < x.cap ? (int)e : x.cap;
    flat = !causal || e > x.cap;  // (drafts without pages: no row sees them)
    if constexpr (WIN) back = 0, fixed = true;
  }
  // A window of `window` slots (0: none) for rows whose places are their order
  // or, with still set, lie somewhere behind the committed slots.
  __host__ __device__ __forceinline__ void slide(int window, bool still) {
    const long long e = (long long)len + M / group;
    back = e > end || window >= e ? 0 : window;
    fixed = still;
  }
  __host__ __device__ __forceinline__ int skip(int rt) const {  // units before the tile's first
    if (!WIN || back == 0) return 0;
    const int at = len - back + 1 + (fixed ? 0 : (int)((unsigned)(BM * rt) / (unsigned)group));
    return at > 0 ? at / unit : 0;
  }
  // those of the tiles before rt
  __host__ __device__ __forceinline__ int skipped(int rt) const {
    if (!WIN || back == 0) return 0;
    if (fixed) return rt * skip(0);
    const int c = len - back + 1, i0 = c >= 0 ? 0 : (int)((unsigned)(-c * group + BM - 1) / (unsigned)BM);
    return rt <= i0 ? 0 : (int)floor_sum(rt - i0, group * unit, BM, group * c + BM * i0);
  }
  // (a tile without keys has one unit, which writes its zeros)
  __host__ __device__ __forceinline__ int all() const { return end > 0 ? (end + unit - 1) / unit : 1; }
  __host__ __device__ __forceinline__ int tile_end(int rt) const {
    if (flat) return end;
    const int last = (rt + 1) * BM < M ? (rt + 1) * BM - 1 : M - 1;
    return len + last / group + 1;
  }
  __host__ __device__ __forceinline__ int units(int rt) const {
    return (flat ? all() : (tile_end(rt) + unit - 1) / unit) - skip(rt);
  }
  // units of the tiles before rt (rt < tiles)
  __host__ __device__ __forceinline__ int before(int rt) const {
    if (flat) return rt * all() - skipped(rt);
    return (int)floor_sum(rt, group * unit, BM, BM - 1 + group * (len + unit)) - skipped(rt);
  }
  __host__ __device__ __forceinline__ int sum() const { return tiles == 0 ? 0 : before(tiles - 1) + units(tiles - 1); }
  // the tile that holds unit u of the head's: units grow by a line, their sum
  // by a parabola, whose root is close
  __host__ __device__ __forceinline__ int find(int u) const {
    if (WIN && back) {  // (neither a line nor a parabola: halves)
      int lo = 0, hi = tiles - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before(mid) <= u) lo = mid;
        else hi = mid - 1;
      }
      return lo;
    }
    if (flat) return u / all();
    if (tiles <= 1) return 0;
    const float first = (float)units(0), grow = (float)(units(tiles - 1) - units(0)) / (float)(tiles - 1);
    const float h = first - 0.5f * grow;
    int rt = grow > 0.f ? (int)((sqrtf(h * h + 2.f * grow * (float)u) - h) / grow) : (int)((float)u / first);
    rt = rt < 0 ? 0 : rt > tiles - 1 ? tiles - 1 : rt;
    while (rt > 0 && before(rt) > u) --rt;
    while (rt + 1 < tiles && before(rt + 1) <= u) ++rt;
    return rt;
  }
};

// (64-bit divisions are long: most counts are short)
__host__ __device__ __forceinline__ long long ceil_div(long long a, int b) {
  return a >> 31 ? (a + b - 1) / b : (long long)(((uint32_t)a + (uint32_t)b - 1) / (uint32_t)b);
}

// What a wave knows of its workgroup's run and of the tile it works on: the
// same in every lane.
struct Tile {
  int seq, row0, len, head, rt;
  int b0, b1;         // blocks of the tile to work on
  int M, group, kend;
  int n, cap;         // (of its entry)
  int parts;          // with the first of several parts: how many, else 0
  bool whole, causal;
  bool first;         // the tile's first part
};
struct Run {
  long long u, u_end;  // this run's next and last unit
  long long quota;     // units of a run
  int w;               // this run (behind the last: none)
  int per;             // blocks of a unit
  int back;            // (as in Batch)
  bool fixed;
};

// The run's part of tile rt, from unit u0 of its nu on.
template <int BM, int BN, bool WIN>
__host__ __device__ __forceinline__ Tile cut(Run& r, const Geo<BM, WIN>& g, const Entry& x, int head, int rt, int u0,
                                             int nu, bool causal) {
  const int u1 = (int)(nu - u0 < r.u_end - r.u ? nu : u0 + (r.u_end - r.u));
  Tile t{};
  t.head = head;
  t.rt = rt;
  t.seq = x.seq;
  t.row0 = x.row0;
  t.n = x.n;
  t.cap = x.cap;
  t.len = x.len;
  t.M = g.M;
  t.group = g.group;
  t.causal = causal;
  t.kend = g.tile_end(rt);
  const int s = g.skip(rt);
  t.b0 = (s + u0) * r.per;
  const int nb = t.kend > 0 ? (t.kend + BN - 1) / BN : 1;
  t.b1 = (s + u1) * r.per < nb ? (s + u1) * r.per : nb;
  t.whole = u0 == 0 && u1 == nu;
  t.first = u0 == 0;
  t.parts = t.whole || u0 > 0 ? 0 : (int)(r.quota == 1 ? r.u + nu - 1 : (r.u + nu - 1) / r.quota) - r.w + 1;
  r.u += u1 - u0;
  return t;
}

// What deal() has to know of the batch.
struct Batch {
  int n_ent, nkv, group, wgs;
  bool causal;
  int back = 0;        // slots of a window (0: none), for Geo::slide()
  bool fixed = false;
};

// All entries' units stand in a row and are dealt out in equal runs, so that
// uneven sequences load the chip evenly. A unit is a block of keys of a tile,
// and a run may begin and end inside tiles: at most two of its tiles are
// shared with other runs. Where there are few tiles (at most half as many as
// workgroups), a unit is as many blocks of one tile as give every workgroup at
// most one unit: a run that crossed into another tile would start twice for
// a few blocks each. deal() finds the tile at r.u; with `first` set it works
// out the run of workgroup `wg` before. Every wave does so for itself; its
// lanes hold 64 entries at a time: load(c0) fetches those from c0 on,
// count(causal, unit) works out their tiles and units (and returns the sum),
// tiles() sums their tiles, at(u) is the lane whose units hold the chunk's unit
// u, and entry(), units() and before() are what that lane has.
template <int BM, int BN, int LONG, bool WIN = false, typename Lanes>
__host__ __device__ __forceinline__ Tile deal(Run& r, bool first, const Batch& a, int wg, Lanes& lanes) {
  const int n_ent = a.n_ent, nkv = a.nkv;
  if constexpr (WIN) r.back = a.back, r.fixed = a.fixed;
  long long base = 0, total = 0;
  // One loop over the entries, in passes: 0 counts blocks and tiles, 1 counts
  // units of several blocks, 2 finds the unit. (One copy of the code: what a
  // short call waits for most is instructions.)
  int pass = first ? 0 : 2, per = first ? 1 : r.per;
  long long tiles = 0;
  for (int c0 = 0;;) {
    // (what the pass before left in the lanes is its last 64 entries: with more
    // of them than that, every pass fetches its own)
    if (pass != 1 || n_ent > 64) lanes.load(c0);
    const long long all = lanes.count(a.causal, BN * per);
    if (pass == 2) {
      if (r.u < base + all) break;
      base += all;
      c0 += 64;
      if (c0 >= n_ent) return Tile{};  // (no entry holds it: the lengths changed under the call)
      continue;
    }
    total += all;
    if (pass == 0) tiles += lanes.tiles() * nkv;
    c0 += 64;
    if (c0 < n_ent) continue;
    c0 = 0;
    if (pass == 0 && 2 * tiles <= a.wgs) {
      per = (int)ceil_div(total, a.wgs - (int)tiles);
      // LONG times that where two workgroups of a CU share its matrix cores and
      // an average tile still makes four parts: two sequences of 2,000 slots,
      // trees of 60, 32 heads on 8 of 128, 23.8 us and 27.0; eight of 4,000,
      // trees of 40, 8 on 1, 27.0 and 28.9, of 64 23.0 and 22.6. With fewer parts
      // whole CUs would wait: ten uneven sequences of 500 to 8,000, 32 on 8 of
      // 128, 126 us so and 81.
      if (LONG > 1 && (float)per * (float)(4 * LONG) * (float)tiles <= (float)total) per *= LONG;
      // A part of b blocks of the tile's B costs b steps here and the join B / b
      // parts, so b stays at a multiple of sqrt(B) or above. One sequence, 8
      // heads on 1 of 128, with that and without: a token behind 60,000 slots
      // 24.9 us and 44.8; trees of 24 behind 8,000 28.8 us and 73.8, behind
      // 60,000 50.5 us and 78.1.
      constexpr float C = BM == 32 ? 16.f : 4.f;
      if ((float)per * (float)per * (C * (float)tiles) < (float)total)
        per = (int)ceilf(Lanes::root((float)total / (C * (float)tiles)));
      pass = 1;
      if (per > 1) {
        total = 0;
        continue;
      }
      per = 1;
    }
    r.per = per;
    r.quota = pass == 1 || total <= a.wgs ? 1 : ceil_div(total, a.wgs);
    // Workgroups go round the eight XCDs: each XCD takes an eighth of the runs,
    // consecutive ones, so that its L2 serves K and V of neighbouring tiles
    // once (and the join what was written there), and few runs still use every
    // XCD's share of the memory.
    const int runs = r.quota == 1 ? (int)total : (int)ceil_div(total, (int)r.quota), share = (runs + 7) >> 3;
    const int i = wg >> 3;
    r.w = i < share ? (wg & 7) * share + i : a.wgs;
    r.u = r.w * r.quota;
    r.u_end = r.u + r.quota < total ? r.u + r.quota : total;
    if (r.u >= r.u_end) return Tile{};
    if (n_ent <= 64) break;
    pass = 2;
  }
  const int el = lanes.at(r.u - base);
  const Entry x = lanes.entry(el);
  const int persum = lanes.units(el);
  const long long at = r.u - (base + lanes.before(el));
  Geo<BM, WIN> g;
  g.set(a.group, a.causal, x, BN * per);
  if constexpr (WIN) g.slide(a.back, a.fixed);
  // (a head's units fit 31 bits; most entries' do as well. Divisions are long,
  // and a short call waits for each: one head and one tile need none.)
  const int head = nkv == 1 ? 0 : at >> 31 ? (int)(at / persum) : (int)((uint32_t)at / (uint32_t)persum);
  const int rem = (int)(at - (long long)head * persum);
  int rt = 0, u0 = rem, nu = persum;
  if (g.tiles > 1) {
    rt = g.find(rem);
    u0 = rem - g.before(rt);
    nu = g.units(rt);
  }
  return cut<BM, BN, WIN>(r, g, x, head, rt, u0, nu, a.causal);
}
// The tile behind t in the run, which holds it from its first unit on: the
// next of its head, or of the next head; behind the entry's last head it is for
// deal() to find (more: false).
template <int BM, int BN, bool WIN = false>
__host__ __device__ __forceinline__ bool more(Run& r, Tile& t, int nkv) {
  const Entry x = {t.seq, t.row0, t.n, t.len, t.cap};
  Geo<BM, WIN> g;
  g.set(t.group, t.causal, x, BN * r.per);
  if constexpr (WIN) g.slide(r.back, r.fixed);
  const bool same = t.rt + 1 < g.tiles;
  const int head = same ? t.head : t.head + 1, rt = same ? t.rt + 1 : 0;
  if (head >= nkv) return false;
  t = cut<BM, BN, WIN>(r, g, x, head, rt, 0, g.units(rt), t.causal);
  return true;
}

}  // namespace pg
}  // namespace vla
