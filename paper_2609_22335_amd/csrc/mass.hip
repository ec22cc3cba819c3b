// The weight that slots of a paged KV cache receive from a step's rows: for
// every KV head and slot the sum over rows and heads of the group of
// exp(score - lse), scores as in the attention that made the log-sum-exps.
#include "tree_dev.h"

namespace vla {
namespace {

constexpr int KT = 128, QT = 32;  // slots of a tile (32 to a wave), queries of a step

struct MassArgs {
  Args a;  // (first: fresh() finds it)
  float* mass;  // the layer's, [n_seqs][nkv][slots]
  float* part;  // [2 target][KT]
  int target;   // units that a launch wants at least (0: tiles are not cut)
};

// A tile of KT slots of one entry and KV head.
struct Spot {
  Tile t;
  int kt;
};

// The batch's tiles in a row, 64 entries a time, one to a lane. With a window
// an entry's first tile is that of the first slot that a row may see.
struct Row64 {
  const Args& a;
  Entry x;
  int kt0, nkt;
  long long all, incl, base;
  int c0, most;  // (rows of the largest entry, once counted)

  __device__ __forceinline__ void load(int c) {
    c0 = c;
    const int i = c + (int)(threadIdx.x & 63);
    x = Entry{-1, 0, 0, 0, 0};
    if (i < a.r.n_ent) x = entry_of(a.c, a.r, i);
    const long long e = (long long)x.len + x.n;
    const int end = e < x.cap ? (int)e : x.cap;
    int first = a.window ? x.len - a.window + 1 : 0;
    kt0 = first > 0 && x.n > 0 ? first / KT : 0;
    nkt = x.n > 0 && end > 0 ? (end + KT - 1) / KT - kt0 : 0;
    all = (long long)nkt * a.c.nkv;
    incl = wave_scan(all);
  }
  // the sum of all tiles
  __device__ __forceinline__ long long count() {
    long long sum = 0;
    int top = 0;
    for (int c = 0; c < a.r.n_ent; c += 64) {
      load(c);
      sum += lane_of(incl, 63);
      top = max(top, x.n);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = max(top, __shfl_xor(top, d));
    most = uni(top);
    return sum;
  }
  // How many units a tile's queries are cut into where there are few tiles, so
  // that a launch has `target`; a unit keeps CUT steps, which its start (keys,
  // first queries: two round trips) is worth: fp32 trees of 17 to 61 rows behind
  // 30 to 700 slots 19 us, with units of at least eight steps 32 us.
  __device__ __forceinline__ int cuts(long long tiles, int target) const {
    constexpr int CUT = 2;
    if (tiles >= target) return 1;
    const int steps = (int)(((long long)most * a.group + QT - 1) / QT);
    return (int)min((target + tiles - 1) / tiles, (long long)((steps + CUT - 1) / CUT));
  }
  __device__ __forceinline__ void begin() {
    base = 0;
    if (a.r.n_ent > 64 || a.r.n_ent == 0) load(0);
  }
  // tile i (ascending from call to call)
  __device__ __forceinline__ bool at(long long i, Spot& s) {
    while (true) {
      const long long sum = lane_of(incl, 63);
      if (i < base + sum) break;
      if (c0 + 64 >= a.r.n_ent) return false;
      base += sum;
      load(c0 + 64);
    }
    const int l = __ffsll(__ballot(base + incl > i)) - 1;
    const int k = (int)(i - base - (lane_of(incl, l) - lane_of(all, l)));
    const int n = __builtin_amdgcn_readlane(nkt, l);
    Tile& t = s.t;
    t = Tile{};
    t.head = k / n;
    s.kt = k - t.head * n + __builtin_amdgcn_readlane(kt0, l);
    t.seq = __builtin_amdgcn_readlane(x.seq, l);
    t.row0 = __builtin_amdgcn_readlane(x.row0, l);
    t.n = __builtin_amdgcn_readlane(x.n, l);
    t.len = __builtin_amdgcn_readlane(x.len, l);
    t.cap = __builtin_amdgcn_readlane(x.cap, l);
    t.group = a.group;
    t.M = t.n * a.group;
    t.causal = !a.mask && !a.span;
    t.kend = (int)min((long long)t.len + t.n, (long long)t.cap);
    return true;
  }
};

// Steps (tiles of QT queries) of which a query may see a slot of tile kt.
__device__ __forceinline__ int2 steps_of(const Args& a, const Tile& t, int kt) {
  const int nq = (t.M + QT - 1) / QT, s0 = kt * KT;
  if (a.mask && s0 >= t.len) return make_int2(0, 0);  // (a tree's drafts begin at nothing)
  int q0 = 0, q1 = nq;
  if (t.causal && s0 > t.len) q0 = (int)((unsigned)((s0 - t.len) * t.group) / QT);
  if (a.window && !a.depth) {
    const long long last = (long long)s0 + KT - 1 + a.window - t.len;  // first row past the window of the last slot
    if (last * t.group < t.M) q1 = last > 0 ? (int)((last * t.group + QT - 1) / QT) : 0;
  }
  return make_int2(q0, q1 > q0 ? q1 : q0);
}

__device__ __forceinline__ void put_mass(const MassArgs& m, const Tile& t, int slot, float got) {
  if (slot >= t.kend) return;
  float* to = m.mass + ((size_t)t.seq * m.a.c.nkv + t.head) * ((size_t)m.a.c.max_pages << m.a.c.page_lg) + slot;
  *to = slot < t.len ? *to + got : m.a.mask ? 0.f : got;
}

// A lane's key: which slot, where it lies (page -1: nowhere), and its place.
struct Key {
  int slot, page, place;
};
__device__ __forceinline__ int page_id(const Args& a, const Tile& t, int slot) {
  return slot < t.kend ? a.c.table[(size_t)t.seq * a.c.max_pages + (slot >> a.c.page_lg)] : -1;
}
template <typename T, int NQ>
__device__ __forceinline__ void load_key(const Args& a, const Tile& t, int slot, int id, u32x4 (&kf)[NQ]) {
  const int h = (threadIdx.x >> 5) & 1, hb = a.c.hd * (int)sizeof(T);
  const bool have = (unsigned)id < (unsigned)a.c.n_pages;
  const char* kp = a.k + (((size_t)(have ? id : 0) * a.c.nkv + t.head) * a.c.page + (slot & (a.c.page - 1))) * (size_t)hb;
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int ch = 2 * i + h;
    kf[i] = ch * 16 < hb ? *(const u32x4*)(kp + ch * 16) : u32x4{0, 0, 0, 0};
  }
}
__device__ __forceinline__ Key key_of(const Args& a, const Tile& t, int slot, int id) {
  Key k{slot, (unsigned)id < (unsigned)a.c.n_pages ? id : -1, slot};
  if (a.depth && slot >= t.len && slot < t.kend) k.place = place_of(a, t, t.row0 + slot - t.len, slot - t.len);
  return k;
}

// What the weights of 32 queries need beside their products: the log-sum-exp
// (units of log2(e); plus infinity for one that gives nothing), slope, place,
// and the slots that it sees.
template <int N>
struct Asks {
  float lse[N], slope[N];
  int place[N], lo[N], own[N];
};
// Query m of the tile's rows (behind the last: one that gives nothing).
struct Ask {
  float lse, slope;
  Row r;
  __device__ __forceinline__ void load(const Args& a, const Tile& t, int m, int tok, int g) {
    if (m >= t.M) tok = t.n - 1, g = t.group - 1;
    const int hq = t.head * t.group + g;
    r = row_of<true>(t, tok);
    lse = a.lse[(size_t)(t.row0 + tok) * a.nq + hq];
    slope = a.slopes ? a.slopes[hq] * LOG2E : 0.f;
    if (m >= t.M) lse = INFINITY;
  }
  template <int N>
  __device__ __forceinline__ void put(Asks<N>& to, int i) const {
    to.lse[i] = lse - lse == 0.f ? lse * LOG2E : INFINITY;
    to.slope[i] = slope, to.place[i] = r.place, to.lo[i] = r.lo, to.own[i] = r.own;
  }
};

// The lane's sum over 32 queries of exp(score - lse), x their products with its
// key (element j: query 8 (j / 4) + j % 4 + 4 h). `partly`: some of the wave's
// 32 keys are not seen by some of the queries.
template <typename T, int N>
__device__ __forceinline__ float weigh(f32x16& x, const Args& a, const Tile& t, const Key& key, const Asks<N>& q, int q0,
                                       bool partly) {
  const int h4 = 4 * (int)((threadIdx.x >> 5) & 1);
  const bool plain = a.cap2 == 0.f && !a.slopes;
  f32x4 ls[4];
#pragma unroll
  for (int j4 = 0; j4 < 4; ++j4) ls[j4] = *(const f32x4*)(q.lse + q0 + 8 * j4 + h4);
  if (!plain) {
    if (a.cap2 > 0.f) {
      cap_scores<T>(x, a);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] *= a.c2;
    }
    if (a.slopes) {
#pragma unroll
      for (int j4 = 0; j4 < 4; ++j4) {
        const f32x4 sl = *(const f32x4*)(q.slope + q0 + 8 * j4 + h4);
        const int4 pl = *(const int4*)(q.place + q0 + 8 * j4 + h4);
        const int p4[4] = {pl.x, pl.y, pl.z, pl.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[4 * j4 + i] = __builtin_fmaf(-sl[i], __builtin_fabsf((float)(p4[i] - key.place)), x[4 * j4 + i]);
      }
    }
  }
  const float c = plain ? a.c2 : 1.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) x[j] = ex2(__builtin_fmaf(x[j], c, -ls[j / 4][j % 4]));
  if (partly) {
    const int far = a.window ? a.window : 0x7FFFFFFF;
    const bool have = key.page >= 0 && !(a.mask && key.slot >= t.len);  // (a tree's drafts begin at nothing)
#pragma unroll
    for (int j4 = 0; j4 < 4; ++j4) {
      const int4 own = *(const int4*)(q.own + q0 + 8 * j4 + h4), lo = *(const int4*)(q.lo + q0 + 8 * j4 + h4);
      const int4 pl = *(const int4*)(q.place + q0 + 8 * j4 + h4);
      const int o4[4] = {own.x, own.y, own.z, own.w}, l4[4] = {lo.x, lo.y, lo.z, lo.w}, p4[4] = {pl.x, pl.y, pl.z, pl.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool see = have && key.slot < o4[i] && key.slot >= l4[i] && p4[i] - key.place < far;
        x[4 * j4 + i] = see ? x[4 * j4 + i] : 0.f;
      }
    }
  }
  float add[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) add[i] = (x[i] + x[4 + i]) + (x[8 + i] + x[12 + i]);
  float sum = (add[0] + add[1]) + (add[2] + add[3]);
  // a key that is not finite makes NaN of rows that give nothing as well
  if (__any(sum != sum)) {
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) sum += ls[j / 4][j % 4] < INFINITY ? x[j] : 0.f;
  }
  return sum;
}

// Whether queries of tokens tok0 .. tok1 see any of slots kb .. kb + 31, and
// whether one of them may not see one of those.
__device__ __forceinline__ void look(const Args& a, const Tile& t, int kb, int tok0, int tok1, bool& live, bool& partly) {
  live = kb < t.kend;
  partly = kb + 32 > t.kend || a.span || (a.window && a.depth) || (a.mask && kb + 32 > t.len);
  if (t.causal) {
    live = live && t.len + tok1 >= kb;
    partly = partly || t.len + tok0 + 1 < kb + 32;
  }
  if (a.window && !a.depth) {
    live = live && (long long)t.len + tok0 - a.window < kb + 31;
    partly = partly || (long long)t.len + tok1 - a.window >= kb;
  }
}

template <typename T, int HDP>
constexpr int mass_waves() {
  return HDP * (int)sizeof(T) <= 256 ? 3 : 2;
}

// Few rows to a sequence: bound by the cache's bandwidth. Each wave streams its
// own 32 keys of a tile through its own two stages in the LDS, the next tile's
// on their way while these are worked on, without a barrier where a sequence's
// queries are one step (they stay in registers then). What slots have is read
// and written for eight tiles at once: a load that is waited for would wait for
// the keys on their way as well. 16 single tokens behind 8,000 to 65,000 slots,
// 32 heads on 8 of 128 (0.99 GB): 193 us, 5.1 TB/s; with keys loaded straight
// into registers, 32 bytes of a row at a time, 281 us.
template <typename T, int HDP>
__global__ __launch_bounds__(256, (many_waves<T, HDP>())) void k_mass_few(MassArgs m) {
  constexpr int RB = HDP * (int)sizeof(T), NQ = RB / 32, HOLD = 8;
  typedef Loader<T, HDP, 1, 16> Ld;
  const Args& a = m.a;
  // (by name: the compiler lets reads of one stage run beside loads into the other only where it can tell them apart)
  __shared__ __attribute__((aligned(1024))) unsigned char sA[4][32 * RB], sB[4][32 * RB], sQ[QT * RB];
  __shared__ __attribute__((aligned(16))) Asks<QT> sAsk;
  __shared__ float sGot[4][HOLD][32];
  const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
  const int hb = a.c.hd * (int)sizeof(T);
  Row64 row{a};
  const long long tiles = row.count();
  const long long quota = (tiles + gridDim.x - 1) / gridDim.x;
  long long u = (long long)blockIdx.x * quota;
  const long long end = min(tiles, u + quota);
  if (u >= end) return;
  row.begin();
  Spot s;
  while (u < end) {
    if (!row.at(u, s)) break;
    const Tile& t = s.t;
    const int last = (t.kend + KT - 1) / KT;  // the tiles that the run has of this entry and head: kt .. k1 - 1
    const int k1 = (int)min((long long)last, s.kt + (end - u));
    u += k1 - s.kt;
    Ld ld;
    ld.set(t);
    Place at[2], nat[2];
    auto block = [&](int kt) { return kt * KT + wv * 32; };
    ld.look(block(s.kt), at);
    ld.issue(a.k, (LB*)sA[wv], at, 0);
    auto fetch = [&](int q0) {  // a step's queries
      __syncthreads();
#pragma unroll
      for (int i = 0; i < QT * RB / 16 / 256; ++i) {
        const int c = tid + 256 * i, r = c / (RB / 16), ch = c % (RB / 16);
        const int mm = q0 + r < t.M ? q0 + r : t.M - 1, tok = mm / t.group;
        const char* qp = (const char*)a.q + ((size_t)(t.row0 + tok) * (size_t)a.ldq +
                                             (size_t)(t.head * t.group + (mm - tok * t.group)) * a.c.hd) * sizeof(T);
        *(u32x4*)(sQ + r * RB + ((ch ^ swz<RB, 16>(r)) * 16)) = ch * 16 < hb ? *(const u32x4*)(qp + ch * 16) : u32x4{0, 0, 0, 0};
      }
      if (tid < QT) {
        const int mm = q0 + tid < t.M ? q0 + tid : t.M - 1, tok = mm / t.group;
        Ask k;
        k.load(a, t, q0 + tid, tok, mm - tok * t.group);
        k.put(sAsk, tid);
      }
      __syncthreads();
    };
    auto chunk = [&](const LB* st, int i) {
      return *(const LDS_AS u32x4*)(st + l32 * RB + (((2 * i + h) ^ swz<RB, 16>(l32)) * 16));
    };
    u32x4 qf[NQ];
    // the sum over a step's queries (from q0 on) for the lane's key of the block
    auto step = [&](const LB* st, int kb, int q0, const Place (&p)[2]) {
      const int q1 = min(q0 + QT, t.M) - 1;
      bool live, partly;
      look(a, t, kb, q0 / t.group, q1 / t.group, live, partly);
      if (!live) return 0.f;
      const uint32_t have = ld.paged(p);
      const Key key = key_of(a, t, kb + l32, (have >> l32) & 1u ? 0 : -1);
      partly = partly || ld.hole(kb, p);
      f32x16 x;
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = 0.f;
      u32x4 kf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) kf[i] = chunk(st, i);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        x = mma(qf[i], kf[i & 3], x, T());
        if (i + 4 < NQ) kf[i & 3] = chunk(st, i + 4);
      }
      wait_lds();
      return weigh<T>(x, a, t, key, sAsk, 0, partly);
    };
    int held = 0;  // tiles whose sums are in the LDS, the last of them before kt
    auto flush = [&](int kt) {
      wait_lds();
      const int from = block(kt - held);
      float* to = m.mass + ((size_t)t.seq * a.c.nkv + t.head) * ((size_t)a.c.max_pages << a.c.page_lg);
      float old[HOLD / 2];
#pragma unroll
      for (int i = 0; i < HOLD / 2; ++i) {
        const int k = 2 * i + h, slot = from + k * KT + l32;
        old[i] = k < held && slot < t.len ? to[slot] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < HOLD / 2; ++i) {
        const int k = 2 * i + h, slot = from + k * KT + l32;
        if (k < held && slot < t.kend) to[slot] = slot >= t.len && a.mask ? 0.f : old[i] + sGot[wv][k][l32];
      }
      held = 0;
    };
    auto keep = [&](float got, int kt) {
      got = sum_x32(got);
      if (h == 0) sGot[wv][held][l32] = got;
      if (++held == HOLD || kt + 1 == k1) flush(kt + 1);
    };
    if (t.M <= QT) {
      fetch(0);
#pragma unroll
      for (int i = 0; i < NQ; ++i) qf[i] = chunk((const LB*)sQ, i);
      for (int kt = s.kt; kt < k1; kt += 2) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          LB *st = b ? (LB*)sB[wv] : (LB*)sA[wv], *nx = b ? (LB*)sA[wv] : (LB*)sB[wv];
          if (kt + b >= k1) break;
          const bool more = kt + b + 1 < k1;
          if (more) {
            ld.look(block(kt + b + 1), nat);
            ld.issue(a.k, nx, nat, 0);
            wait_vm<Ld::NI>();
          } else {
            wait_vm<0>();
          }
          keep(step(st, block(kt + b), 0, at), kt + b);
          at[0] = nat[0], at[1] = nat[1];
        }
      }
    } else {
      for (int kt = s.kt; kt < k1; ++kt) {
        LB* st = (LB*)sA[wv];
        if (kt > s.kt) {
          ld.look(block(kt), at);
          ld.issue(a.k, st, at, 0);
        }
        const int2 q = steps_of(a, t, kt);
        float got = 0.f;
        wait_vm<0>();
        for (int qt = q.x; qt < q.y; ++qt) {
          fetch(qt * QT);
#pragma unroll
          for (int i = 0; i < NQ; ++i) qf[i] = chunk((const LB*)sQ, i);
          got += step(st, block(kt), qt * QT, at);
        }
        wait_lds();
        keep(got, kt);
      }
    }
  }
}

// Many rows to a sequence: bound by exponentials (a quarter of the vector
// rate) beside the matrix cores. Keys stay in registers, queries go by in steps
// of 64 through two stages in the LDS, the next step on its way: one barrier to
// a step, and the products of a step's second half beside the exponentials of
// its first. Two chunks of 2,000 rows behind 2,000 to 6,000 slots, 32 heads on 8
// of 128 (150 GFLOP): 221 us, 0.68 PFLOP/s; with steps of 32 and a third stage
// 255 us, with queries through registers 641 us.
template <typename T, int HDP>
__global__ __launch_bounds__(256, (mass_waves<T, HDP>())) void k_mass_many(MassArgs m) {
  constexpr int QS = 2 * QT, RB = HDP * (int)sizeof(T), NQ = RB / 32, CPR = RB / 16, RPI = 1024 / RB, NI = QS / RPI;
  constexpr int LW = NI / 4;  // loads of a stage by a wave
  static_assert(LW >= 1 && LW <= 8, "a wave loads whole pieces of a stage");
  constexpr int AS = 256;  // queries whose asks are fetched at a time, one a thread
  const Args& a = m.a;
  __shared__ __attribute__((aligned(1024))) unsigned char s0[QS * RB], s1[QS * RB];
  __shared__ __attribute__((aligned(16))) Asks<AS> sAsk[2];
  const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
  const int hb = a.c.hd * (int)sizeof(T), group = a.group;
  Row64 row{a};
  const long long tiles = row.count();
  if (tiles == 0) return;
  const int cuts = row.cuts(tiles, m.target);
  // Workgroups go round the eight XCDs: each takes an eighth of the units, so
  // that its L2 serves a head's queries to neighbouring tiles (221 us against 225).
  // Within it units go by in turn, since later slots are seen by fewer rows.
  const long long units = tiles * cuts, share = (units + 7) >> 3, step_by = gridDim.x >> 3;
  row.begin();
  Spot s;
  for (long long v = blockIdx.x >> 3; v < share; v += step_by) {
    const long long u = (blockIdx.x & 7) * share + v;
    if (u >= units) break;
    const long long tile = cuts > 1 ? u / cuts : u;
    if (!row.at(tile, s)) break;
    const Tile& t = s.t;
    const int cut = (int)(u - tile * cuts);
    const int2 all = steps_of(a, t, s.kt);
    const int q0 = all.x + (int)((long long)(all.y - all.x) * cut / cuts);
    const int q1 = all.x + (int)((long long)(all.y - all.x) * (cut + 1) / cuts);
    const int slot = s.kt * KT + wv * 32 + l32, kb = s.kt * KT + wv * 32;
    float acc = 0.f;
    if (q0 < q1) {
      const int id = page_id(a, t, slot);
      u32x4 kf[NQ];
      load_key<T>(a, t, slot, id, kf);
      const Key key = key_of(a, t, slot, id);
      const bool hole = __any(key.page < 0);
      const int per = QS / group, rest = QS - per * group;  // tokens and heads that a step goes on by
      int tok0 = (int)((unsigned)(q0 * QT) / (unsigned)group), g0 = q0 * QT - tok0 * group;  // of the step that is loaded next
      const int lrow = lane / CPR, lchunk = (lane % CPR) ^ swz<RB, 16>(lrow);
      const uint32_t ldb = (uint32_t)(a.ldq * (long long)sizeof(T));
      const char* qp = (const char*)a.q + ((size_t)(t.row0 + tok0) * (size_t)a.ldq + (size_t)(t.head * group) * a.c.hd) * sizeof(T);
      int qn = q0;  // the step that is loaded next
      auto offset = [&](int i) {  // of what this lane loads in its i-th load, from qp on
        const int r0 = (i * 4 + wv) * RPI, r = r0 + lrow, ch = lchunk ^ swz<RB, 16>(r0);
        int g = g0 + r, tk = (int)((unsigned)g / (unsigned)group);
        g -= tk * group;
        if (qn * QT + r >= t.M) tk = t.n - 1 - tok0, g = group - 1;
        return HDP * (int)sizeof(T) != hb && ch * 16 >= hb ? OOB : (uint32_t)tk * ldb + (uint32_t)(g * hb + ch * 16);
      };
      uint32_t off[8];
#pragma unroll
      for (int i = 0; i < LW; ++i) off[i] = offset(i);
      auto issue = [&](LB* dst) {
        if (qn < q1) {
          // (the same from step to step where the group divides it)
          if (rest != 0 || qn * QT + QS > t.M)
#pragma unroll
            for (int i = 0; i < LW; ++i) off[i] = offset(i);
          const Rsrc rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(qp), (short)0, 0x7FFFFFFF, 0x00020000);
#pragma unroll
          for (int i = 0; i < LW; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LDS_AS void*)(dst + (i * 4 + wv) * 1024), 16, off[i], 0, 0, 0);
          const int was = tok0;
          tok0 += per, g0 += rest;
          if (g0 >= group) g0 -= group, ++tok0;
          qp += (size_t)(uint32_t)(tok0 - was) * ldb;
        }
        qn += 2;
      };
      Ask ask;
      int am = q0 * QT + tid;  // the query whose ask this thread fetches next
      auto ask_for = [&] {
        const int mm = am < t.M ? am : t.M - 1, tok = (int)((unsigned)mm / (unsigned)group);
        ask.load(a, t, am, tok, mm - tok * group);
        am += AS;
      };
      __syncthreads();  // the last unit's stages and asks are worked off
      issue((LB*)s0);
      ask_for();
      ask.put(sAsk[0], tid);
      int st0 = (int)((unsigned)(q0 * QT) / (unsigned)group), sg0 = q0 * QT - st0 * group;  // first query of the step at hand
      auto step = [&](auto phase, int qt) {
        constexpr int P = decltype(phase)::value;
        LB *at = P ? (LB*)s1 : (LB*)s0, *to = P ? (LB*)s0 : (LB*)s1;
        const int k = (qt - q0) >> 1, ab = (k >> 2) & 1, i0 = (k & 3) * QS;
        if ((k & 3) == 3) ask.put(sAsk[ab ^ 1], tid);
        wait_vm<0>();  // this step's queries are here,
        barrier();     // and the other stage is worked off
        issue(to);
        if ((k & 3) == 0 && qt + 8 < q1) ask_for();
        int n0 = st0 + per, ng = sg0 + rest;
        if (ng >= group) ng -= group, ++n0;
        const int tok1 = min(ng ? n0 : n0 - 1, t.n - 1);
        bool live, partly;
        look(a, t, kb, st0, tok1, live, partly);
        st0 = n0, sg0 = ng;
        if (a.span && live) {  // (nobody of the step sees them: documents)
          const Asks<AS>& q = sAsk[ab];
          const int i = i0 + lane;
          live = __any(q.own[i] > kb && q.lo[i] < kb + 32);
          partly = kb + 32 > t.kend || __any(q.own[i] < kb + 32 || q.lo[i] > kb) || (a.window && a.depth) ||
                   (a.mask && kb + 32 > t.len);
        }
        partly = partly || hole;
        if (!live) return;
        f32x16 x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          u32x4 qf[NQ];
#pragma unroll
          for (int i = 0; i < NQ; ++i)
            qf[i] = *(const LDS_AS u32x4*)(at + (e * QT + l32) * RB + (((2 * i + h) ^ swz<RB, 16>(l32)) * 16));
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < 16; ++j) x[e][j] = 0.f;
#pragma unroll
          for (int i = 0; i < NQ; ++i) x[e] = mma(qf[i], kf[i], x[e], T());
        }
        acc += weigh<T>(x[0], a, t, key, sAsk[ab], i0, partly);
        if (qt + 1 < q1) acc += weigh<T>(x[1], a, t, key, sAsk[ab], i0 + QT, partly);
      };
      for (int qt = q0;; qt += 4) {
        step(std::integral_constant<int, 0>(), qt);
        if (qt + 2 >= q1) break;
        step(std::integral_constant<int, 1>(), qt + 2);
        if (qt + 4 >= q1) break;
      }
    }
    acc = sum_x32(acc);
    if (cuts > 1) {
      if (h == 0) m.part[u * KT + wv * 32 + l32] = acc;
    } else if (h == 0) {
      put_mass(m, t, slot, acc);
    }
  }
}

// Tiles whose queries went to several units: their sums, in order.
__global__ __launch_bounds__(KT) void k_mass_join(MassArgs m) {
  Row64 row{m.a};
  const long long tiles = row.count();
  if (tiles == 0) return;
  const int cuts = row.cuts(tiles, m.target);
  if (cuts == 1) return;
  row.begin();
  Spot s;
  for (long long i = blockIdx.x; i < tiles; i += gridDim.x) {
    if (!row.at(i, s)) break;
    float got = 0.f;
    for (int c = 0; c < cuts; ++c) got += m.part[(i * cuts + c) * KT + threadIdx.x];
    put_mass(m, s.t, s.kt * KT + (int)threadIdx.x, got);
  }
}

// Many rows to a sequence: more than one step of queries, on average; up to
// there a tile's queries need no barrier. (Rows so far apart that a step's
// offsets pass 31 bits take the other kernel.)
bool mass_many(const MassDesc& d) {
  const long long rows = (long long)d.t.r.n_rows * (d.t.nq / d.t.c.nkv), esz = d.t.c.dtype == DT_BF16 ? 2 : 4;
  return rows > (long long)QT * d.t.r.n_ent && d.t.ldq * esz <= (1ll << 31) / (2 * QT + 2);
}
int mass_wgs(const MassDesc& d) {
  const bool wide = pad_hd(d.t.c.dtype, d.t.c.hd) * (d.t.c.dtype == DT_BF16 ? 2 : 4) > 256;
  return std::max(8, d.t.cus / 8 * 8) * (mass_many(d) ? (wide ? 2 : 3) : (wide ? 1 : 2));
}
// Units that a launch wants: more than one to a workgroup, since they are uneven.
// (For the scratch's size the row stride does not count.)
int mass_target(const MassDesc& d) {
  const long long rows = (long long)d.t.r.n_rows * (d.t.nq / d.t.c.nkv);
  return rows > (long long)QT * d.t.r.n_ent ? 12 * std::max(8, d.t.cus / 8 * 8) : 0;
}

template <typename T, int HDP>
void run_mass(const MassDesc& d, const MassArgs& m, hipStream_t st) {
  const dim3 grid(mass_wgs(d)), wg(256);
  if (m.target) hipLaunchKernelGGL((k_mass_many<T, HDP>), grid, wg, 0, st, m);
  else hipLaunchKernelGGL((k_mass_few<T, HDP>), grid, wg, 0, st, m);
}

}  // namespace

size_t mass_scratch(const MassDesc& d) { return (size_t)2 * mass_target(d) * KT * 4; }

hipError_t launch_mass(const MassDesc& x, hipStream_t st) {
  const TreeAttnDesc& d = x.t;
  if (d.r.n_rows <= 0 || d.r.n_ent <= 0) return hipSuccess;
  MassArgs m{};
  Args& a = m.a;
  a.c = d.c;
  a.r = d.r;
  a.nq = d.nq;
  a.group = d.nq / d.c.nkv;
  a.q = d.q;
  a.ldq = d.ldq;
  a.mask = d.mask;
  a.mask_words = d.mask_words;
  a.c2 = d.s.scale * LOG2E;
  shape_args(d.s, &a);
  a.lse = d.lse;
  const size_t layer = (size_t)d.layer * d.c.n_pages * d.c.nkv * d.c.page * d.c.hd * (d.c.dtype == DT_BF16 ? 2 : 4);
  a.k = (const char*)d.c.k + layer;
  m.mass = x.mass + (size_t)d.layer * d.c.n_seqs * d.c.nkv * ((size_t)d.c.max_pages << d.c.page_lg);
  m.part = (float*)d.scratch;
  m.target = mass_many(x) ? mass_target(x) : 0;
  const int hdp = pad_hd(d.c.dtype, d.c.hd);
  if (d.c.dtype == DT_BF16) {
    if (hdp == 64) run_mass<uint16_t, 64>(x, m, st);
    else if (hdp == 128) run_mass<uint16_t, 128>(x, m, st);
    else run_mass<uint16_t, 256>(x, m, st);
  } else {
    if (hdp > 128) return hipErrorInvalidValue;
    if (hdp == 64) run_mass<float, 64>(x, m, st);
    else run_mass<float, 128>(x, m, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || m.target == 0) return e;
  hipLaunchKernelGGL(k_mass_join, dim3(mass_wgs(x)), dim3(KT), 0, st, m);
  return hipGetLastError();
}

}  // namespace vla
