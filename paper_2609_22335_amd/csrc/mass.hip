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
  int c0;

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
    for (int c = 0; c < a.r.n_ent; c += 64) {
      load(c);
      sum += lane_of(incl, 63);
    }
    return sum;
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

template <typename T, int HDP>
__global__ __launch_bounds__(256, 2) void k_mass(MassArgs m) {
  constexpr int RB = HDP * (int)sizeof(T), NQ = RB / 32, LD = QT * RB / 16 / 256;
  static_assert(LD >= 1, "a thread stages whole chunks");
  const Args& a = m.a;
  __shared__ __attribute__((aligned(1024))) unsigned char sQ[2][QT * RB];
  // of a step's queries: lse (log2 units; plus infinity where it gives nothing), slope, place, first and last slot seen
  __shared__ __attribute__((aligned(16))) float sLse[2][QT], sSlope[2][QT];
  __shared__ __attribute__((aligned(16))) int sPlace[2][QT], sLo[2][QT], sOwn[2][QT];
  const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
  const int hb = a.c.hd * (int)sizeof(T);
  Row64 row{a};
  const long long tiles = row.count();
  if (tiles == 0) return;
  // a tile's queries go to `cuts` units where there are few tiles
  int cuts = 1;
  if (m.target > 0 && tiles < m.target) cuts = (int)((m.target + tiles - 1) / tiles);
  const long long units = tiles * cuts, wgs = gridDim.x;
  // few tiles: units in turn, since later slots are seen by fewer rows; else runs of neighbouring tiles
  const long long quota = cuts > 1 ? 1 : (units + wgs - 1) / wgs, stride = cuts > 1 ? wgs : 1;
  long long u = (long long)blockIdx.x * quota, end = cuts > 1 ? units : min(units, u + quota);
  if (u >= end) return;
  row.begin();
  Spot s;
  int held_seq = -1, held_head = -1, held_row0 = -1;  // whose queries are staged, where one step is all
  u32x4 kf[NQ], qn[LD];
  float nl = 0.f, nsl = 0.f;
  Row nr{};
  for (; u < end; u += stride) {
    const long long tile = cuts > 1 ? u / cuts : u;
    if (!row.at(tile, s)) break;
    const Tile& t = s.t;
    const int cut = (int)(u - tile * cuts);
    const int2 all = steps_of(a, t, s.kt);
    const int q0 = all.x + (int)((long long)(all.y - all.x) * cut / cuts);
    const int q1 = all.x + (int)((long long)(all.y - all.x) * (cut + 1) / cuts);
    const int slot = s.kt * KT + wv * 32 + l32, kb = s.kt * KT + wv * 32;
    // the lane's key
    const int page = page_of(a.c, t.seq, slot, t.kend);
    const bool have = page >= 0;
    const char* kp = a.k + (((size_t)(have ? page : 0) * a.c.nkv + t.head) * a.c.page + (have ? slot & (a.c.page - 1) : 0)) * (size_t)hb;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int ch = 2 * i + h;
      kf[i] = ch * 16 < hb ? *(const u32x4*)(kp + ch * 16) : u32x4{0, 0, 0, 0};
    }
    int key = slot;
    if (a.depth && slot >= t.len && slot < t.kend) key = place_of(a, t, t.row0 + slot - t.len, slot - t.len);
    auto fetch = [&](int qt) {
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int c = tid + 256 * i, r = c / (RB / 16), ch = c % (RB / 16);
        const int mm = qt * QT + r < t.M ? qt * QT + r : t.M - 1, tok = mm / t.group;
        const char* qp = (const char*)a.q + ((size_t)(t.row0 + tok) * (size_t)a.ldq +
                                             (size_t)(t.head * t.group + (mm - tok * t.group)) * a.c.hd) * sizeof(T);
        qn[i] = ch * 16 < hb ? *(const u32x4*)(qp + ch * 16) : u32x4{0, 0, 0, 0};
      }
      if (tid < QT) {
        const int mm = qt * QT + tid, mc = mm < t.M ? mm : t.M - 1, tok = mc / t.group;
        const int hq = t.head * t.group + (mc - tok * t.group);
        nr = row_of<true>(t, tok);
        const float v = a.lse[(size_t)(t.row0 + tok) * a.nq + hq];
        nl = mm < t.M && v - v == 0.f ? v * LOG2E : INFINITY;
        nsl = a.slopes ? a.slopes[hq] * LOG2E : 0.f;
      }
    };
    auto stage = [&](int b) {
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int c = tid + 256 * i, r = c / (RB / 16), ch = c % (RB / 16);
        *(u32x4*)(sQ[b] + r * RB + ((ch ^ swz<RB, 16>(r)) * 16)) = qn[i];
      }
      if (tid < QT) {
        sLse[b][tid] = nl, sSlope[b][tid] = nsl, sPlace[b][tid] = nr.place;
        sLo[b][tid] = nr.lo, sOwn[b][tid] = nr.own;
      }
    };
    const bool one = t.M <= QT, again = one && t.seq == held_seq && t.head == held_head && t.row0 == held_row0;
    if (q0 < q1) held_seq = one ? t.seq : -1, held_head = t.head, held_row0 = t.row0;
    float acc = 0.f;
    if (!again && q0 < q1) {
      __syncthreads();  // the last unit's queries are worked off
      fetch(q0);
      stage(0);
      __syncthreads();
    }
    for (int qt = q0; qt < q1; ++qt) {
      const int b = one ? 0 : (qt - q0) & 1;
      if (qt + 1 < q1) fetch(qt + 1);
      const int own = sOwn[b][l32], lo = sLo[b][l32];
      const bool live = __any(own > kb && lo < kb + 32) && kb < t.kend;
      if (live) {
        bool partly = __any(own < kb + 32 || lo > kb) || kb + 32 > t.kend || !__all(have);
        if ((a.mask || (a.window && a.depth)) && kb + 32 > t.len) partly = true;
        f32x16 x;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = 0.f;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const u32x4 qf = *(const u32x4*)(sQ[b] + l32 * RB + (((2 * i + h) ^ swz<RB, 16>(l32)) * 16));
          x = mma(qf, kf[i], x, T());
        }
        // (element j: query 8 (j / 4) + j % 4 + 4 h of the step, the lane's key)
        const bool plain = a.cap2 == 0.f && !a.slopes;
        if (a.cap2 > 0.f) cap_scores<T>(x, a);
        else if (!plain)
#pragma unroll
          for (int j = 0; j < 16; ++j) x[j] *= a.c2;
        float add = 0.f;
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          const int r = 8 * j4 + 4 * h;
          const f32x4 ls = *(const f32x4*)(sLse[b] + r);
          if (a.slopes) {
            const f32x4 sl = *(const f32x4*)(sSlope[b] + r);
            const int4 pl = *(const int4*)(sPlace[b] + r);
            const int p4[4] = {pl.x, pl.y, pl.z, pl.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[4 * j4 + i] = __builtin_fmaf(-sl[i], __builtin_fabsf((float)(p4[i] - key)), x[4 * j4 + i]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[4 * j4 + i] = ex2(plain ? __builtin_fmaf(x[4 * j4 + i], a.c2, -ls[i]) : x[4 * j4 + i] - ls[i]);
          if (partly) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              bool see = have && slot < sOwn[b][r + i] && slot >= sLo[b][r + i];
              if (a.mask && slot >= t.len) see = false;  // (a tree's drafts begin at nothing)
              if (a.window) see = see && (long long)sPlace[b][r + i] - key < a.window;
              x[4 * j4 + i] = see ? x[4 * j4 + i] : 0.f;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) add += x[4 * j4 + i];
        }
        // a key that is not finite makes NaN of rows that give nothing as well
        if (__any(add != add)) {
          add = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) add += sLse[b][8 * (j / 4) + j % 4 + 4 * h] < INFINITY ? x[j] : 0.f;
        }
        acc += add;
      }
      if (qt + 1 < q1) {
        stage(b ^ 1);
        __syncthreads();
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
  if (tiles == 0 || tiles >= m.target) return;
  const int cuts = (int)((m.target + tiles - 1) / tiles);
  row.begin();
  Spot s;
  for (long long i = blockIdx.x; i < tiles; i += gridDim.x) {
    if (!row.at(i, s)) break;
    float got = 0.f;
    for (int c = 0; c < cuts; ++c) got += m.part[(i * cuts + c) * KT + threadIdx.x];
    put_mass(m, s.t, s.kt * KT + (int)threadIdx.x, got);
  }
}

int mass_wgs(const MassDesc& d) { return std::max(8, d.t.cus / 8 * 8) * 2; }
// Units that a launch wants: more than one to a workgroup, since they are uneven.
int mass_target(const MassDesc& d) {
  const long long rows = (long long)d.t.r.n_rows * (d.t.nq / d.t.c.nkv);
  return rows > (long long)QT * d.t.r.n_ent ? 4 * mass_wgs(d) : 0;
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
  m.target = mass_target(x);
  const dim3 grid(mass_wgs(x)), wg(256);
  const int hdp = pad_hd(d.c.dtype, d.c.hd);
  if (d.c.dtype == DT_BF16) {
    if (hdp == 64) hipLaunchKernelGGL((k_mass<uint16_t, 64>), grid, wg, 0, st, m);
    else if (hdp == 128) hipLaunchKernelGGL((k_mass<uint16_t, 128>), grid, wg, 0, st, m);
    else hipLaunchKernelGGL((k_mass<uint16_t, 256>), grid, wg, 0, st, m);
  } else {
    if (hdp > 128) return hipErrorInvalidValue;
    if (hdp == 64) hipLaunchKernelGGL((k_mass<float, 64>), grid, wg, 0, st, m);
    else hipLaunchKernelGGL((k_mass<float, 128>), grid, wg, 0, st, m);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || m.target == 0) return e;
  hipLaunchKernelGGL(k_mass_join, dim3(mass_wgs(x)), dim3(KT), 0, st, m);
  return hipGetLastError();
}

}  // namespace vla
