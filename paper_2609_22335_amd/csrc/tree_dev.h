// Attention of drafted tokens over a paged KV cache: every row attends to all
// committed slots of its sequence and to the drafts that its mask names (or,
// without a mask, to the drafts up to itself).
//
// The rows of one sequence and KV head (tokens x query heads of the group)
// form tiles that share K and V. Scores are computed transposed (S^T = K Q^T),
// so that a lane holds one query: the running maximum and sum are one value a
// lane, and the probabilities are, without leaving their registers, the right
// operand of O^T += V^T P^T.
//
// With SH the scores are shaped before the softmax (capped, biased by the
// distance), rows see spans or windows of slots, and the log-sum-exp goes out
// beside the result. Each kernel is compiled without (tree.hip) and with it
// (scores.hip).
#pragma once
#include <algorithm>
#include <type_traits>

#include "paged_dev.h"

namespace vla {
using namespace pg;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
// Pointers into the LDS are typed as such: the compiler must not lose sight of
// their address space.
#define LDS_AS __attribute__((address_space(3)))
typedef LDS_AS unsigned char LB;
typedef __amdgpu_buffer_rsrc_t Rsrc;
constexpr uint32_t OOB = 0x80000000u;
constexpr float LOG2E = 1.4426950408889634f;

// s_waitcnt operand that leaves n vector memory operations in flight
constexpr int vmcnt(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }
template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt(vmcnt(N));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() {
  wait_lds();  // (this wave's writes are in the LDS; loads into it may be on their way)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// All waves meet; what this one has in flight stays there.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct Args {
  PagedCache c;
  PagedRows r;
  int nq, group;
  const void* q;
  void* out;
  long long ldq, ldo;
  const uint32_t* mask;
  int mask_words;
  float c2;  // scale * log2(e)
  // (SH) Scores are worked on in units of log2(e): cap2 = cap log2(e) (0: no
  // cap) and k1 = 2 scale log2(e) / cap.
  float k1, cap2;
  const float* slopes;
  const int32_t* depth;
  const int2* span;
  int window;
  float* lse;
  const char* k;  // the layer's K and V
  const char* v;
  float* part;   // [2 W][rows][hd], then [2 W][rows][2]
  int4* desc;    // [W][2]: what the join reads
  int wgs;       // W
};

// The kernel's arguments, loaded anew: what a rare or late part of a kernel
// reads need not stand in scalar registers throughout its loop.
__device__ __forceinline__ const Args& fresh() {
  auto p = (const __attribute__((address_space(4))) Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Args*)p;
}

__device__ __forceinline__ long long lane_of(long long v, int i) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, i);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(v >> 32), i);
  return (long long)(((unsigned long long)hi << 32) | lo);
}

// A wave's entries for deal(), one a lane.
template <int BM, bool SH>
struct Lanes {
  const Args& a;
  Entry x;
  Geo<BM, SH> g;
  int persum;
  long long all, incl;

  static __device__ __forceinline__ float root(float v) { return __builtin_amdgcn_sqrtf(v); }
  __device__ __forceinline__ void load(int c0) {
    const int i = c0 + (int)(threadIdx.x & 63);
    x = Entry{-1, 0, 0, 0, 0};
    if (i < a.r.n_ent) x = entry_of(a.c, a.r, i);
  }
  __device__ __forceinline__ long long count(bool causal, int unit) {
    g.set(a.group, causal, x, unit);
    if constexpr (SH) g.slide(a.window, a.depth != nullptr);
    persum = g.sum();
    all = (long long)persum * a.c.nkv;
    incl = wave_scan(all);
    return lane_of(incl, 63);
  }
  __device__ __forceinline__ long long tiles() { return __builtin_amdgcn_readlane(wave_scan(g.tiles), 63); }
  __device__ __forceinline__ int at(long long u) { return __ffsll(__ballot(incl > u)) - 1; }
  __device__ __forceinline__ Entry entry(int l) {
    return Entry{__builtin_amdgcn_readlane(x.seq, l), __builtin_amdgcn_readlane(x.row0, l),
                 __builtin_amdgcn_readlane(x.n, l), __builtin_amdgcn_readlane(x.len, l),
                 __builtin_amdgcn_readlane(x.cap, l)};
  }
  __device__ __forceinline__ int units(int l) { return __builtin_amdgcn_readlane(persum, l); }
  __device__ __forceinline__ long long before(int l) { return lane_of(incl, l) - lane_of(all, l); }
};
template <int BM, int BN, int LONG, bool SH>
__device__ __forceinline__ Tile dealt(Run& r, bool first) {
  const Args& a = fresh();
  Lanes<BM, SH> lanes{a};
  Batch b{a.r.n_ent, a.c.nkv, a.group, a.wgs, a.mask == nullptr};
  if constexpr (SH) b.causal = b.causal && a.span == nullptr, b.back = a.window, b.fixed = a.depth != nullptr;
  return deal<BM, BN, LONG, SH>(r, first, b, (int)blockIdx.x, lanes);
}
// The tile behind t in the run.
template <int BM, int BN, int LONG, bool SH>
__device__ __forceinline__ Tile next(Run& r, const Tile& t) {
  Tile n = t;
  return more<BM, BN, SH>(r, n, fresh().c.nkv) ? n : dealt<BM, BN, LONG, SH>(r, false);
}
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

// 16-byte chunk c of row r (of RB bytes) of a tile sits at position
// c ^ swz(r). The LDS serves 256 bytes a cycle when they lie in different
// 16-byte columns of a 256-byte line: with the swizzle over 16 columns 16 rows
// read at one chunk (K fragments) do, and so do four rows read at four chunks
// (V, transposed). 128 bf16 a row: K 245 and V 147 bytes a cycle, against 128
// and 118 over 8 columns. Those take fewer addresses (the rest of a fragment's
// is an immediate) and do where the LDS is not what a wave waits for.
template <int RB, int COLS>
__device__ __forceinline__ constexpr int swz(int r) {
  return COLS == 8 ? ((r & 3) << 1) | ((r >> 2) & 1)
         : RB == 128 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
}
// Byte b of a row whose first byte's column is x (a lane's constant): the part
// that the swizzle reaches, and the rest, an immediate.
template <int RB, int COLS>
__device__ __forceinline__ int turned(int x, int b) {
  constexpr int IN = (RB < 16 * COLS ? RB : 16 * COLS) - 1;
  return (x ^ (b & IN)) + (b & ~IN);
}

__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c, uint16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c, float) {
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  return c;
}

// max and sum over lanes l and l ^ 32
__device__ __forceinline__ float max_x32(float x) {
  const uint32_t v = __float_as_uint(x);
  auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_x32(float x) {
  const uint32_t v = __float_as_uint(x);
  auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// Where 16 slots lie: their first row in the cache's bytes from the layer's
// base, and the bytes from there on that may be read (to the page's end, the
// last key at most; 0 without a page).
struct Place {
  uint32_t lo, hi, bytes;
};

// Loads of 32 keys' K or V into the LDS, by the part `part` of PARTS waves.
// A buffer resource spans what is left of one page of one head: slots behind
// the last key and chunks behind the head dim lie out of its range and become
// zeros.
template <typename T, int HDP, int PARTS, int COLS>
struct Loader {
  static constexpr int RB = HDP * (int)sizeof(T), CPR = RB / 16, RPI = 1024 / RB, NI = 32 / RPI;
  int lrow, lchunk, hb;  // the lane's row and chunk of a load; bytes of a row in memory
  uint32_t pbytes;       // a page's part of one KV head
  const __attribute__((address_space(4))) int32_t* table;
  int page, page_lg, n_pages, nkv, head, kend;

  __device__ __forceinline__ void set(const Tile& t) {
    const Args& a = fresh();
    const int lane = threadIdx.x & 63;
    lrow = lane / CPR;
    lchunk = (lane % CPR) ^ swz<RB, COLS>(lrow);
    hb = a.c.hd * (int)sizeof(T);
    pbytes = (uint32_t)(a.c.page * hb);
    table = (const __attribute__((address_space(4))) int32_t*)(a.c.table + (size_t)t.seq * a.c.max_pages);
    page = a.c.page, page_lg = a.c.page_lg, n_pages = a.c.n_pages, nkv = a.c.nkv, head = t.head, kend = t.kend;
  }
  __device__ __forceinline__ Place place(int s0) const {
    const int left = kend - s0;
    const int id = left > 0 ? table[s0 >> page_lg] : -1;
    const bool ok = (unsigned)id < (unsigned)n_pages;
    const int at = s0 & (page - 1), room = page - at;
    const unsigned long long off =
        (unsigned long long)(uint32_t)((ok ? id : 0) * nkv + head) * pbytes + (uint32_t)(at * hb);
    return Place{(uint32_t)off, (uint32_t)(off >> 32), ok ? (uint32_t)((left < room ? left : room) * hb) : 0u};
  }
  // The same by lanes, for the halves of 32 blocks of 32 slots from block j
  // on: lane i's page, and from it its place (nothing from block j1 on).
  __device__ __forceinline__ int page_id(int j, int j1) const {
    const int lane = threadIdx.x & 63, s0 = 32 * j + 16 * lane;
    return table[s0 < kend && s0 < 32 * j1 ? s0 >> page_lg : 0];
  }
  // (returns whether slots without a page are among them)
  __device__ __forceinline__ bool spread(int j, int j1, int id, uint32_t& lo, uint32_t& hi, uint32_t& bytes) const {
    const int lane = threadIdx.x & 63, s0 = 32 * j + 16 * lane, left = kend - s0;
    const bool in = left > 0 && s0 < 32 * j1, ok = in && (unsigned)id < (unsigned)n_pages;
    const int at = s0 & (page - 1), room = page - at;
    const unsigned long long off =
        (unsigned long long)(uint32_t)((ok ? id : 0) * nkv + head) * pbytes + (uint32_t)(at * hb);
    lo = (uint32_t)off, hi = (uint32_t)(off >> 32), bytes = ok ? (uint32_t)((left < room ? left : room) * hb) : 0u;
    return __any(in && !ok);
  }
  // the places of slots kb and kb + 16 (which may lie in different pages)
  __device__ __forceinline__ void look(int kb, Place (&p)[2]) const {
    p[0] = place(kb);
    p[1] = place(kb + 16);
  }
  // A table may have no page for slots before the last key: nobody sees those.
  // Whether the slots from kb on have any such, by their places, and a bit for
  // each slot that has a page.
  __device__ __forceinline__ bool hole(int kb, const Place (&p)[2]) const {
    return (kb < kend && p[0].bytes == 0) || (kb + 16 < kend && p[1].bytes == 0);
  }
  __device__ __forceinline__ uint32_t paged(const Place (&p)[2]) const {
    return (p[0].bytes ? 0xFFFFu : 0u) | (p[1].bytes ? 0xFFFF0000u : 0u);
  }
  __device__ __forceinline__ uint32_t paged(int kb) const {
    Place p[2];
    look(kb, p);
    return paged(p);
  }
  __device__ __forceinline__ void issue(const char* src, LB* dst, const Place (&p)[2], int part) const {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const Rsrc rs = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char*>(src) + (((unsigned long long)p[hh].hi << 32) | p[hh].lo), (short)0, (int)p[hh].bytes,
          0x00020000);
      constexpr int PER = NI / 2;  // loads of a half, dealt out to the parts
#pragma unroll
      for (int i = 0; i < PER; i += PER >= PARTS ? PARTS : 1) {
        // (with fewer loads than parts, the halves go to different parts)
        if (PER < PARTS && hh * PER + i != part) continue;
        const int in = PER >= PARTS ? i + part : i;  // the load's place in its half
        const int r0 = in * RPI, idx = hh * PER + in;
        const int ch = lchunk ^ swz<RB, COLS>(r0);
        uint32_t off = (uint32_t)((r0 + lrow) * hb + ch * 16);
        if (HDP * (int)sizeof(T) != hb && ch * 16 >= hb) off = OOB;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LDS_AS void*)(dst + idx * 1024), 16, off, 0, 0, 0);
      }
    }
  }
};

// What a lane knows of its query's row: which one, and the slots that it sees
// at most, lo .. own - 1 (SH: lo, its place, and its slope in units of log2(e)).
struct Row {
  int row, own;
  int lo, place;
  float slope2;
};
// The place of row `row`, draft `tok` of the tile's sequence.
__device__ __forceinline__ int place_of(const Args& a, const Tile& t, int row, int tok) {
  if (!a.depth) return t.len + tok;
  const int d = a.depth[row];
  return t.len + (d < 0 ? 0 : d < (1 << 30) - 1 ? d : (1 << 30) - 1);
}
template <bool SH>
__device__ __forceinline__ Row row_of(const Tile& t, int tok) {
  Row x;
  x.row = t.row0 + tok;
  x.own = t.causal && t.len + tok + 1 < t.kend ? t.len + tok + 1 : t.kend;
  if constexpr (SH) {
    const Args& a = fresh();
    x.place = place_of(a, t, x.row, tok);
    x.lo = 0;
    if (a.span) {
      const int2 sp = a.span[x.row];
      x.lo = sp.x < 0 ? 0 : sp.x < t.kend ? sp.x : t.kend;
      x.own = sp.y < 0 ? 0 : sp.y < x.own ? sp.y : x.own;
    }
    if (a.window) {
      // (drafts whose places are not their slots are looked at one by one)
      int w = x.place - a.window + 1;
      if (a.depth && w > t.len) w = t.len;
      x.lo = w > x.lo ? w : x.lo;
    }
  }
  return x;
}
// Blocks from slot `safe` on and below slot `low` may hold slots that a row of
// the tile does not see; none sees one outside first .. last - 1.
struct Bounds {
  int safe, low, first, last;
};
template <int BM, bool SH>
__device__ __forceinline__ Bounds bounds_of(const Tile& t) {
  Bounds x;
  const int top = t.causal ? t.len + t.rt * BM / t.group + 1 : t.len;
  x.safe = top < t.kend ? top : t.kend;
  if constexpr (SH) {
    const Args& a = fresh();
    x.low = x.first = 0;
    x.last = t.kend;
    if (a.span || (a.window && a.depth)) {
      int own = 0x7FFFFFFF, lo = 0, first = 0x7FFFFFFF, last = 0;
      bool far = false;  // a draft may lie `window` or more places before a row (none lies before t.len)
#pragma unroll
      for (int i = 0; i < (BM + 63) / 64; ++i) {
        const int m = t.rt * BM + 64 * i + (int)(threadIdx.x & (BM < 64 ? BM - 1 : 63)), mc = m < t.M ? m : t.M - 1;
        const Row r = row_of<true>(t, mc / t.group);
        own = r.own < own ? r.own : own;
        lo = r.lo > lo ? r.lo : lo;
        first = r.lo < first ? r.lo : first;
        last = r.own > last ? r.own : last;
        far = far || r.place - t.len >= a.window;
      }
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        own = min(own, __shfl_xor(own, d));
        lo = max(lo, __shfl_xor(lo, d));
        first = min(first, __shfl_xor(first, d));
        last = max(last, __shfl_xor(last, d));
      }
      x.low = uni(lo), x.first = uni(first), x.last = uni(last);
      own = uni(own);
      x.safe = a.span && !a.mask ? own : own < x.safe ? own : x.safe;
      // (lo does not pass t.len: those drafts are looked at one by one)
      if (a.window && a.depth && __any(far)) x.safe = min(x.safe, t.len);
    } else if (a.window) {
      const int m1 = (t.rt + 1) * BM < t.M ? (t.rt + 1) * BM - 1 : t.M - 1;
      const int w1 = t.len + m1 / t.group - a.window + 1, w0 = t.len + t.rt * BM / t.group - a.window + 1;
      x.low = w1 > 0 ? w1 : 0;
      x.first = w0 > 0 ? w0 : 0;
    }
  }
  return x;
}
// The tile's blocks cut down to those of which a row sees something (one block
// is left of a part of which none is seen).
template <int BN>
__device__ __forceinline__ void narrow(Tile& t, const Bounds& x) {
  const int b0 = max(t.b0, x.first / BN), b1 = min(t.b1, (x.last + BN - 1) / BN);
  if (b0 < b1) t.b0 = b0, t.b1 = b1;
  else t.b1 = t.b0 + 1;
}

// Bit i: this lane's query sees slot kb + i (kb + 32 may pass the last key).
template <bool SH>
__device__ __forceinline__ uint32_t seen_bits(const Tile& t, int kb, const Row& x) {
  const int n = x.own - kb;
  uint32_t see = n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
  if constexpr (SH) {
    const int lo = x.lo - kb;
    if (lo > 0) see &= lo >= 32 ? 0u : 0xFFFFFFFFu << lo;
  }
  if (!t.causal && kb + 32 > t.len && (!SH || fresh().mask)) {
    const Args& a = fresh();
    const int j0 = kb - t.len;  // draft of bit 0
    uint32_t bits;
    const uint32_t* mw = a.mask + (size_t)x.row * a.mask_words;
    if (j0 >= 0) {
      const int wi = j0 >> 5, sh = j0 & 31;
      const uint32_t lo = wi < a.mask_words ? mw[wi] : 0u, hi = wi + 1 < a.mask_words ? mw[wi + 1] : 0u;
      bits = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
    } else {
      bits = (mw[0] << -j0) | ((1u << -j0) - 1u);
    }
    see &= bits;
  }
  if constexpr (SH) {
    const Args& a = fresh();
    if (a.window && a.depth && kb + 32 > t.len) {
#pragma unroll 1
      for (int i = kb < t.len ? t.len - kb : 0; i < 32 && kb + i - t.len < t.n; ++i) {
        const int j = kb + i - t.len;
        if ((long long)x.place - place_of(a, t, t.row0 + j, j) >= a.window) see &= ~(1u << i);
      }
    }
  }
  return see;
}

// S^T of NS x 32 keys (rows) and the lane's query. Fragments are read a set of
// four ahead of the products that use them: the compiler would wait for each
// read in turn.
template <typename T, int HDP, int NS, int NQ>
__device__ __forceinline__ void scores(const LB* kt, const u32x4 (&qf)[NQ], f32x16 (&s)[NS]) {
  constexpr int RB = HDP * (int)sizeof(T), SETS = NS * NQ / 4;
  const int l32 = threadIdx.x & 31, h = (threadIdx.x >> 5) & 1;
  const LB* base = kt + l32 * RB;
  const int x = (h ^ swz<RB, 8>(l32)) * 16;
  u32x4 kf[2][4];
  auto read = [&](int set) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      kf[set & 1][i] = *(const LDS_AS u32x4*)(base + turned<RB, 8>(x, (set % (NQ / 4) * 4 + i) * 32) +
                                             set / (NQ / 4) * 32 * RB);
  };
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int j = 0; j < 16; ++j) s[n][j] = 0.f;
  read(0);
#pragma unroll
  for (int set = 0; set < SETS; ++set) {
    if (set + 1 < SETS) read(set + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      s[set / (NQ / 4)] = mma(kf[set & 1][i], qf[set % (NQ / 4) * 4 + i], s[set / (NQ / 4)], T());
  }
}

// Probabilities as operands of the second product, in bf16 as the sum of two
// bf16 values: with few rows the matrix cores wait for memory anyway. (With
// many they are rounded once: an error of at most 2^-8 of each, as much as the
// result's own rounding may make.)
struct Probs {
  u32x4 hi[2], lo[2];
};
__device__ __forceinline__ void round_probs(const f32x16& s, Probs& p) {
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    uint32_t hw[4], lw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = s[8 * kk + 2 * i], p1 = s[8 * kk + 2 * i + 1];
      hw[i] = bf2(p0, p1);
      lw[i] = bf2(p0 - __uint_as_float(hw[i] << 16), p1 - __uint_as_float(hw[i] & 0xFFFF0000u));
    }
    p.hi[kk] = u32x4{hw[0], hw[1], hw[2], hw[3]};
    p.lo[kk] = u32x4{lw[0], lw[1], lw[2], lw[3]};
  }
}

// O^T += V^T P^T over NS x 32 keys. The first set of V's fragments (16 keys,
// every column) is read by first(), before the softmax; each further set
// before the products of the one ahead of it.
template <typename T, int HDP, int NS>
struct Values {
  static constexpr int RB = HDP * (int)sizeof(T), NDT = HDP / 32;
  u32x4 vf[2][sizeof(T) == 2 ? NDT : 1];
  const LB* base;
  int x;

  __device__ __forceinline__ void read(int set) {
    if constexpr (sizeof(T) == 2) {
      // 16 lanes read four keys of 16 head-dim columns, transposed: lane i
      // gets column i, the operand's keys 4 h .. + 3 and 8 + 4 h .. + 3
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        auto tr = [&](int k0) {
          const LB* q = base + turned<RB, 8>(x ^ (swz<RB, 8>(k0) * 16), dt * 64) + k0 * RB;
          return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)q));
        };
        const u32x2 u0 = tr(16 * set), u1 = tr(16 * set + 8);
        vf[set & 1][dt] = u32x4{u0.x, u0.y, u1.x, u1.y};
      }
    }
  }
  __device__ __forceinline__ void first(const LB* vt) {
    const int lane = threadIdx.x & 63, h = lane >> 5, il = lane & 15;
    if constexpr (sizeof(T) == 2) {
      base = vt + (4 * h + (il >> 2)) * RB + 8 * (il & 1);
      x = ((2 * ((lane >> 4) & 1) + ((il & 3) >> 1)) ^ swz<RB, 8>(4 * h + (il >> 2))) * 16;
    } else {
      base = vt;
      x = 0;
    }
    read(0);
  }
  __device__ __forceinline__ void add(const f32x16 (&s)[NS], const Probs (&p)[NS], f32x16 (&o)[NDT]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int set = 0; set < 2 * NS; ++set) {
        if (set + 1 < 2 * NS) read(set + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] = mma(vf[set & 1][dt], p[set >> 1].hi[set & 1], o[dt], T());
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] = mma(vf[set & 1][dt], p[set >> 1].lo[set & 1], o[dt], T());
      }
    } else {
      const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int key = 8 * (j / 4) + j % 4 + 4 * h;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const int d = 32 * dt + l32;
            const float v = *(const LDS_AS float*)(base + (32 * n + key) * RB + (((d / 4) ^ swz<RB, 8>(key)) * 16) + (d % 4) * 4);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[n][j], o[dt], 0, 0, 0);
          }
        }
    }
  }
};

// A masked key's V may hold anything, and 0 x inf is not 0. In blocks of which
// a row may be masked, values that are not finite are replaced by zeros before
// the product (clean_values, by PARTS waves; true when there was one), and
// added afterwards to the rows that see them (add_odd_values): a weight is
// positive, so the sum is what the value alone makes it.
__device__ __forceinline__ uint32_t odd_bits(uint32_t w, uint16_t) {
  return ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u) | ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u);
}
__device__ __forceinline__ uint32_t odd_bits(uint32_t w, float) {
  return (w & 0x7F800000u) == 0x7F800000u ? 0xFFFFFFFFu : 0u;
}
template <typename T, int HDP, int PARTS>
__device__ __forceinline__ bool clean_values(LB* vt, int part) {
  constexpr int NI = HDP * (int)sizeof(T) * 32 / 1024, U = NI / PARTS < 4 ? NI / PARTS : 4;
  LDS_AS u32x4* at = (LDS_AS u32x4*)(vt + part * 1024 + (threadIdx.x & 63) * 16);
  bool odd = false;
#pragma unroll 1
  for (int i = 0; i < NI / PARTS; i += U) {
    u32x4 c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) c[u] = at[(i + u) * PARTS * 64];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const u32x4 b = {odd_bits(c[u].x, T()), odd_bits(c[u].y, T()), odd_bits(c[u].z, T()), odd_bits(c[u].w, T())};
      if (b.x | b.y | b.z | b.w) {
        at[(i + u) * PARTS * 64] = c[u] & ~b;
        odd = true;
      }
    }
  }
  return __any(odd);
}
// Slots kb .. kb + 31, of which the lane's query sees `see`.
template <typename T, int HDP>
__device__ __forceinline__ void add_odd_values(const Tile& t, int kb, uint32_t see, f32x16 (&o)[HDP / 32]) {
  const Args& a = fresh();
  const int h = (threadIdx.x >> 5) & 1, hd = a.c.hd;
#pragma unroll 1
  for (int kk = 0; kk < 32; ++kk) {
    if (kb + kk >= t.kend) return;
    const int p = a.c.table[(size_t)t.seq * a.c.max_pages + ((kb + kk) >> a.c.page_lg)];
    if ((unsigned)p >= (unsigned)a.c.n_pages) continue;
    const T* row = (const T*)a.v + (((size_t)p * a.c.nkv + t.head) * a.c.page + ((kb + kk) & (a.c.page - 1))) * hd;
#pragma unroll
    for (int dt = 0; dt < HDP / 32; ++dt) {
      asm volatile("" ::: "memory");  // few loads at a time: this path is rare, its registers are not
#pragma unroll
      for (int j4 = 0; j4 < 4; ++j4) {
        const int d = 32 * dt + 8 * j4 + 4 * h;
        if (d >= hd) continue;
        uint32_t v[4];
        if constexpr (sizeof(T) == 2) {
          const u32x2 u = *(const u32x2*)(row + d);
          v[0] = u.x << 16, v[1] = u.x & 0xFFFF0000u, v[2] = u.y << 16, v[3] = u.y & 0xFFFF0000u;
        } else {
          const u32x4 u = *(const u32x4*)(row + d);
          v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (((see >> kk) & 1u) && (v[i] & 0x7F800000u) == 0x7F800000u) o[dt][4 * j4 + i] += __uint_as_float(v[i]);
      }
    }
  }
}

// Scores q k of 32 keys from kb on become cap tanh(scale q k / cap) - slope
// |distance|, in units of log2(e). tanh y = 1 - 2 / (e^{2 y} + 1), whose error
// is up to 9 2^-24 of the cap; fp32, and caps from CAP_LARGE on, take tanh's odd
// series where that would be more than the score's own rounding (y^2 below 1/4:
// what is cut off is less than 2^-23 of y).
constexpr float CAP_LARGE = 256.f;  // of cap2: 2^-13 of a score's unit
template <typename T>
__device__ __forceinline__ void cap_scores(f32x16& s, const Args& a) {
  const bool exact = sizeof(T) == 4 || a.cap2 >= CAP_LARGE;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float z = s[j] * a.k1;  // 2 y log2(e)
    float v = __builtin_fmaf(-2.f * a.cap2, __builtin_amdgcn_rcpf(ex2(z) + 1.f), a.cap2);
    if (exact) {
      const float y = z * 0.34657359f, y2 = y * y;  // (ln 2 / 2)
      float p = 0.0035921280f;                      // 21844 / 6081075
      p = __builtin_fmaf(p, y2, -0.0088632355f);    // -1382 / 155925
      p = __builtin_fmaf(p, y2, 0.021869488f);      // 62 / 2835
      p = __builtin_fmaf(p, y2, -0.053968254f);     // -17 / 315
      p = __builtin_fmaf(p, y2, 0.13333333f);       // 2 / 15
      p = __builtin_fmaf(p, y2, -0.33333333f);      // -1 / 3
      v = y2 < 0.25f ? a.cap2 * __builtin_fmaf(y * y2, p, y) : v;
    }
    s[j] = v;
  }
}
template <typename T>
__device__ __forceinline__ void shape(f32x16& s, const Args& a, const Tile& t, int kb, const Row& x) {
  const int h4 = 4 * (int)((threadIdx.x >> 5) & 1);
  if (a.cap2 > 0.f) {
    cap_scores<T>(s, a);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] *= a.c2;
  }
  if (a.slopes) {
    if (a.depth && kb + 32 > t.len) {  // drafts whose places are not their slots
      const int k = kb + (int)(threadIdx.x & 31), d = k - t.len;
      const int key = d < 0 ? k : place_of(a, t, t.row0 + (d < t.n ? d : t.n - 1), d);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float gap = (float)(x.place - __shfl(key, 8 * (j / 4) + j % 4 + h4));
        s[j] = __builtin_fmaf(-x.slope2, __builtin_fabsf(gap), s[j]);
      }
    } else {
      const float gap = (float)(x.place - kb - h4);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        s[j] = __builtin_fmaf(-x.slope2, __builtin_fabsf(gap - (float)(8 * (j / 4) + j % 4)), s[j]);
    }
  }
}
__device__ __forceinline__ float log_sum(float mx, float l) {
  return l > 0.f || l != l ? (mx + __builtin_amdgcn_logf(l)) * 0.69314718f : -INFINITY;
}

// One step of the running softmax over NS x 32 keys: s becomes the
// probabilities, o and l are rescaled when a row's maximum has grown by 2^8
// or more (sums of probabilities up to 2^8 lose nothing).
template <int NDT, int NS>
__device__ __forceinline__ void soften(f32x16 (&s)[NS], float c2, float& mx, float& l, f32x16 (&o)[NDT]) {
  float bm = s[0][0];
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int j = 0; j < 16; ++j) bm = fmaxf(bm, s[n][j]);
  bm = max_x32(bm) * c2;
  if (__any(bm > mx + 8.f)) {
    const float mn = fmaxf(mx, bm);
    const float f = mn == -INFINITY ? 1.f : ex2(mx - mn);
    mx = mn;
    l *= f;
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] *= f;
  }
  const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[n][j] = ex2(__builtin_fmaf(s[n][j], c2, -ref));
      l += s[n][j];
    }
}

__device__ __forceinline__ void hide(f32x16& s, uint32_t see, float none = -INFINITY) {
  const uint32_t half = see >> (4 * ((threadIdx.x >> 5) & 1));
#pragma unroll
  for (int j = 0; j < 16; ++j) s[j] = (half >> (8 * (j / 4) + j % 4)) & 1u ? s[j] : none;
}

// The lane's query (row m of the tile's rows, clamped to the last).
template <typename T, int NQ>
__device__ __forceinline__ void load_query(const Tile& t, int mc, u32x4 (&qf)[NQ]) {
  const Args& a = fresh();
  const int tok = mc / t.group, h = (threadIdx.x >> 5) & 1, hd = a.c.hd;
  const T* qp = (const T*)a.q + (size_t)(t.row0 + tok) * (size_t)a.ldq +
                (size_t)(t.head * t.group + (mc - tok * t.group)) * hd;
#pragma unroll
  for (int s = 0; s < NQ; ++s) {
    const int d0 = (2 * s + h) * El<T>::VEC;
    qf[s] = d0 < hd ? *(const u32x4*)(qp + d0) : u32x4{0, 0, 0, 0};
  }
}

// Where row mm of the tile goes, and four results of it.
template <typename T>
__device__ __forceinline__ T* out_row(const Args& a, const Tile& t, int mm) {
  const int tk = mm / t.group;
  return (T*)a.out + (size_t)(t.row0 + tk) * (size_t)a.ldo + (size_t)(t.head * t.group + (mm - tk * t.group)) * a.c.hd;
}
template <typename T>
__device__ __forceinline__ void put4(T* dst, float inv, const float (&v)[4]) {
  if constexpr (sizeof(T) == 2) *(u32x2*)dst = u32x2{bf2(v[0] * inv, v[1] * inv), bf2(v[2] * inv, v[3] * inv)};
  else *(f32x4*)dst = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
}
__device__ __forceinline__ float inverse(float l) { return l > 0.f || l != l ? 1.f / l : 0.f; }

// The workgroup's run of blocks: calls f(tile, slot) for each of its tiles,
// slot being where a shared tile's part goes; what other workgroups hold of the last one is written down for the
// join.
template <int BM, int BN, int LONG, bool SH, typename F>
__device__ __forceinline__ void for_tiles(int wgs, F&& f) {
  Run r;
  Tile t = dealt<BM, BN, LONG, SH>(r, true);
  int4 desc = make_int4(0, 0, 0, 0), more = desc;
  while (t.b1 > t.b0) {
    if (t.parts) {
      desc = make_int4(t.parts, t.row0, t.head * t.group, t.rt);
      more = make_int4(t.M, t.group, r.w, 0);
    }
    f(t, 2 * r.w + ((SH ? t.first : t.b0 == 0) ? 1 : 0));
    if (r.u >= r.u_end) break;
    wait_vm<0>();  // no store of this tile in the next one's counts
    __syncthreads();
    t = next<BM, BN, LONG, SH>(r, t);
  }
  if (threadIdx.x == 0) {
    int4* to = fresh().desc + 2 * ((int)(blockIdx.x & 7) * (wgs >> 3) + (int)(blockIdx.x >> 3));  // by XCD
    to[0] = desc;
    to[1] = more;
  }
}

// Waves per SIMD (workgroups per CU) that a kernel's registers are to leave room for.
template <typename T, int HDP>
constexpr int many_waves() {
  return HDP * (int)sizeof(T) <= 256 ? 2 : 1;
}

// Few rows to a sequence: tiles of 32 rows, bound by the cache's bandwidth.
// Each wave streams its own 32 keys of a block of 128 through its own part of
// the LDS, without a barrier: the next K is on its way during softmax and
// P V, the next V during the next scores. The four waves' results are merged
// at the end. 16 single tokens behind 8,000 to 65,000 slots, 32 heads on 8 of
// 128 (1.85 GB): 332 us, 5.6 TB/s.
template <typename T, int HDP, bool SH>
__global__ __launch_bounds__(256, (many_waves<T, HDP>())) void k_tree_few(Args a) {
  constexpr int BM = 32, BN = 128;
  constexpr int RB = HDP * (int)sizeof(T), NQ = RB / 32, NDT = HDP / 32;
  typedef Loader<T, HDP, 1, 8> Ld;
  static_assert(2 * Ld::NI < 60, "loads in flight");
  __shared__ __attribute__((aligned(1024))) unsigned char sK[4][32 * RB];
  __shared__ __attribute__((aligned(1024))) unsigned char sV[4][32 * RB];
  __shared__ float sM[4][32], sL[4][32], sF[4][32];
  __shared__ long long sAt[32];
  for_tiles<BM, BN, 1, SH>(a.wgs, [&](const Tile& dealt_tile, int slot) {
    const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
    Tile t = dealt_tile;
    const Bounds lim = bounds_of<BM, SH>(t);
    if constexpr (SH) narrow<BN>(t, lim);
    Ld ld;
    ld.set(t);
    const int kb0 = t.b0 * BN + wv * 32;
    LB *kl = (LB*)sK[wv], *vl = (LB*)sV[wv];
    Place at[2];
    const int m = t.rt * BM + l32, mc = m < t.M ? m : t.M - 1, tok = mc / t.group;
    u32x4 qf[NQ];
    load_query<T, NQ>(t, mc, qf);
    ld.look(kb0, at);
    ld.issue(a.k, kl, at, 0);
    ld.issue(a.v, vl, at, 0);
    Row me = row_of<SH>(t, tok);
    if constexpr (SH) me.slope2 = a.slopes ? a.slopes[t.head * t.group + (mc - tok * t.group)] * LOG2E : 0.f;
    auto partly = [&](int kb) { return kb + 32 > lim.safe || (SH && kb < lim.low); };
    f32x16 o[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float mx = -INFINITY, l = 0.f;
    bool odd = false;
    wait_vm<0>();  // (the first block waits for the query as well)
    for (int b = t.b0; b < t.b1; ++b) {
      const int kb = b * BN + wv * 32;
      const bool more = b + 1 < t.b1, masked = partly(kb) || ld.hole(kb, at);
      const uint32_t see = masked ? seen_bits<SH>(t, kb, me) & ld.paged(at) : 0u;
      if (b > t.b0) wait_vm<Ld::NI>();  // K is here, V may be on its way
      f32x16 s[1];
      scores<T, HDP, 1, NQ>(kl, qf, s);
      wait_lds();
      if (more) {
        ld.look(kb + BN, at);
        ld.issue(a.k, kl, at, 0);
      }
      if constexpr (SH) shape<T>(s[0], a, t, kb, me);
      if (masked) hide(s[0], see);
      soften<NDT, 1>(s, SH ? 1.f : a.c2, mx, l, o);
      Probs p[1];
      if constexpr (sizeof(T) == 2) round_probs(s[0], p[0]);
      if (more) wait_vm<Ld::NI>();  // V is here, the next K may be on its way
      else wait_vm<0>();
      if (masked) {
        odd |= clean_values<T, HDP, 1>(vl, 0);
        wait_lds();
      }
      Values<T, HDP, 1> vv;
      vv.first(vl);
      vv.add(s, p, o);
      wait_lds();
      if (more) ld.issue(a.v, vl, at, 0);
    }
    l = sum_x32(l);
    if (odd)
      for (int b = t.b0; b < t.b1; ++b) {
        const int kb = b * BN + wv * 32;
        ld.look(kb, at);
        if (partly(kb) || ld.hole(kb, at)) add_odd_values<T, HDP>(t, kb, seen_bits<SH>(t, kb, me), o);
      }
    // the four waves' results: each puts its own into the LDS (columns of the
    // first half where K was, the others where V was), two waves work out what
    // each counts for, then 256 threads add four columns of a row each, four
    // rows' reads out at once
    constexpr int HC = HDP / 2, CG = HDP / 4;
    const int rows = t.M - t.rt * BM < 32 ? t.M - t.rt * BM : 32;
    if (h == 0) sM[wv][l32] = mx, sL[wv][l32] = l;
    barrier();  // (every wave is done with K and V)
    if (l32 < rows) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        LDS_AS float* so = dt < NDT / 2 ? (LDS_AS float*)sK : (LDS_AS float*)sV;
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          const int c4 = (8 * dt + 2 * j4 + h) % (HC / 4);  // four columns
          *(LDS_AS f32x4*)(so + ((wv * 32 + l32) * HC) + ((c4 ^ (l32 & 7)) * 4)) =
              f32x4{o[dt][4 * j4], o[dt][4 * j4 + 1], o[dt][4 * j4 + 2], o[dt][4 * j4 + 3]};
        }
      }
    }
    const Args& z = fresh();
    float* pm = z.part + 2ll * z.wgs * BM * HDP + (size_t)slot * BM * 2;
    if (tid < 128) {
      const int k = tid >> 5, r = tid & 31;
      const float top = fmaxf(fmaxf(sM[0][r], sM[1][r]), fmaxf(sM[2][r], sM[3][r]));
      float den = 0.f, mine = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = sM[i][r] == -INFINITY ? 0.f : ex2(sM[i][r] - top);
        den = __builtin_fmaf(f, sL[i][r], den);
        mine = i == k ? f : mine;
      }
      sF[k][r] = t.whole ? mine * inverse(den) : mine;
      if (k == 0) {
        if (t.whole) {
          const int mm = t.rt * BM + r, tk = mm / t.group;
          sAt[r] = (long long)(t.row0 + tk) * z.ldo + (long long)(t.head * t.group + (mm - tk * t.group)) * z.c.hd;
          if constexpr (SH)
            if (z.lse && r < rows)
              z.lse[(size_t)(t.row0 + tk) * z.nq + t.head * t.group + (mm - tk * t.group)] = log_sum(top, den);
        } else if (r < rows) {
          pm[2 * r] = top, pm[2 * r + 1] = den;
        }
      }
    }
    barrier();
    const int total = rows * CG;
#pragma unroll 1
    for (int i0 = tid; i0 < total; i0 += 1024) {
      f32x4 y[4][4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + 256 * u < total ? i0 + 256 * u : i0, lm = i / CG, c4 = i % CG;
        const LDS_AS float* so = c4 < CG / 2 ? (const LDS_AS float*)sK : (const LDS_AS float*)sV;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          y[u][k] = *(const LDS_AS f32x4*)(so + ((k * 32 + lm) * HC) + (((c4 % (CG / 2)) ^ (lm & 7)) * 4));
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + 256 * u, lm = i / CG, col = i % CG * 4;
        if (i >= total) break;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) v += sF[k][lm] * y[u][k];
        if (t.whole) {
          const float w[4] = {v.x, v.y, v.z, v.w};
          if (col < z.c.hd) put4<T>((T*)z.out + sAt[lm] + col, 1.f, w);
        } else {
          *(f32x4*)(z.part + ((size_t)slot * BM + lm) * HDP + col) = v;
        }
      }
    }
  });
}

// What the many-row kernels do with the rows of a wave: row m's sums o over l,
// to out or, where a tile is shared, to the part `slot`.
template <typename T, int HDP, bool SH>
__device__ __forceinline__ void finish(const Tile& t, int slot, int wv, int m, float mx, float l,
                                       const f32x16 (&o)[HDP / 32]) {
  constexpr int BM = 128, NDT = HDP / 32;
  const Args& z = fresh();
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5, hd = z.c.hd;
  if (m >= t.M) return;
  if (t.whole) {
    const float inv = inverse(l);
    T* dst = out_row<T>(z, t, m) + 4 * h;
    if constexpr (SH)
      if (z.lse && h == 0) {
        const int tk = m / t.group;
        z.lse[(size_t)(t.row0 + tk) * z.nq + t.head * t.group + (m - tk * t.group)] = log_sum(mx, l);
      }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      if (32 * dt >= hd) break;
#pragma unroll
      for (int j4 = 0; j4 < 4; ++j4) {
        const float v[4] = {o[dt][4 * j4], o[dt][4 * j4 + 1], o[dt][4 * j4 + 2], o[dt][4 * j4 + 3]};
        put4<T>(dst + 32 * dt + 8 * j4, inv, v);
      }
    }
    return;
  }
  float* po = z.part + ((size_t)slot * BM + wv * 32) * HDP;
  float* pm = z.part + 2ll * z.wgs * BM * HDP + ((size_t)slot * BM + wv * 32) * 2;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int j4 = 0; j4 < 4; ++j4)
      // (in lane order: whole lines)
      *(f32x4*)(po + ((dt * 4 + j4) * 64 + lane) * 4) =
          f32x4{o[dt][4 * j4], o[dt][4 * j4 + 1], o[dt][4 * j4 + 2], o[dt][4 * j4 + 3]};
  if (h == 0) pm[2 * l32] = mx, pm[2 * l32 + 1] = l;
}

// Many rows to a sequence in bf16: tiles of 128 rows, 32 to a wave, bound by
// the matrix cores (and, over seconds, by the power that they may draw: the
// same call on zeros takes four fifths of the time). A wave keeps its matrix
// core and its vector unit busy side by side: the products K Q^T of the next
// 32 keys are issued between the exponentials of these, and V^T P^T between
// the last of those and the next maxima. Fragments are read four products
// ahead, also across the barrier in the middle of a step, and loads are out
// two steps ahead. Against one block after another, scores, softmax, products
// (both with two workgroups on a CU): chunks of 2,000 rows behind 4,000 slots,
// 32 heads on 8, 277 us against 293 at head dim 64 and 387 against 390 (0.85
// PFLOP/s, two sequences) at 128; 8 on 1 at head dim 256, one workgroup on a
// CU, 381 against 435.
// With CURVED (scores capped and not biased) the scores are kept as
// r = 1 / (e^{2 y} + 1), which is worked out beside the products of V: cap tanh y
// = cap (1 - 2 r), one product and sum before the exponential as for plain
// scores, and the largest score is the smallest r.
template <int HDP, bool SH, bool CURVED>
__global__ __launch_bounds__(256, (many_waves<uint16_t, HDP>())) void k_tree_many(Args a) {
  typedef uint16_t T;
  constexpr int BM = 128, BN = 32, RB = HDP * 2, NQ = RB / 32, NDT = HDP / 32;
  typedef Loader<T, HDP, 4, 16> Ld;
  constexpr int LW = Ld::NI / 2;  // loads of a stage by a wave
  // With two waves to a SIMD the new maxima are looked at beside products that
  // are out; a wave on its own is faster with that between its steps (head dim
  // 256, as above: 375 us against 420; head dim 64, two waves: 285 and 276).
  constexpr bool PAIR = many_waves<T, HDP>() == 2;
  constexpr int UP = PAIR ? 2 : 0;
  // A stage of the ring holds V of a block and K of the next one. (By name: the
  // compiler lets reads of one stage run beside loads into another only where
  // it can tell them apart.)
  __shared__ __attribute__((aligned(1024))) unsigned char s0[64 * RB], s1[64 * RB], s2[64 * RB], s3[64 * RB];
  __shared__ int sOdd;
  for_tiles<BM, BN, many_waves<T, HDP>(), SH>(a.wgs, [&](const Tile& dealt_tile, int slot) {
    const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6), l32 = lane & 31, h = lane >> 5, il = lane & 15;
    if (tid == 0) sOdd = 0;  // (barriers follow)
    Tile t = dealt_tile;
    const Bounds lim = bounds_of<BM, SH>(t);  // (of all of the tile's rows: the waves clean V together)
    if constexpr (SH) narrow<BN>(t, lim);
    Ld ld;
    ld.set(t);
    auto stage = [&](int i) -> LB* {
      const int S = i & 3;
      return S == 0 ? (LB*)s0 : S == 1 ? (LB*)s1 : S == 2 ? (LB*)s2 : (LB*)s3;
    };
    // Where 32 blocks lie: lane i holds the place of half i. (A scalar look-up a
    // step would make every read of the LDS behind it wait.)
    uint32_t lo = 0, hi = 0, bytes = 0;
    int id = ld.page_id(t.b0, t.b1);
    bool hole = false;          // slots without a page have been met: every block is looked at from then on
    auto window = [&](int j) {  // of blocks j .. j + 31, and the next one's pages on their way
      hole |= ld.spread(j, t.b1, id, lo, hi, bytes);
      id = ld.page_id(j + 32, t.b1);
    };
    Place pk[2] = {}, pv[2];  // K of block j, V of j - 1
    auto look = [&](int j) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = 2 * ((j - t.b0) & 31) + e;
        pv[e] = pk[e];
        pk[e] = Place{(uint32_t)__builtin_amdgcn_readlane((int)lo, at), (uint32_t)__builtin_amdgcn_readlane((int)hi, at),
                      (uint32_t)__builtin_amdgcn_readlane((int)bytes, at)};
      }
    };
    auto issue = [&](LB* st) {
      ld.issue(a.k, st, pk, wv);
      ld.issue(a.v, st + 32 * RB, pv, wv);
    };
    const int m = t.rt * BM + wv * 32 + l32, mc = m < t.M ? m : t.M - 1, tok = mc / t.group;
    u32x4 qf[NQ];
    load_query<T, NQ>(t, mc, qf);
    window(t.b0);
    look(t.b0);
    ld.issue(a.k, (LB*)s0, pk, wv);
    look(t.b0 + 1);
    issue((LB*)s1);
    // (the first wait leaves the loads behind here in flight, the next one the
    // last stage's)
    __builtin_amdgcn_sched_barrier(LDS_ORDER);
    look(t.b0 + 2);
    issue((LB*)s2);
    __builtin_amdgcn_sched_barrier(LDS_ORDER);
    look(t.b0 + 3);
    issue((LB*)s3);
    Row me = row_of<SH>(t, tok);
    if constexpr (SH) me.slope2 = a.slopes ? a.slopes[t.head * t.group + (mc - tok * t.group)] * LOG2E : 0.f;
    // whether a row of the tile may not see a slot of block b
    auto partly = [&](int b) { return (b + 1) * BN > lim.safe || (SH && b * BN < lim.low); };
    const f32x16 zero = {0.f};
    f32x16 o[NDT], s[2];  // scores of two blocks, in turn
#pragma unroll
    for (int i = 0; i < NDT; ++i) o[i] = zero;
    float mx = -INFINITY, l = 0.f, ref = 0.f, bm = 0.f;
    // fragments: K's of 16 of the head dim and 32 keys; V's, transposed, of 16
    // keys and 32 of the head dim
    u32x4 kf[4], vf[2][NDT], p[2];
    const int kx = (h ^ swz<RB, 16>(l32)) * 16, kr = l32 * RB;
    const int vr = (4 * h + (il >> 2)) * RB + 8 * (il & 1);
    const int vx = ((2 * ((lane >> 4) & 1) + ((il & 3) >> 1)) ^ swz<RB, 16>(4 * h + (il >> 2))) * 16;
    auto read_k = [&](const LB* st, int i) { kf[i & 3] = *(const LDS_AS u32x4*)(st + kr + turned<RB, 16>(kx, i * 32)); };
    auto read_v = [&](const LB* st, int kk, int dt) {
      auto tr = [&](int k0) {
        const LB* q = st + 32 * RB + vr + turned<RB, 16>(vx ^ (swz<RB, 16>(k0) * 16), dt * 64) + k0 * RB;
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)q));
      };
      const u32x2 u0 = tr(16 * kk), u1 = tr(16 * kk + 8);
      vf[kk][dt] = u32x4{u0.x, u0.y, u1.x, u1.y};
    };
    auto fence = [&] { __builtin_amdgcn_sched_barrier(0); };
    auto seen = [&](int kb) {
      const uint32_t see = seen_bits<SH>(t, kb, me);
      return hole ? see & ld.paged(kb) : see;
    };
    auto top = [&](float x, float y) { return CURVED ? fminf(x, y) : fmaxf(x, y); };
    auto cover = [&](f32x16& x, uint32_t see) {  // scores that their rows do not see
      hide(x, see, CURVED ? INFINITY : -INFINITY);
      bm = x[0];
#pragma unroll
      for (int j = 1; j < 16; ++j) bm = top(bm, x[j]);
    };
    auto bend = [&](float x) { return __builtin_amdgcn_rcpf(ex2(x * a.k1) + 1.f); };
    // (as soften())
    auto raise = [&] {
      bm = max_x32(bm) * (SH ? 1.f : a.c2);
      if (__any(bm > mx + 8.f)) {
        const float mn = fmaxf(mx, bm);
        const float f = mn == -INFINITY ? 1.f : ex2(mx - mn);
        mx = mn;
        l *= f;
#pragma unroll
        for (int i = 0; i < NDT; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[i][j] *= f;
      }
      ref = mx == -INFINITY ? 0.f : mx;
    };
    // probabilities j0 .. j1 - 1 of the lane's 16, rounded once for the products
    auto soft = [&](f32x16& cur, int j0, int j1) {
#pragma unroll
      for (int j = j0; j < j1; ++j) {
        cur[j] = ex2(CURVED ? __builtin_fmaf(cur[j], -2.f * a.cap2, a.cap2 - ref)
                            : SH ? cur[j] - ref : __builtin_fmaf(cur[j], a.c2, -ref));
        l += cur[j];
        if (j & 1) p[j >> 3][(j >> 1) & 3] = bf2(cur[j - 1], cur[j]);
        asm volatile("" : "+v"(l));  // (here, not behind the step's branches)
      }
    };
    // Step b, P = (b - b0) % 4: scores of block b + 1 (behind the last block,
    // of zeros), probabilities and products of block b.
    auto step = [&](auto phase, int b) {
      constexpr int P = decltype(phase)::value, JQ = 12;
      const LB *st = stage(P + 1), *sn = stage(P + 2);
      f32x16 &cur = s[P & 1], &nxt = s[(P + 1) & 1];
      const bool hidden = partly(b + 1) || hole;
      const uint32_t see = hidden ? seen((b + 1) * BN) : 0u;  // (its loads are out early)
      if (partly(b) || hole) {
        if (clean_values<T, HDP, 4>((LB*)st + 32 * RB, wv)) sOdd = 1;
        wait_lds();
        barrier();
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        if (i == UP && PAIR) raise();
        nxt = mma(kf[i & 3], qf[i], i ? nxt : zero, T());
        if (i + 4 < NQ) read_k(st, i + 4);
        else
#pragma unroll
          for (int dt = NDT * (i - NQ + 4) / 4; dt < NDT * (i - NQ + 5) / 4; ++dt) read_v(st, 0, dt);
        if (i == 2) look(b + 4);
        if (i >= UP) soft(cur, (i - UP) * JQ / (NQ - UP), (i + 1 - UP) * JQ / (NQ - UP));
        fence();
      }
      wait_vm<LW>();  // stage b + 1 is here, b + 2 may be on its way,
      meet();         // and stage b - 1 is worked off
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        o[dt] = mma(vf[0][dt], p[0], o[dt], T());
        read_v(st, 1, dt);
        soft(cur, JQ + dt * (16 - JQ) / NDT, JQ + (dt + 1) * (16 - JQ) / NDT);
        if (dt == 0) ld.issue(a.k, stage(P), pk, wv);
        if (dt == 1) ld.issue(a.v, stage(P) + 32 * RB, pv, wv);
        if constexpr (CURVED) {
#pragma unroll
          for (int j = 8 * dt / NDT; j < 8 * (dt + 1) / NDT; ++j) nxt[j] = bend(nxt[j]);
        }
        fence();
      }
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        o[dt] = mma(vf[1][dt], p[1], o[dt], T());
#pragma unroll
        for (int i = 4 * dt / NDT; i < 4 * (dt + 1) / NDT; ++i) read_k(sn, i);
#pragma unroll
        for (int j = 16 * dt / NDT; j < 16 * (dt + 1) / NDT && (!SH || CURVED); ++j) {
          if (CURVED && j >= 8) nxt[j] = bend(nxt[j]);
          bm = j ? top(bm, nxt[j]) : nxt[0];
        }
        asm volatile("" : "+v"(bm));
        fence();
      }
      if constexpr (SH && !CURVED) {
        shape<T>(nxt, a, t, (b + 1) * BN, me);
        bm = nxt[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) bm = fmaxf(bm, nxt[j]);
      }
      if (hidden) cover(nxt, see);
      if constexpr (CURVED) bm = __builtin_fmaf(-2.f * a.cap2, bm, a.cap2);
      if (!PAIR && b + 1 < t.b1) raise();
    };
    // the first block's scores
    wait_vm<2 * LW>();
    barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i) read_k((LB*)s0, i);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      s[0] = mma(kf[i & 3], qf[i], i ? s[0] : zero, T());
      if (i + 4 < NQ) read_k((LB*)s0, i + 4);
      fence();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) read_k((LB*)s1, i);
    if constexpr (CURVED) {
#pragma unroll
      for (int j = 0; j < 16; ++j) s[0][j] = bend(s[0][j]);
    } else if constexpr (SH) {
      shape<T>(s[0], a, t, t.b0 * BN, me);
    }
    bm = s[0][0];
#pragma unroll
    for (int j = 1; j < 16; ++j) bm = top(bm, s[0][j]);
    if (partly(t.b0) || hole) cover(s[0], seen(t.b0 * BN));
    if constexpr (CURVED) bm = __builtin_fmaf(-2.f * a.cap2, bm, a.cap2);
    if (!PAIR) raise();
    for (int b = t.b0;; b += 4) {
      if (((b - t.b0) & 31) == 28) window(b + 4);
      step(std::integral_constant<int, 0>(), b);
      if (b + 1 >= t.b1) break;
      step(std::integral_constant<int, 1>(), b + 1);
      if (b + 2 >= t.b1) break;
      step(std::integral_constant<int, 2>(), b + 2);
      if (b + 3 >= t.b1) break;
      step(std::integral_constant<int, 3>(), b + 3);
      if (b + 4 >= t.b1) break;
    }
    wait_vm<0>();  // (loads of blocks behind the last, which bring zeros)
    l = sum_x32(l);
    if (sOdd)  // (written before the last step's barrier)
      for (int b = t.b0; b < t.b1; ++b)
        if (partly(b) || hole) add_odd_values<T, HDP>(t, b * BN, seen_bits<SH>(t, b * BN, me), o);
    finish<T, HDP, SH>(t, slot, wv, m, mx, l, o);
  });
}

// Many rows to a sequence in fp32: tiles of 128 rows, 32 to a wave, bound by
// the matrix cores. The four waves share a ring of two blocks in the LDS, the
// next one on its way while one is worked on: one barrier to a block. A block
// is two tiles of 32 keys, at head dim 128 one, so that there are more blocks
// to deal out: eight caches of 1,000 slots, 8 heads on 1, trees of 40 rows 35.0
// us against 40.6, of 64 39.0 against 41.6; two chunks of 1,000 rows behind
// 2,000, 32 heads on 8, 750 us against 704.
template <int HDP, bool SH>
__global__ __launch_bounds__(256, (many_waves<float, HDP>())) void k_tree_many32(Args a) {
  typedef float T;
  constexpr int BM = 128, BN = HDP <= 64 ? 64 : 32, NS = BN / 32;
  constexpr int RB = HDP * (int)sizeof(T), NQ = RB / 32, NDT = HDP / 32;
  typedef Loader<T, HDP, 4, 8> Ld;
  __shared__ __attribute__((aligned(1024))) unsigned char sK0[NS * 32 * RB], sK1[NS * 32 * RB];
  __shared__ __attribute__((aligned(1024))) unsigned char sV0[NS * 32 * RB], sV1[NS * 32 * RB];
  __shared__ int sOdd;
  for_tiles<BM, BN, 1, SH>(a.wgs, [&](const Tile& dealt_tile, int slot) {
    const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6), l32 = lane & 31, h = lane >> 5;
    if (tid == 0) sOdd = 0;  // (a barrier of the first block follows)
    Tile t = dealt_tile;
    const Bounds lim = bounds_of<BM, SH>(t);  // (of all of the tile's rows: the waves clean V together)
    if constexpr (SH) narrow<BN>(t, lim);
    Ld ld;
    ld.set(t);
    Place at[NS][2];
    bool hole = false;  // (as in k_tree_many)
    auto look = [&](int b) {
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        ld.look(b * BN + 32 * n, at[n]);
        hole |= ld.hole(b * BN + 32 * n, at[n]);
      }
    };
    auto issue = [&](const char* src, LB* dst) {
#pragma unroll
      for (int n = 0; n < NS; ++n) ld.issue(src, dst + n * 32 * RB, at[n], wv);
    };
    const int m = t.rt * BM + wv * 32 + l32, mc = m < t.M ? m : t.M - 1, tok = mc / t.group;
    u32x4 qf[NQ];
    load_query<T, NQ>(t, mc, qf);
    look(t.b0);
    issue(a.k, (LB*)sK0);
    issue(a.v, (LB*)sV0);
    Row me = row_of<SH>(t, tok);
    if constexpr (SH) me.slope2 = a.slopes ? a.slopes[t.head * t.group + (mc - tok * t.group)] * LOG2E : 0.f;
    // whether a row of the tile may not see one of `n` slots from kb on
    auto partly = [&](int kb, int n) { return kb + n > lim.safe || (SH && kb < lim.low); };
    f32x16 o[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float mx = -INFINITY, l = 0.f;
    look(t.b0 + 1);
    auto step = [&](auto stage, int b) {
      // (by name: the compiler lets reads of one stage run beside loads into
      // the other only where it can tell them apart)
      constexpr int S = decltype(stage)::value;
      LB *kt = S ? (LB*)sK1 : (LB*)sK0, *vt = S ? (LB*)sV1 : (LB*)sV0;
      LB *kn = S ? (LB*)sK0 : (LB*)sK1, *vn = S ? (LB*)sV0 : (LB*)sV1;
      wait_vm<0>();  // this wave's part of the block is here,
      barrier();     // so are the others', and the other block is worked off
      if (b + 1 < t.b1) issue(a.k, kn);
      const int kb = b * BN;
      f32x16 s[NS];
      scores<T, HDP, NS, NQ>(kt, qf, s);
      // (loads take their turns at issue: these go out beside the products)
      if (b + 1 < t.b1) issue(a.v, vn);
      if constexpr (SH) {
#pragma unroll
        for (int n = 0; n < NS; ++n) shape<T>(s[n], a, t, kb + 32 * n, me);
      }
      if (partly(kb, BN) || hole) {
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          uint32_t see = seen_bits<SH>(t, kb + 32 * n, me);
          if (hole) see &= ld.paged(kb + 32 * n);
          hide(s[n], see);
          if (clean_values<T, HDP, 4>(vt + n * 32 * RB, wv)) sOdd = 1;
        }
        wait_lds();
        barrier();
      }
      Values<T, HDP, NS> vv;
      vv.first(vt);
      look(b + 2);
      soften<NDT, NS>(s, SH ? 1.f : a.c2, mx, l, o);
      vv.add(s, {}, o);
    };
    for (int b = t.b0; b < t.b1; b += 2) {
      step(std::integral_constant<int, 0>(), b);
      if (b + 1 < t.b1) step(std::integral_constant<int, 1>(), b + 1);
    }
    l = sum_x32(l);
    if (sOdd)  // (written before the last block's barrier)
      for (int kb = t.b0 * BN; kb < t.b1 * BN; kb += 32)
        if (partly(kb, 32) || hole) add_odd_values<T, HDP>(t, kb, seen_bits<SH>(t, kb, me), o);
    finish<T, HDP, SH>(t, slot, wv, m, mx, l, o);
  });
}

// The join: tiles whose keys several workgroups shared out, from their parts
// (part 0 in the last slot of its run, the others in the first slots of the
// runs behind it). How many tiles there are only the descriptors tell, so a
// fixed number of workgroups (a launch pays for every one) reads them all,
// lists the work in the LDS and goes through it in turn. With up to four parts
// each wave does a piece of its own, all parts in flight; with more, the four
// waves take every fourth part of one piece, four at a time, so that sixteen
// parts cost one round trip, and their sums meet in the LDS in wave order.
// Bound by its round trips (3.9 us for four parts of eight rows), with many
// rows by what the parts hold (27 MB in 9.6 us, 81 MB in 20).
constexpr int JOIN_MOST = 1024;  // runs
__device__ __forceinline__ size_t part_slot(int w, int i) { return (size_t)(2ll * (w + i) + (i == 0 ? 1 : 0)); }

// One batch of four parts with maxima m and sums l, values v: into top, den, o.
template <typename V, int N>
__device__ __forceinline__ void join_parts(const float (&m)[4], const float (&l)[4], const V (&v)[4][N], float& top,
                                           float& den, V (&o)[N]) {
  const float mt = fmaxf(top, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
  const float back = top == -INFINITY ? 0.f : ex2(top - mt);
  den *= back;
#pragma unroll
  for (int t = 0; t < N; ++t) o[t] *= back;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = m[i] == -INFINITY ? 0.f : ex2(m[i] - mt);
    den = __builtin_fmaf(f, l[i], den);
#pragma unroll
    for (int t = 0; t < N; ++t) o[t] += f * v[i][t];
  }
  top = mt;
}

// BM = 32: parts are row-major; a piece is one row, a lane HDP / 64 columns of
// it. BM = 128: parts lie in the order in which the waves hold them; a piece
// is 32 columns of 32 rows, a lane four of every eight columns of its row.
template <typename T, int HDP, int BM, bool SH>
__global__ __launch_bounds__(256) void k_tree_join(Args a) {
  constexpr bool MANY = BM == 128;
  constexpr int C = MANY ? 4 : HDP / 64, N = MANY ? 4 : 1, NDT = HDP / 32;
  typedef float fc __attribute__((ext_vector_type(C)));
  __shared__ int sPre[JOIN_MOST + 1];
  __shared__ int sWave[4];
  __shared__ fc sO[4][N][64];
  __shared__ float sT[4][64], sD[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, l32 = lane & 31, h = lane >> 5, hd = a.c.hd;
  // pieces of a tile that workgroups take at once: one, or four of few parts
  auto takes = [&](const int4& d, const int4& e) {
    if (d.x == 0) return 0;
    const int rows = e.x - d.w * BM < BM ? e.x - d.w * BM : BM;
    const int pieces = MANY ? (rows + 31) / 32 * ((hd + 31) / 32) : rows;
    return d.x <= 4 ? (pieces + 3) / 4 : pieces;
  };
  int before = 0;
  for (int c0 = 0; c0 < a.wgs; c0 += 256) {
    const int w = c0 + tid;
    const int cnt = w < a.wgs ? takes(a.desc[2 * w], a.desc[2 * w + 1]) : 0;
    const int incl = wave_scan(cnt);
    if (lane == 63) sWave[wv] = incl;
    __syncthreads();
    int off = before;
#pragma unroll
    for (int k = 0; k < 4; ++k) off += k < wv ? sWave[k] : 0, before += sWave[k];
    if (w < a.wgs) sPre[w + 1] = off + incl;
    __syncthreads();
  }
  if (tid == 0) sPre[0] = 0;
  __syncthreads();
  const float* pm = a.part + 2ll * a.wgs * BM * HDP;
  // what workgroups of this XCD wrote
  const int xcd = blockIdx.x & 7, last = sPre[(xcd + 1) * (a.wgs >> 3)];
  for (int take = sPre[xcd * (a.wgs >> 3)] + (blockIdx.x >> 3); take < last; take += gridDim.x >> 3) {
    int lo = 0, hi = a.wgs - 1;  // the descriptor of its tile
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (sPre[mid] <= take) lo = mid;
      else hi = mid - 1;
    }
    const int k = uni(lo);
    const int4 d = a.desc[2 * k], e = a.desc[2 * k + 1];
    const int n = d.x, M = e.x, group = e.y, w = e.z, m0 = d.w * BM;
    const bool own = n <= 4;  // a piece to each wave
    const int piece = own ? (take - sPre[k]) * 4 + wv : take - sPre[k];
    const int nd = (hd + 31) / 32, rg = MANY ? piece / nd : 0, dt = MANY ? piece % nd : 0;
    const int lm = MANY ? rg * 32 + l32 : piece;  // the lane's row of the tile
    // (rows behind the last have nothing written: theirs is not used)
    const bool live = MANY ? m0 + rg * 32 < M : m0 + lm < M;
    const int lr = live ? lm : 0;
    const float* po = a.part + (MANY ? (live ? rg : 0) * 32 * HDP + (dt * 256 + lane) * 4 : lr * HDP + lane * C);
    float top = -INFINITY, den = 0.f;
    fc o[N];
#pragma unroll
    for (int t = 0; t < N; ++t) o[t] = (fc)0.f;
    const int by = own ? 1 : 4;
    for (int i0 = own ? 0 : wv; i0 < n; i0 += 16) {
      float m[4], l[4];
      fc v[4][N];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = i0 + by * i < n;
        const size_t s = part_slot(w, in ? i0 + by * i : i0) * BM;
        const f32x2 ml = *(const f32x2*)(pm + (s + lr) * 2);
        m[i] = in ? ml.x : -INFINITY;
        l[i] = in ? ml.y : 0.f;
#pragma unroll
        for (int t = 0; t < N; ++t) {
          const fc y = *(const fc*)(po + s * HDP + t * 256);
          v[i][t] = in ? y : (fc)0.f;
        }
      }
      join_parts(m, l, v, top, den, o);
    }
    auto put = [&](const fc& x, float inv, int col) {
      const int mm = m0 + lm, tk = mm / group;
      if (mm >= M || col >= hd) return;
      T* dst = (T*)a.out + (size_t)(d.y + tk) * (size_t)a.ldo + (size_t)(d.z + mm - tk * group) * hd + col;
      float r[C];
#pragma unroll
      for (int t = 0; t < C; ++t) r[t] = x[t] * inv;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int t = 0; t < C; ++t) dst[t] = r[t];
      } else if constexpr (C == 1) {
        dst[0] = (T)bf2(r[0], 0.f);
      } else {
        uint32_t u[C / 2];
#pragma unroll
        for (int t = 0; t < C / 2; ++t) u[t] = bf2(r[2 * t], r[2 * t + 1]);
        __builtin_memcpy(__builtin_assume_aligned(dst, 2 * C), u, 2 * C);
      }
    };
    // (a lane of a row's first columns writes its log-sum-exp)
    auto put_sum = [&](float mx, float l) {
      if constexpr (SH) {
        const int mm = m0 + lm, tk = mm / group;
        if (a.lse && mm < M && (MANY ? dt == 0 && h == 0 : lane == 0))
          a.lse[(size_t)(d.y + tk) * a.nq + d.z + (mm - tk * group)] = log_sum(mx, l);
      }
    };
    if (own) {
      const float inv = inverse(den);
      if (live) put_sum(top, den);
      if (live) {
#pragma unroll
        for (int t = 0; t < N; ++t) put(o[t], inv, MANY ? 32 * dt + 8 * t + 4 * h : lane * C);
      }
      continue;
    }
#pragma unroll
    for (int t = 0; t < N; ++t) sO[wv][t][lane] = o[t];
    sT[wv][lane] = top;
    sD[wv][lane] = den;
    __syncthreads();
    if (live && wv < N) {  // (BM = 128: a wave to the columns 8 wv .. + 7)
      float m4[4], l4[4], t1 = -INFINITY, d1 = 0.f;
      fc v4[4][1], o1[1] = {(fc)0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) m4[k] = sT[k][lane], l4[k] = sD[k][lane], v4[k][0] = sO[k][wv][lane];
      join_parts(m4, l4, v4, t1, d1, o1);
      put(o1[0], inverse(d1), MANY ? 32 * dt + 8 * wv + 4 * h : lane * C);
      if (wv == 0) put_sum(t1, d1);
    }
    __syncthreads();
  }
}

// Head dims between the templates run as the next one, whose products and sums
// they pay for: eight prompts of 500 rows, 32 heads on 8, 51 us at 32 and 61 at
// 64, 69 at 96 and 84 at 128; 40 heads on 8, 131 us at 160 and 166 at 256.
inline int pad_hd(int dtype, int hd) { return hd <= 64 ? 64 : hd <= 128 ? 128 : 256; }

// Many rows to a sequence (on average more than 128, at head dims up to 64 more
// than 192, in fp32 more than 256): tiles of 128 rows, whose waves share K and
// V. Below that the two are close (at head dim 256 64 rows 22.3 us in tiles of
// 32, 19.8 in tiles of 128), and tiles of 32 keep more of the probabilities.
// Trees over 8 query heads on one KV head, 160, 192 and 256 rows in tiles of
// 32 / 128: eight caches of 4,000 slots at head dim 128 22.8 / 21.3, 25.5 / 21.7
// and 27.7 / 23.0 us, at 64 18.1 / 19.8, 20.0 / 19.9 and 21.5 / 20.3; two of
// 30,000 at 128 36.7 / 34.1, 38.5 / 33.8 and 41.6 / 34.1; eight of 2,000 at 256
// 25.1 / 25.0, 27.0 / 25.3 and 28.3 / 27.6. In fp32, eight of 1,000 at 128, 192,
// 256 and 320 rows: 24.8 / 27.3, 30.6 / 29.8, 36.9 / 34.0; four of 4,000 34.9 /
// 42.1, 39.3 / 43.0, 44.6 / 50.3.
// All of those are even batches. The lengths are on the device, so the average
// counts padding and knows nothing of mixed batches, which pay for it: a prompt
// of 2,000 rows, 32 heads on 8 of 128, 93 us on its own and 197 beside 127
// entries of padding; beside 60 single tokens behind 700 slots 131 us, and 203
// with 67 entries of padding as well.
inline int tile_rows(const TreeAttnDesc& d) {
  const long long rows = (long long)d.r.n_rows * (d.nq / d.c.nkv);
  const long long many = d.c.dtype == DT_F32 ? 256 : d.c.hd <= 64 ? 192 : 128;
  return rows > many * d.r.n_ent ? 128 : 32;
}
// Workgroups, each with a run of blocks: as many as the CUs hold.
inline int tree_wgs(const TreeAttnDesc& d) {
  const int esz = d.c.dtype == DT_BF16 ? 2 : 4;
  const int per = pad_hd(d.c.dtype, d.c.hd) * esz <= 256 ? 2 : 1;
  return std::min(std::max(8, d.cus / 8 * 8) * per, JOIN_MOST);
}

template <typename T, int HDP, bool SH>
hipError_t run(const TreeAttnDesc& d, const Args& a, hipStream_t st) {
  const int rows = tile_rows(d);
  if (rows == 32) hipLaunchKernelGGL((k_tree_few<T, HDP, SH>), dim3(a.wgs), dim3(256), 0, st, a);
  else if constexpr (sizeof(T) == 2) {
    if (SH && a.cap2 > 0.f && a.cap2 < CAP_LARGE && !a.slopes) hipLaunchKernelGGL((k_tree_many<HDP, SH, SH>), dim3(a.wgs), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_tree_many<HDP, SH, false>), dim3(a.wgs), dim3(256), 0, st, a);
  }
  else hipLaunchKernelGGL((k_tree_many32<HDP, SH>), dim3(a.wgs), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (at most as many as there can be pieces to take)
  const long long tiles = ((long long)d.r.n_rows * a.group / rows + d.r.n_ent) * d.c.nkv;
  const int joins = (int)std::min({(long long)4 * d.cus / 8, 128ll, (tiles * (rows == 32 ? 32 : HDP / 8) + 7) / 8}) * 8;
  if (rows == 32) hipLaunchKernelGGL((k_tree_join<T, HDP, 32, SH>), dim3(joins), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_tree_join<T, HDP, 128, SH>), dim3(joins), dim3(256), 0, st, a);
  return hipGetLastError();
}

// The scores' part of the arguments.
inline void shape_args(const ScoreDesc& x, Args* a) {
  a->cap2 = x.cap * LOG2E;
  a->k1 = x.cap > 0.f ? 2.f * x.scale * LOG2E / x.cap : 0.f;
  a->slopes = x.slopes;
  a->depth = x.depth;
  a->span = (const int2*)x.span;
  a->window = x.window;
}

template <bool SH>
hipError_t launch(const TreeAttnDesc& d, hipStream_t st) {
  if (d.r.n_rows <= 0 || d.r.n_ent <= 0) return hipSuccess;
  Args a{};
  a.c = d.c;
  a.r = d.r;
  a.nq = d.nq;
  a.group = d.nq / d.c.nkv;
  a.q = d.q;
  a.out = d.out;
  a.ldq = d.ldq;
  a.ldo = d.ldo;
  a.mask = d.mask;
  a.mask_words = d.mask_words;
  a.c2 = d.s.scale * LOG2E;
  if constexpr (SH) {
    shape_args(d.s, &a);
    a.lse = d.lse;
  }
  const size_t layer = (size_t)d.layer * d.c.n_pages * d.c.nkv * d.c.page * d.c.hd * (d.c.dtype == DT_BF16 ? 2 : 4);
  a.k = (const char*)d.c.k + layer;
  a.v = (const char*)d.c.v + layer;
  a.wgs = tree_wgs(d);
  a.desc = (int4*)d.scratch;
  a.part = (float*)((char*)d.scratch + (size_t)a.wgs * 32);
  const int hdp = pad_hd(d.c.dtype, d.c.hd);
  if (d.c.dtype == DT_BF16)
    return hdp == 64 ? run<uint16_t, 64, SH>(d, a, st) : hdp == 128 ? run<uint16_t, 128, SH>(d, a, st)
                                                                    : run<uint16_t, 256, SH>(d, a, st);
  if (hdp > 128) return hipErrorInvalidValue;
  return hdp == 64 ? run<float, 64, SH>(d, a, st) : run<float, 128, SH>(d, a, st);
}

}  // namespace
}  // namespace vla
