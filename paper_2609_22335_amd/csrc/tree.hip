// Attention of drafted tokens over a paged KV cache: every row attends to all
// committed slots of its sequence and to the drafts that its mask names (or,
// without a mask, to the drafts up to itself).
//
// The rows of one sequence and KV head (tokens x query heads of the group)
// form tiles that share K and V. Scores are computed transposed (S^T = K Q^T),
// so that a lane holds one query: the running maximum and sum are one value a
// lane, and the probabilities are, without leaving their registers, the right
// operand of O^T += V^T P^T.
#include <algorithm>

#include "paged_dev.h"

namespace vla {
using namespace pg;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
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
  const char* k;  // the layer's K and V
  const char* v;
  float* part;   // [2 W][rows][hd], then [2 W][rows][2]
  int4* desc;    // [W]
  int wgs;       // W
  int min_quota;
};

// Tiles of an entry: BM rows by blocks of BN keys.
template <int BM, int BN>
struct Geo {
  int tiles, nb_all;  // row tiles of a head; blocks of a tile with every key
  int end, len, M, group;
  bool causal;
  __device__ __forceinline__ void set(const Args& a, const Entry& x) {
    group = a.group;
    M = x.n * group;
    tiles = (M + BM - 1) / BM;
    len = x.len;
    const long long e = (long long)x.len + x.n;
    end = e < x.cap ? (int)e : x.cap;
    causal = a.mask == nullptr;
    nb_all = blocks(end);
  }
  // (a tile without keys has one block, which writes its zeros)
  static __device__ __forceinline__ int blocks(int keys) { return keys > 0 ? (keys + BN - 1) / BN : 1; }
  __device__ __forceinline__ int tile_end(int rt) const {
    if (!causal) return end;
    const int last = (rt + 1) * BM < M ? (rt + 1) * BM - 1 : M - 1;
    const int e = len + last / group + 1;
    return e < end ? e : end;
  }
  __device__ __forceinline__ int nb(int rt) const { return causal ? blocks(tile_end(rt)) : nb_all; }
  // blocks of one head's tiles
  __device__ __forceinline__ int sum() const {
    if (!causal || tiles == 0) return tiles * nb_all;
    int s = 0;
    for (int rt = 0; rt < tiles; ++rt) s += nb(rt);
    return s;
  }
};

// What every workgroup works out for itself: all entries' blocks in a row,
// dealt out in equal runs, so that uneven sequences load the chip evenly.
// Lanes hold 64 entries at a time.
template <int BM, int BN>
struct Deal {
  long long total = 0;
  int chunk0 = 0;          // first entry of the lanes' chunk
  long long base = 0;      // blocks before the chunk
  long long incl = 0;      // inclusive prefix of the lane's entry in it
  long long units = 0;     // the lane's entry's blocks
  int persum = 0;          // of one head
  Entry x;

  __device__ __forceinline__ void load(const Args& a, int c0) {
    const int e = c0 + (threadIdx.x & 63);
    units = 0;
    persum = 0;
    x = Entry{-1, 0, 0, 0, 0};
    if (e < a.r.n_ent) {
      x = entry_of(a.c, a.r, e);
      Geo<BM, BN> g;
      g.set(a, x);
      persum = g.sum();
      units = (long long)persum * a.c.nkv;
    }
    incl = units;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const long long y = __shfl_up(incl, m);
      if ((threadIdx.x & 63) >= m) incl += y;
    }
    chunk0 = c0;
  }
  // lane i's value in every lane, in scalar registers
  static __device__ __forceinline__ long long lane_of(long long v, int i) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, i);
    const int hi = __builtin_amdgcn_readlane((int)(v >> 32), i);
    return (long long)(((unsigned long long)(uint32_t)hi << 32) | lo);
  }
  __device__ __forceinline__ void init(const Args& a) {
    total = 0;
    for (int c0 = 0; c0 < a.r.n_ent; c0 += 64) {
      load(a, c0);
      total += lane_of(incl, 63);
    }
    if (a.r.n_ent > 64) load(a, 0);
    base = 0;
  }
  // The entry that holds unit u (chunks are only walked forward).
  __device__ __forceinline__ int locate(const Args& a, long long u) {
    long long all = lane_of(incl, 63);
    while (u >= base + all) {
      base += all;
      load(a, chunk0 + 64);
      all = lane_of(incl, 63);
    }
    return __ffsll(__ballot(base + incl > u)) - 1;
  }
};

// 16-byte chunk c of row r sits at position c ^ swz(r): rows that a fragment
// read takes together start in different banks.
template <typename T, int HDP>
__device__ __forceinline__ constexpr int swz(int r) {
  constexpr int RB = HDP * (int)sizeof(T);  // bytes of a row
  if (sizeof(T) == 4) return RB >= 256 ? (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1) : 0;
  if (RB >= 256) return ((r & 3) << 2) | ((r >> 2) & 3);
  return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

__device__ __forceinline__ f32x16 mma(uint4 a, uint4 b, f32x16 c, uint16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ f32x16 mma(uint4 a, uint4 b, f32x16 c, float) {
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

// RW row groups of 32 rows and KW = 4 / RW key groups of 32 keys to the four
// waves: RW = 1 for few rows (each wave streams its own keys, the waves'
// results are merged at the end), RW = 4 for many.
template <typename T, int HDP, int RW>
__global__ __launch_bounds__(256, 1) void k_tree(Args a) {
  constexpr int KW = 4 / RW, BM = 32 * RW, BN = 32 * KW;
  constexpr int ESZ = sizeof(T), RB = HDP * ESZ, CPR = RB / 16;  // row bytes, chunks
  constexpr int RPI = 1024 / RB;                                 // rows of a load
  constexpr int NI = 32 / RPI, NIW = NI / RW;                    // loads of a key group's tile, a wave's
  constexpr int NQ = RB / 32, NDT = HDP / 32;
  constexpr bool HALF = ESZ == 2;
  static_assert(NIW >= 1 && 2 * NIW < 60, "loads in flight");
  __shared__ __attribute__((aligned(1024))) unsigned char sK[KW][32 * RB];
  __shared__ __attribute__((aligned(1024))) unsigned char sV[KW][32 * RB];
  __shared__ float sM[4][32], sL[4][32];

  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = RW == 1 ? wv : 0, rw = RW == 1 ? 0 : wv;
  const int l32 = lane & 31, h = lane >> 5;
  const int hd = a.c.hd;
  // consecutive runs of blocks on one XCD (workgroups go round the eight)
  const int w = (int)(blockIdx.x & 7) * (a.wgs >> 3) + (int)(blockIdx.x >> 3);

  Deal<BM, BN> deal;
  deal.init(a);
  long long quota = (deal.total + a.wgs - 1) / a.wgs;
  if (quota < a.min_quota) quota = a.min_quota;
  long long u = w * quota;
  const long long u_end = u + quota < deal.total ? u + quota : deal.total;
  int4 desc = make_int4(0, 0, 0, 0);

  // the lane's part of a load: row and 16-byte chunk
  const int lrow = lane / CPR, lpos = lane % CPR;
  const int lchunk = lpos ^ swz<T, HDP>(lrow);

  while (u < u_end) {
    const int el = deal.locate(a, u);
    Entry x;
    x.seq = __builtin_amdgcn_readlane(deal.x.seq, el);
    x.row0 = __builtin_amdgcn_readlane(deal.x.row0, el);
    x.n = __builtin_amdgcn_readlane(deal.x.n, el);
    x.len = __builtin_amdgcn_readlane(deal.x.len, el);
    x.cap = __builtin_amdgcn_readlane(deal.x.cap, el);
    const int persum = __builtin_amdgcn_readlane(deal.persum, el);
    Geo<BM, BN> g;
    g.set(a, x);
    const long long first = deal.base + deal.lane_of(deal.incl, el) - deal.lane_of(deal.units, el);
    const int head = (int)((u - first) / persum);
    int rem = (int)(u - first - (long long)head * persum);
    int rt = 0;
    if (g.causal) {
      while (rem >= g.nb(rt)) rem -= g.nb(rt), ++rt;
    } else {
      rt = rem / g.nb_all;
      rem -= rt * g.nb_all;
    }
    const int nb = g.nb(rt), b0 = rem;
    const int b1 = (int)(nb - b0 < u_end - u ? nb : b0 + (u_end - u));
    const int kend = g.tile_end(rt);

    // this lane's query
    const int m = rt * BM + rw * 32 + l32;
    const bool mine = m < g.M;
    const int mc = mine ? m : g.M - 1;
    const int tok = mc / g.group, row = x.row0 + tok;
    uint4 qf[NQ];
    {
      const T* qp = (const T*)a.q + (size_t)row * (size_t)a.ldq +
                    (size_t)(head * g.group + (mc - tok * g.group)) * hd;
#pragma unroll
      for (int s = 0; s < NQ; ++s) {
        const int d0 = (2 * s + h) * El<T>::VEC;
        qf[s] = d0 < hd ? *(const uint4*)(qp + d0) : make_uint4(0, 0, 0, 0);
      }
    }
    // slots below `own` are seen; the wave needs no mask below `safe`
    const int own = g.causal ? (x.len + tok + 1 < kend ? x.len + tok + 1 : kend) : kend;
    const int m0 = rt * BM + rw * 32;
    const int safe0 = g.causal ? x.len + (m0 < g.M ? m0 : g.M - 1) / g.group + 1 : x.len;
    const int safe = safe0 < kend ? safe0 : kend;

    const int32_t* table = a.c.table + (size_t)x.seq * a.c.max_pages;
    const size_t pbytes = (size_t)a.c.page * hd * ESZ;  // a page's part of one KV head
    // K or V of block b into the LDS. Loads reach at most one page's part of
    // one head, from its base; slots behind the last key and chunks behind the
    // head dim lie out of the resource's range and become zeros.
    auto issue = [&](const char* src, unsigned char* dst, int b) {
      const int kb = b * BN + kg * 32;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int s0 = kb + 16 * hh;
        const int pid = s0 < kend ? ((const __attribute__((address_space(4))) int32_t*)table)[s0 >> a.c.page_lg] : -1;
        const bool ok = (unsigned)pid < (unsigned)a.c.n_pages;
        const int at = s0 & (a.c.page - 1);
        int have = kend - (s0 - at);  // keys from the page's first slot on
        have = !ok || have < 0 ? 0 : have > a.c.page ? a.c.page : have;
        const Rsrc rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(src) + ((size_t)(ok ? pid : 0) * a.c.nkv + head) * pbytes, (short)0, have * hd * ESZ,
            0x00020000);
#pragma unroll
        for (int i = 0; i < NI / 2; ++i) {
          const int idx = hh * (NI / 2) + i;  // rows idx RPI .. + RPI - 1 of the tile
          if (RW > 1 && idx % RW != rw) continue;
          const int r0 = idx * RPI;
          const int ch = lchunk ^ swz<T, HDP>(r0);
          const uint32_t off = (uint32_t)((at + (r0 & 15) + lrow) * hd * ESZ + ch * 16);
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(dst + idx * 1024), 16,
                                                   HDP != hd && ch * 16 >= hd * ESZ ? OOB : off, 0, 0, 0);
        }
      }
    };

    f32x16 o[NDT];
#pragma unroll
    for (int i = 0; i < NDT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float mx = -INFINITY, l = 0.f;

    wait_vm<0>();  // stores of the last tile are out of the count
    barrier();     // and its use of the LDS is over
    issue(a.k, sK[kg], b0);
    issue(a.v, sV[kg], b0);
    for (int b = b0; b < b1; ++b) {
      const int kb = b * BN + kg * 32;
      const bool more = b + 1 < b1;
      wait_vm<NIW>();  // K is here, V may be on its way
      if (RW > 1) barrier();
      f32x16 s;
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const uint4 kf = *(const uint4*)(sK[kg] + l32 * RB + (((2 * t + h) ^ swz<T, HDP>(l32)) * 16));
        s = mma(kf, qf[t], s, T());
      }
      wait_lds();
      if (RW > 1) barrier();
      if (more) issue(a.k, sK[kg], b + 1);

      // masks: bit i of `see` is key kb + i for this lane's query
      const bool masked = kb + 32 > safe;
      uint32_t see = 0xFFFFFFFFu;
      if (masked) {
        const int n = own - kb;
        see = n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
        if (!g.causal && kb + 32 > x.len) {
          const int j0 = kb - x.len;  // draft of bit 0
          uint32_t bits;
          const uint32_t* mw = a.mask + (size_t)row * a.mask_words;
          if (j0 >= 0) {
            const int wi = j0 >> 5, sh = j0 & 31;
            const uint32_t lo = wi < a.mask_words ? mw[wi] : 0u, hi = wi + 1 < a.mask_words ? mw[wi + 1] : 0u;
            bits = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
          } else {
            bits = (mw[0] << -j0) | ((1u << -j0) - 1u);
          }
          see &= bits;
        }
        const uint32_t half = see >> (4 * h);
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = (half >> (8 * (j / 4) + j % 4)) & 1u ? s[j] : -INFINITY;
      }

      // running maximum and sum
      float bm = s[0];
#pragma unroll
      for (int j = 1; j < 16; ++j) bm = fmaxf(bm, s[j]);
      bm = max_x32(bm) * a.c2;
      // rescale only when a row's maximum has grown by 2^8 or more: sums of
      // probabilities up to 2^8 lose nothing
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
      for (int j = 0; j < 16; ++j) s[j] = ex2(__builtin_fmaf(s[j], a.c2, -ref));
      uint4 ph[2], pl[2];
      if constexpr (HALF) {
        // P as the sum of two bf16 values where the matrix cores wait for
        // memory anyway (few rows), else rounded once
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          uint32_t hw[4], lw[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p0 = s[8 * kk + 2 * i], p1 = s[8 * kk + 2 * i + 1];
            hw[i] = bf2(p0, p1);
            const float r0 = __uint_as_float(hw[i] << 16), r1 = __uint_as_float(hw[i] & 0xFFFF0000u);
            if (RW == 1) {
              lw[i] = bf2(p0 - r0, p1 - r1);
              l += p0 + p1;
            } else {
              l += r0 + r1;
            }
          }
          ph[kk] = make_uint4(hw[0], hw[1], hw[2], hw[3]);
          if (RW == 1) pl[kk] = make_uint4(lw[0], lw[1], lw[2], lw[3]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) l += s[j];
      }

      if (more) wait_vm<NIW>();  // V is here, the next K may be on its way
      else wait_vm<0>();
      if (RW > 1) barrier();
      const unsigned char* vt = sV[kg];
      // A masked key's V may hold anything, and 0 x inf is not 0: such a
      // block is added key by key.
      bool odd = false;
      if (masked) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint4 c4 = *(const uint4*)(vt + i * 1024 + lane * 16);
          const uint32_t wd[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            if (HALF) odd |= (wd[t] & 0x7F80u) == 0x7F80u || (wd[t] & 0x7F800000u) == 0x7F800000u;
            else odd |= (wd[t] & 0x7F800000u) == 0x7F800000u;
          }
        }
        odd = __any(odd);
      }
      if (odd) {
        for (int kk = 0; kk < 32; ++kk) {
          const int jj = (kk >> 3) * 4 + (kk & 3);
          float p = s[0];
#pragma unroll
          for (int j = 1; j < 16; ++j) p = jj == j ? s[j] : p;
          p = __shfl(p, l32 + 32 * ((kk >> 2) & 1));
          const bool seen = (see >> kk) & 1u;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int d = 32 * dt + 8 * (j / 4) + 4 * h + j % 4;
              const int ch = (d * ESZ / 16) ^ swz<T, HDP>(kk);
              const unsigned char* vp = vt + kk * RB + ch * 16 + (d * ESZ) % 16;
              const float v = HALF ? __uint_as_float((uint32_t) * (const uint16_t*)vp << 16) : *(const float*)vp;
              if (seen) o[dt][j] = __builtin_fmaf(p, v, o[dt][j]);
            }
        }
      } else if constexpr (HALF) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          // 16 lanes read four keys of 16 head-dim columns, transposed
          const int il = lane & 15, key = 16 * kk + 4 * h + (il >> 2);
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const int ch = 4 * dt + 2 * ((lane >> 4) & 1) + ((il & 3) >> 1);
            auto tr = [&](int k0) {
              const unsigned char* p = vt + k0 * RB + ((ch ^ swz<T, HDP>(k0)) * 16) + 8 * (il & 1);
              return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
            };
            const s16x4 v0 = tr(key), v1 = tr(key + 8);
            const uint2 u0 = __builtin_bit_cast(uint2, v0), u1 = __builtin_bit_cast(uint2, v1);
            const uint4 vf = make_uint4(u0.x, u0.y, u1.x, u1.y);
            o[dt] = mma(vf, ph[kk], o[dt], T());
            if (RW == 1) o[dt] = mma(vf, pl[kk], o[dt], T());
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int key = 8 * (j / 4) + 4 * h + j % 4;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const int d = 32 * dt + l32;
            const float v = *(const float*)(vt + key * RB + (((d / 4) ^ swz<T, HDP>(key)) * 16) + (d % 4) * 4);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[j], o[dt], 0, 0, 0);
          }
        }
      }
      wait_lds();
      if (RW > 1) barrier();
      if (more) issue(a.v, sV[kg], b + 1);
    }
    l = sum_x32(l);

    const bool whole = b0 == 0 && b1 == nb;
    const long long slot = 2ll * w + (b0 == 0 ? 1 : 0);
    if (!whole && b0 == 0) {
      const long long last = (u + nb - 1) / quota;  // the run that holds the tile's last block
      desc = make_int4((int)(last - w) + 1, x.row0, head, rt);
    }
    float* po = a.part + slot * BM * HDP;
    float* pm = a.part + 2ll * a.wgs * BM * HDP + slot * BM * 2;
    // four results of one row: to the output, or the partial
    auto put = [&](int lm, int d, float inv, const float (&v)[4]) {
      if (whole) {
        const int mm = rt * BM + lm;
        if (mm >= g.M || d >= hd) return;
        const int tk = mm / g.group;
        T* dst = (T*)a.out + (size_t)(x.row0 + tk) * (size_t)a.ldo +
                 (size_t)(head * g.group + (mm - tk * g.group)) * hd + d;
        if constexpr (HALF) *(uint2*)dst = make_uint2(bf2(v[0] * inv, v[1] * inv), bf2(v[2] * inv, v[3] * inv));
        else *(f32x4*)dst = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
      } else {
        *(f32x4*)(po + (size_t)lm * HDP + d) = f32x4{v[0], v[1], v[2], v[3]};
      }
    };
    if constexpr (RW == 1) {
      // the four waves' results, half of the columns at a time
      if (h == 0) sM[wv][l32] = mx, sL[wv][l32] = l;
      wait_lds();
      barrier();
      float top = fmaxf(fmaxf(sM[0][l32], sM[1][l32]), fmaxf(sM[2][l32], sM[3][l32]));
      const float f = mx == -INFINITY ? 0.f : ex2(mx - top);
      float* so = (float*)sK;
      constexpr int HC = HDP / 2;  // columns of a half
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
        for (int dt = 0; dt < NDT / 2; ++dt)
#pragma unroll
          for (int j4 = 0; j4 < 4; ++j4) {
            const f32x16& oo = o[hf * (NDT / 2) + dt];
            const int c4 = 8 * dt + 2 * j4 + h;  // four columns
            *(f32x4*)(so + ((wv * 32 + l32) * HC) + ((c4 ^ (l32 & 7)) * 4)) =
                f32x4{oo[4 * j4] * f, oo[4 * j4 + 1] * f, oo[4 * j4 + 2] * f, oo[4 * j4 + 3] * f};
          }
        wait_lds();
        barrier();
        for (int i = tid; i < 32 * (HC / 4); i += 256) {
          const int lm = i / (HC / 4), c4 = i % (HC / 4);
          float v[4] = {0.f, 0.f, 0.f, 0.f};
          const float t4 = fmaxf(fmaxf(sM[0][lm], sM[1][lm]), fmaxf(sM[2][lm], sM[3][lm]));
          float den = 0.f;
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const f32x4 y = *(const f32x4*)(so + ((q4 * 32 + lm) * HC) + ((c4 ^ (lm & 7)) * 4));
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] += y[t];
            den += sM[q4][lm] == -INFINITY ? 0.f : sL[q4][lm] * ex2(sM[q4][lm] - t4);
          }
          put(lm, hf * HC + c4 * 4, den > 0.f || den != den ? 1.f / den : 0.f, v);
          if (!whole && hf == 0 && c4 == 0) pm[2 * lm] = t4, pm[2 * lm + 1] = den;
        }
        wait_lds();
        barrier();
      }
    } else {
      const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          const float v[4] = {o[dt][4 * j4], o[dt][4 * j4 + 1], o[dt][4 * j4 + 2], o[dt][4 * j4 + 3]};
          put(rw * 32 + l32, 32 * dt + 8 * j4 + 4 * h, inv, v);
        }
      if (!whole && h == 0) pm[2 * (rw * 32 + l32)] = mx, pm[2 * (rw * 32 + l32) + 1] = l;
    }
    u += b1 - b0;
  }
  if (tid == 0) a.desc[w] = desc;
}

// Tiles whose keys several workgroups shared out: their partials, in order. A
// workgroup takes eight rows of one tile, a wave two of them.
template <typename T, int HDP, int BM>
__global__ __launch_bounds__(256) void k_tree_join(Args a) {
  const int w = blockIdx.x;
  const int4 d = a.desc[w];
  if (d.x == 0) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, hd = a.c.hd;
  // the entry's rows
  const int row0 = d.y, head = d.z, rt = d.w;
  const int e = wave_find(a.r.start, a.r.n_ent, row0);
  const Entry x = entry_of(a.c, a.r, e < a.r.n_ent ? e : a.r.n_ent - 1);
  constexpr int C = HDP / 64;
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    const int lm = blockIdx.y * 8 + wv * 2 + rr, mm = rt * BM + lm;
    if (mm >= x.n * a.group) continue;
    const float* pm = a.part + 2ll * a.wgs * BM * HDP;
    auto slot = [&](int i) { return i == 0 ? 2ll * w + 1 : 2ll * (w + i); };
    float top = -INFINITY;
    for (int i = lane; i < d.x; i += 64) top = fmaxf(top, pm[(slot(i) * BM + lm) * 2]);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
    float den = 0.f, o[C];
#pragma unroll
    for (int t = 0; t < C; ++t) o[t] = 0.f;
    for (int i0 = 0; i0 < d.x; i0 += 64) {
      float f = 0.f, ld = 0.f;
      if (i0 + lane < d.x) {
        const float m = pm[(slot(i0 + lane) * BM + lm) * 2];
        f = m == -INFINITY ? 0.f : ex2(m - top);
        ld = f == 0.f ? 0.f : f * pm[(slot(i0 + lane) * BM + lm) * 2 + 1];
      }
      const int cnt = d.x - i0 < 64 ? d.x - i0 : 64;
#pragma unroll 8
      for (int i = 0; i < cnt; ++i) {
        const float fi = __shfl(f, i);
        den += __shfl(ld, i);
        const float* po = a.part + (slot(i0 + i) * BM + lm) * HDP + lane * C;
#pragma unroll
        for (int t = 0; t < C; ++t) o[t] += fi == 0.f ? 0.f : fi * po[t];
      }
    }
    const float inv = den > 0.f || den != den ? 1.f / den : 0.f;
    const int tk = mm / a.group;
    T* dst = (T*)a.out + (size_t)(row0 + tk) * (size_t)a.ldo + (size_t)(head * a.group + (mm - tk * a.group)) * hd;
#pragma unroll
    for (int t = 0; t < C; ++t)
      if (lane * C + t < hd) {
        if constexpr (sizeof(T) == 2) dst[lane * C + t] = (T)bf2(o[t] * inv, 0.f);
        else dst[lane * C + t] = o[t] * inv;
      }
  }
}

int pad_hd(int dtype, int hd) { return hd <= 64 ? 64 : hd <= 128 ? 128 : 256; }

// Many rows to a sequence (on average more than two tiles of 32): tiles of
// 128 rows, whose waves share K and V.
int tile_rows(const TreeAttnDesc& d) {
  const long long rows = (long long)d.r.n_rows * (d.nq / d.c.nkv);
  return rows > 64ll * d.r.n_ent ? 128 : 32;
}
int tree_wgs(const TreeAttnDesc& d) { return std::max(8, d.cus / 8 * 8); }

template <typename T, int HDP, int RW>
hipError_t run(const TreeAttnDesc& d, const Args& a, hipStream_t st) {
  hipLaunchKernelGGL((k_tree<T, HDP, RW>), dim3(a.wgs), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_tree_join<T, HDP, 32 * RW>), dim3(a.wgs, 4 * RW), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t tree_attn_scratch(const TreeAttnDesc& d) {
  const size_t w = tree_wgs(d), rows = tile_rows(d), hdp = pad_hd(d.c.dtype, d.c.hd);
  return w * 16 + 2 * w * rows * (hdp + 2) * 4;
}

hipError_t launch_tree_attn(const TreeAttnDesc& d, hipStream_t st) {
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
  a.c2 = d.scale * LOG2E;
  const size_t layer = (size_t)d.layer * d.c.n_pages * d.c.nkv * d.c.page * d.c.hd * (d.c.dtype == DT_BF16 ? 2 : 4);
  a.k = (const char*)d.c.k + layer;
  a.v = (const char*)d.c.v + layer;
  a.wgs = tree_wgs(d);
  a.desc = (int4*)d.scratch;
  a.part = (float*)((char*)d.scratch + (size_t)a.wgs * 16);
  a.min_quota = 1;
  const int hdp = pad_hd(d.c.dtype, d.c.hd), rows = tile_rows(d);
  if (d.c.dtype == DT_BF16) {
    if (rows == 32) {
      return hdp == 64 ? run<uint16_t, 64, 1>(d, a, st) : hdp == 128 ? run<uint16_t, 128, 1>(d, a, st)
                                                                     : run<uint16_t, 256, 1>(d, a, st);
    }
    return hdp == 64 ? run<uint16_t, 64, 4>(d, a, st) : hdp == 128 ? run<uint16_t, 128, 4>(d, a, st)
                                                                   : run<uint16_t, 256, 4>(d, a, st);
  }
  if (hdp > 128) return hipErrorInvalidValue;
  if (rows == 32) return hdp == 64 ? run<float, 64, 1>(d, a, st) : run<float, 128, 1>(d, a, st);
  return hdp == 64 ? run<float, 64, 4>(d, a, st) : run<float, 128, 4>(d, a, st);
}

}  // namespace vla
