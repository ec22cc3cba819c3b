// Kernels of the paged KV cache: per-head norms and rotation with the store
// into pages, and the pages' own book-keeping (who holds which page, copies
// on a fork, accepted drafts moved together). Attention over it is in
// tree_dev.h.
#include <algorithm>

#include "paged_dev.h"

namespace vla {
using namespace pg;

// ---------------------------------------------------------------------------
// RMSNorm of queries and keys per head, rotation, store
// ---------------------------------------------------------------------------

// Rows times groups of heads above which a wave takes three groups. 32 query
// heads and 8 KV heads of 128: 512 rows (3,072 groups) 5.0 us with one and 5.5
// with three, 1,024 rows 7.7 and 6.4, 8,192 rows 47 and 33; 8 and 1 of 256: 512
// rows (2,048) 4.1 and 4.8, 1,024 rows 5.4 and 5.2.
constexpr long long MANY_WAVES = 4096;

// y = R(pos) (x / sqrt(mean(x^2) + eps) * g) for every query and key head, K
// and V into the cache. A wave takes one row and 64 / LPH heads of it at a
// time; a lane holds the two 16-byte chunks that the rotation pairs (elements
// i and i + rot / 2), so the rotation needs no other lane and the mean of
// squares one butterfly over the LPH lanes of a head. Squares, mean, angles
// and rotation are fp32; the result is rounded once.
//
// Bound by memory: every value is read and written once. A wave's loads are out
// before it looks for the row's sequence (four dependent round trips), and
// stores pass the L2 by when there are many rows. With many rows a wave takes
// three groups of heads, so that its look-ups are paid for more bytes; with
// few, one, so that more waves share the latency. 16,000 rows of 48 heads of 128
// (394 MB): 72 us, 5.4 TB/s.
template <typename T, int LPH, int U>
__global__ __launch_bounds__(256) void k_rope_norm(RopeNormDesc d, int parts) {
  constexpr int VEC = El<T>::VEC, HPW = 64 / LPH;
  const int lane = threadIdx.x & 63;
  const long long w = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(w / parts), part = (int)(w % parts);
  if (row >= d.r.n_rows) return;
  // the lane's two chunks: rotated pairs first, then the rest in neighbours
  const int half = d.rot / 2, hd = d.c.hd;
  const int sub = lane % LPH, hs = lane / LPH, np = hd / (2 * VEC), rp = half / VEC;
  const bool on = sub < np, turn = sub < rp;
  const int lo = turn ? sub * VEC : 2 * (rp * VEC) + 2 * (sub - rp) * VEC;
  const int hi = turn ? lo + half : lo + VEC;
  const int gq = (d.nq + HPW - 1) / HPW, gk = (d.c.nkv + HPW - 1) / HPW;
  // group g: 0 queries, 1 keys, 2 values; 3 behind the last
  auto kind_of = [&](int g) { return g < gq ? 0 : g < gq + gk ? 1 : g < gq + 2 * gk ? 2 : 3; };
  auto head_of = [&](int g, int kind) { return (kind == 0 ? g : kind == 1 ? g - gq : g - gq - gk) * HPW + hs; };
  u32x4 ua[U], ub[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int g = part + u * parts, kind = kind_of(g), head = head_of(g, kind);
    const bool live = on && kind < 3 && head < (kind == 0 ? d.nq : d.c.nkv);
    const T* src = (const T*)(kind == 0 ? d.q : kind == 1 ? d.k : d.v) +
                   (size_t)row * (size_t)(kind == 0 ? d.ldq : kind == 1 ? d.ldk : d.ldv);
    src += live ? (size_t)head * hd : 0;
    ua[u] = *(const u32x4*)(src + (live ? lo : 0));
    ub[u] = *(const u32x4*)(src + (live ? hi : 0));
  }
  const int e = wave_find(d.r.start, d.r.n_ent, row);
  if (e >= d.r.n_ent) return;
  const Entry x = entry_of(d.c, d.r, e);
  const int i = row - x.row0;
  if (x.seq < 0 || i < 0 || i >= x.n) return;
  const int slot = x.len + i;
  const int pos = d.pos ? d.pos[row] : slot;
  if (d.rot && (pos < 0 || pos >= d.n_pos)) {
    if (part == 0 && lane == 0) flag(d.c, PG_BAD);
    return;
  }
  const int page = page_of(d.c, x.seq, slot, x.cap);
  if (page < 0 && part == 0 && lane == 0) flag(d.c, PG_OUT);
  const int at = slot & (d.c.page - 1);
  float cs[VEC], sn[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) cs[j] = 1.f, sn[j] = 0.f;
  if (turn) {
    const float* pc = d.cs + (size_t)pos * half + lo;
    const float* ps = d.sn + (size_t)pos * half + lo;
#pragma unroll
    for (int j = 0; j < VEC; j += 4) {
      *(f32x4*)(cs + j) = *(const f32x4*)(pc + j);
      *(f32x4*)(sn + j) = *(const f32x4*)(ps + j);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int g = part + u * parts, kind = kind_of(g), head = head_of(g, kind);
    if (kind == 3) break;
    const bool live = on && head < (kind == 0 ? d.nq : d.c.nkv);
    if (kind < 2) {
      float a[VEC], b[VEC];
      unpack(ua[u], a);
      unpack(ub[u], b);
      const float* gp = kind == 0 ? d.q_gain : d.k_gain;
      if (gp) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) ss = __builtin_fmaf(a[j], a[j], __builtin_fmaf(b[j], b[j], ss));
        if (!on) ss = 0.f;
#pragma unroll
        for (int m = 1; m < LPH; m *= 2) ss += __shfl_xor(ss, m);
        const float inv = 1.f / sqrtf(ss / hd + d.eps);
        const float one = d.gain_plus_one ? 1.f : 0.f;
        if (on) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            a[j] *= inv * (one + gp[lo + j]);
            b[j] *= inv * (one + gp[hi + j]);
          }
        }
      }
      if (turn) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float t = a[j] * cs[j] - b[j] * sn[j];
          b[j] = b[j] * cs[j] + a[j] * sn[j];
          a[j] = t;
        }
      }
      ua[u] = pack(a);
      ub[u] = pack(b);
    }
    if (!live || (kind > 0 && page < 0)) continue;
    T* dst = kind == 0 ? (T*)d.q_out + (size_t)row * (size_t)d.ldo + (size_t)head * hd
                       : (T*)(kind == 1 ? d.c.k : d.c.v) + slot_elem(d.c, d.layer, page, head, at);
    if (U > 1) {
      __builtin_nontemporal_store(ua[u], (u32x4*)(dst + lo));
      __builtin_nontemporal_store(ub[u], (u32x4*)(dst + hi));
    } else {
      *(u32x4*)(dst + lo) = ua[u];
      *(u32x4*)(dst + hi) = ub[u];
    }
  }
}

// Lanes to a head, and what a launch is made of.
struct RopeNormGrid {
  int lph, parts;
  bool many;
  long long wgs;
  explicit RopeNormGrid(const RopeNormDesc& d) {
    const int np = d.c.hd / (d.c.dtype == DT_BF16 ? 16 : 8);  // lanes that a head keeps busy
    lph = np <= 2 ? 2 : np <= 4 ? 4 : np <= 8 ? 8 : 16;
    const int hpw = 64 / lph, groups = (d.nq + hpw - 1) / hpw + 2 * ((d.c.nkv + hpw - 1) / hpw);
    many = (long long)d.r.n_rows * groups > MANY_WAVES;
    parts = many ? (groups + 2) / 3 : groups;
    wgs = ((long long)d.r.n_rows * parts + 3) / 4;
  }
};
bool rope_norm_fits(const RopeNormDesc& d) { return launchable(RopeNormGrid(d).wgs, 256); }

template <typename T, int LPH>
static hipError_t rope_norm_l(const RopeNormDesc& d, const RopeNormGrid& g, hipStream_t st) {
  if (g.many) hipLaunchKernelGGL((k_rope_norm<T, LPH, 3>), dim3((unsigned)g.wgs), dim3(256), 0, st, d, g.parts);
  else hipLaunchKernelGGL((k_rope_norm<T, LPH, 1>), dim3((unsigned)g.wgs), dim3(256), 0, st, d, g.parts);
  return hipGetLastError();
}

template <typename T>
static hipError_t rope_norm_t(const RopeNormDesc& d, hipStream_t st) {
  const RopeNormGrid g(d);
  if (!launchable(g.wgs, 256)) return GRID_FULL;
  return g.lph == 2   ? rope_norm_l<T, 2>(d, g, st)
         : g.lph == 4 ? rope_norm_l<T, 4>(d, g, st)
         : g.lph == 8 ? rope_norm_l<T, 8>(d, g, st)
                      : rope_norm_l<T, 16>(d, g, st);
}

hipError_t launch_rope_norm(const RopeNormDesc& d, hipStream_t st) {
  if (d.r.n_rows <= 0 || d.r.n_ent <= 0) return hipSuccess;
  return d.c.dtype == DT_BF16 ? rope_norm_t<uint16_t>(d, st) : rope_norm_t<float>(d, st);
}

// ---------------------------------------------------------------------------
// Book-keeping. A page is free when no sequence holds it (refs 0), and free
// pages are dealt out lowest first, so what a call gives depends on the
// cache's state alone. One workgroup deals: the work is a scan of refs.
// ---------------------------------------------------------------------------

// Threads of the dealing workgroup: few while one to an entry are enough and
// the pool is small (barriers are most of the call: release, fork and reserve
// of 16 pairs 15.8 us with 256 threads and 17.3 with 1,024, of 250 pairs 51.1
// and 51.8), many where refs take long to scan.
constexpr int PT_FEW = 256, PT_MANY = 1024;
inline bool few_to_deal(const PagedCache& c, int n) { return n <= PT_FEW && c.n_pages <= 4 * 8 * PT_FEW; }

__global__ void k_pages_init(PagedCache c) {
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < (long long)c.n_seqs * c.max_pages) c.table[i] = -1;
  if (i < c.n_seqs) c.lens[i] = c.held[i] = 0;
  if (i < c.n_pages) c.refs[i] = 0;
  if (i == 0) *c.status = 0;
}

hipError_t launch_pages_init(const PagedCache& c, hipStream_t st) {
  const long long n = std::max({(long long)c.n_seqs * c.max_pages, (long long)c.n_pages, 1ll});
  const long long wgs = (n + 255) / 256;
  if (!launchable(wgs, 256)) return GRID_FULL;
  hipLaunchKernelGGL(k_pages_init, dim3((unsigned)wgs), dim3(256), 0, st, c);
  return hipGetLastError();
}

// Pages for len + rows slots of every entry, entries in order.
template <int PT>
__global__ __launch_bounds__(PT) void k_pages_reserve(PagedCache c, PagedRows r) {
  __shared__ int sList[PT], sOff[PT], sHeld[PT];
  __shared__ __attribute__((aligned(16))) int sSeq[PT];
  const int tid = threadIdx.x;
  const unsigned bits0 = free_bits(c, 0);
  int pos = 0;
  for (int base = 0; base < r.n_ent; base += PT) {
    const int e = base + tid;
    int seq = -1, held = 0, need = 0;
    if (e < r.n_ent) {
      const Entry x = entry_of(c, r, e);
      seq = x.seq;
      if (seq >= 0) {
        held = x.cap >> c.page_lg;
        const long long pages = ((long long)x.len + x.n + c.page - 1) >> c.page_lg;
        if (pages > c.max_pages) flag(c, PG_OUT);
        need = (int)(pages < c.max_pages ? pages : c.max_pages) - held;
        if (need < 0) need = 0;
      }
    }
    __syncthreads();  // the last round's lists are read
    sSeq[tid] = seq;
    sHeld[tid] = held;
    __syncthreads();
    // a sequence that is listed twice: the first entry counts
    if (need > 0) {
      bool again = false;
#pragma unroll 4
      for (int j = 0; j < tid; j += 4) {
        const int4 o = *(const int4*)(sSeq + j);
        const int q = tid - j;  // entries of these four that come before
        again = again || o.x == seq || (o.y == seq && q > 1) || (o.z == seq && q > 2) || (o.w == seq && q > 3);
      }
      if (again) need = 0;
    }
    // (64 bits: where start descends, entries name the same rows again and again.
    // No more are given than the pool has, so the offsets may end at 2^31 - 1.)
    long long sum;
    const long long at = block_scan<PT>((long long)need, &sum);
    const int off = (int)std::min(at, 0x7FFFFFFFll), total = (int)std::min(sum, 0x7FFFFFFFll);
    sOff[tid] = off;
    __syncthreads();
    int given = 0;
    while (given < total) {
      const int want = total - given < PT ? total - given : PT;
      const int got = take_free<PT>(c, bits0, &pos, want, sList);
      if (tid < got) {
        // the last entry whose pages start at or before this rank (entries
        // without pages share their offset with the next one)
        const int rank = given + tid;
        int lo = 0, hi = PT - 1;
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (sOff[mid] <= rank) lo = mid;
          else hi = mid - 1;
        }
        const int p = sList[tid];
        c.table[(size_t)sSeq[lo] * c.max_pages + sHeld[lo] + (rank - sOff[lo])] = p;
        c.refs[p] = 1;
      }
      given += got;
      __syncthreads();
      if (got < want) break;
    }
    if (need > 0) {
      const int mine = given - off < 0 ? 0 : given - off < need ? given - off : need;
      c.held[seq] = held + mine;
      if (mine < need) flag(c, PG_OUT);
    }
    __syncthreads();
    __threadfence_block();
  }
}

hipError_t launch_pages_reserve(const PagedCache& c, const PagedRows& r, hipStream_t st) {
  if (r.n_ent <= 0) return hipSuccess;
  if (few_to_deal(c, r.n_ent)) hipLaunchKernelGGL(k_pages_reserve<PT_FEW>, dim3(1), dim3(PT_FEW), 0, st, c, r);
  else hipLaunchKernelGGL(k_pages_reserve<PT_MANY>, dim3(1), dim3(PT_MANY), 0, st, c, r);
  return hipGetLastError();
}

// Fork, first half: who holds what. A pair may be made when both sequences are
// in range and the child was empty; it is made when no such pair before it has
// the same child, no such pair has its parent as child, and there is a page
// for its last slots. Pairs go by in rounds of PT; what may be made is told by
// made while there is more than one round.
template <int PT>
__global__ __launch_bounds__(PT) void k_pages_fork(PagedCache c, int n, const int32_t* src, const int32_t* dst,
                                                   int32_t* made) {
  __shared__ int sList[PT], sSrc[PT], sFull[PT];
  __shared__ __attribute__((aligned(16))) int sDst[PT];
  const int tid = threadIdx.x;
  const unsigned bits0 = free_bits(c, 0);
  auto may = [&](int s, int t) {
    const bool in = s >= 0 && s < c.n_seqs && t >= 0 && t < c.n_seqs && s != t;
    const int at = in ? t : 0;
    return in && (c.held[at] | c.lens[at]) == 0;
  };
  // what a pair's children are compared with is the state before the call, so
  // with several rounds all of it is looked at first
  if (n > PT) {
    for (int i = tid; i < n; i += PT) made[i] = may(src[i], dst[i]);
    __syncthreads();
  }
  auto child_of = [&](int i) {
    if (i >= n) return -1;
    const int t = dst[i];
    return (n > PT ? made[i] & 1 : may(src[i], t)) ? t : -1;
  };
  int pos = 0;
  for (int base = 0; base < n; base += PT) {
    const int i = base + tid;
    int s = -1, t = child_of(i), len = 0, full = 0, need = 0;
    if (i < n) s = src[i];
    bool ok = t >= 0;
    for (int b = 0; b < n; b += PT) {
      __syncthreads();
      sDst[tid] = b == base ? t : child_of(b + tid);
      __syncthreads();
      if (ok) {
        const int cnt = n - b < PT ? n - b : PT;  // (-1 behind the last)
#pragma unroll 4
        for (int j = 0; j < cnt; j += 4) {
          const int4 o = *(const int4*)(sDst + j);
          const int q = i - b - j;  // pairs of these four that come before
          ok = ok && o.x != s && o.y != s && o.z != s && o.w != s && !(o.x == t && q > 0) && !(o.y == t && q > 1) &&
               !(o.z == t && q > 2) && !(o.w == t && q > 3);
        }
      }
    }
    if (ok) {
      int h = c.held[s];
      h = h < 0 ? 0 : h > c.max_pages ? c.max_pages : h;
      const int l = c.lens[s], cap = h << c.page_lg;
      len = l < 0 ? 0 : l < cap ? l : cap;
      full = len >> c.page_lg;
      need = (len & (c.page - 1)) != 0;
    }
    int total;
    const int rank = block_scan<PT>(need, &total);
    const int got = take_free<PT>(c, bits0, &pos, total, sList);
    if (need && rank >= got) {  // no page for its last slots
      ok = false;
      flag(c, PG_OUT);
    }
    // (with several rounds, later ones still ask what may have been made: a
    // second bit tells what was)
    if (i < n) made[i] = n > PT ? (t >= 0 ? 1 : 0) | (ok ? 2 : 0) : ok;
    if (ok) {
      c.lens[t] = len;
      c.held[t] = full + need;
      if (need) {
        const int p = sList[rank];
        c.table[(size_t)t * c.max_pages + full] = p;
        c.refs[p] = 1;
      }
    }
    __syncthreads();
    sSrc[tid] = s;
    sDst[tid] = ok ? t : -1;
    sFull[tid] = full;
    __syncthreads();
    // the full pages are shared, 16 lanes to a pair
    for (int j = tid >> 4; j < PT && base + j < n; j += PT / 16) {
      if (sDst[j] < 0) continue;
      const int32_t* from = c.table + (size_t)sSrc[j] * c.max_pages;
      int32_t* to = c.table + (size_t)sDst[j] * c.max_pages;
      for (int k = tid & 15; k < sFull[j]; k += 64) {
        int p[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) p[u] = from[k + 16 * u < sFull[j] ? k + 16 * u : k];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (k + 16 * u < sFull[j]) {
            to[k + 16 * u] = p[u];
            if ((unsigned)p[u] < (unsigned)c.n_pages) atomicAdd(c.refs + p[u], 1);
          }
      }
    }
  }
  if (n > PT) {
    __syncthreads();
    for (int i = tid; i < n; i += PT) made[i] = made[i] >> 1;
  }
}

// Fork, second half: the used slots of the last page, K and V of FORK_HEADS
// heads (of all layers) to a workgroup, so that the descriptors' round trips
// are paid for more bytes. Bound by memory: 64 children, 306 MB in 54 us, 5.6
// TB/s (72 us with stores through the L2).
constexpr int FORK_HEADS = 4;
__global__ __launch_bounds__(256) void k_pages_copy(PagedCache c, const int32_t* src, const int32_t* dst,
                                                    const int32_t* made, int esz, int groups) {
  const int i = blockIdx.x / groups, g0 = blockIdx.x % groups * FORK_HEADS;
  const int ok = made[i], s = src[i], t = dst[i];
  if (!ok) return;
  const int len = c.lens[t], part = len & (c.page - 1), col = len >> c.page_lg;
  if (!part || col >= c.max_pages) return;
  const int ps = c.table[(size_t)s * c.max_pages + col], pt = c.table[(size_t)t * c.max_pages + col];
  if ((unsigned)ps >= (unsigned)c.n_pages || (unsigned)pt >= (unsigned)c.n_pages) return;
  const int chunks = part * c.hd * esz / 16, heads = c.layers * c.nkv;
  size_t from[FORK_HEADS], to[FORK_HEADS];
#pragma unroll
  for (int k = 0; k < FORK_HEADS; ++k) {
    const int g = g0 + k < heads ? g0 + k : heads - 1;
    from[k] = slot_elem(c, g / c.nkv, ps, g % c.nkv, 0) * esz;
    to[k] = slot_elem(c, g / c.nkv, pt, g % c.nkv, 0) * esz;
  }
  for (int j = threadIdx.x; j < chunks; j += 256) {
    u32x4 a[FORK_HEADS], b[FORK_HEADS];
#pragma unroll
    for (int k = 0; k < FORK_HEADS; ++k) {
      a[k] = ((const u32x4*)((const char*)c.k + from[k]))[j];
      b[k] = ((const u32x4*)((const char*)c.v + from[k]))[j];
    }
#pragma unroll
    for (int k = 0; k < FORK_HEADS; ++k) {
      if (g0 + k < heads) {
        __builtin_nontemporal_store(a[k], (u32x4*)((char*)c.k + to[k]) + j);
        __builtin_nontemporal_store(b[k], (u32x4*)((char*)c.v + to[k]) + j);
      }
    }
  }
}

static int copy_groups(const PagedCache& c) { return (c.layers * c.nkv + FORK_HEADS - 1) / FORK_HEADS; }
bool fork_fits(const PagedCache& c, int n) { return launchable((long long)n * copy_groups(c), 256); }
hipError_t launch_pages_fork(const PagedCache& c, int n, const int32_t* src, const int32_t* dst, int32_t* made,
                             hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const int groups = copy_groups(c);
  const long long wgs = (long long)n * groups;
  if (!fork_fits(c, n)) return GRID_FULL;
  if (few_to_deal(c, n)) hipLaunchKernelGGL(k_pages_fork<PT_FEW>, dim3(1), dim3(PT_FEW), 0, st, c, n, src, dst, made);
  else hipLaunchKernelGGL(k_pages_fork<PT_MANY>, dim3(1), dim3(PT_MANY), 0, st, c, n, src, dst, made);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)wgs), dim3(256), 0, st, c, src, dst, made,
                     c.dtype == DT_BF16 ? 2 : 4, groups);
  return hipGetLastError();
}

// A workgroup to a listed sequence. Counts go down by atomics whose order
// does not show; a sequence that is listed twice is empty the second time.
__global__ __launch_bounds__(256) void k_pages_release(PagedCache c, const int32_t* seqs) {
  __shared__ int sHeld;
  const int s = seqs[blockIdx.x];
  if (s < 0 || s >= c.n_seqs) return;
  if (threadIdx.x == 0) {
    const int h = atomicExch(c.held + s, 0);
    sHeld = h < 0 ? 0 : h > c.max_pages ? c.max_pages : h;
    c.lens[s] = 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < sHeld; i += 256) {
    int32_t* t = c.table + (size_t)s * c.max_pages + i;
    const int p = *t;
    *t = -1;
    if ((unsigned)p < (unsigned)c.n_pages) atomicSub(c.refs + p, 1);
  }
}

hipError_t launch_pages_release(const PagedCache& c, int n, const int32_t* seqs, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  if (!launchable(n, 256)) return GRID_FULL;
  hipLaunchKernelGGL(k_pages_release, dim3(n), dim3(256), 0, st, c, seqs);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Commit: accepted drafts move together
// ---------------------------------------------------------------------------

// Whether an entry's accepted list holds ascending drafts of its n, as far as
// thread `me` of `all` looks at it.
__device__ __forceinline__ bool kept_fine(const int32_t* kept, int n, int a, int me, int all) {
  bool ok = true;
  for (int j = me; j < a; j += all) {
    const int k = kept[j], b = j ? kept[j - 1] : -1;
    ok = ok && k >= 0 && k < n && k > b;
  }
  return ok;
}
__device__ __forceinline__ void grow(const PagedCache& c, const Entry& x, int a, bool fine) {
  if (!fine) {
    flag(c, PG_BAD);
    return;
  }
  const bool fits = x.len + a <= x.cap;
  if (!fits) flag(c, PG_OUT);
  c.lens[x.seq] = fits ? x.len + a : x.cap;
}

// Draft kept[j] moves to the slot of draft j. A thread owns one 16-byte
// column of one layer's K or V head and takes the drafts in order: a list
// ascends, so kept[j] >= j and no draft is written over before it is read
// (groups are read whole before they are written). With one workgroup to an
// entry (gridDim.y 1) it sets the new length as well. Bound by memory: 64
// entries' drafts, 89 MB in 19 us; few by seven dependent round trips, 7 us.
constexpr int KMOVE = 256;  // drafts whose places are worked out at a time
__global__ __launch_bounds__(1024) void k_pages_move(PagedCache c, PagedRows r, const int32_t* kept,
                                                     const int32_t* n_kept, int cpr, int esz) {
  __shared__ int2 sFrom[KMOVE], sTo[KMOVE];  // page, slot in it
  __shared__ int sCount;
  const int e = blockIdx.x, tid = threadIdx.x;
  const Entry x = entry_of(c, r, e);
  const int a = n_kept[e];
  if (x.seq < 0) return;
  const int32_t* list = kept + x.row0;
  const bool count = a >= 0 && a <= x.n;
  const bool fine = __syncthreads_and(count && kept_fine(list, x.n, a, tid, blockDim.x));
  const int per = blockDim.x / cpr, mine = tid / cpr, chunk = tid % cpr, combos = 2 * c.layers * c.nkv;
  for (int j0 = 0; fine && j0 < a; j0 += KMOVE) {
    __syncthreads();
    if (tid < 64) {  // the first wave lists what moves
      int n = 0;
      for (int q = 0; q < KMOVE; q += 64) {
        const int j = j0 + q + tid;
        const bool in = j < a;
        const int from = x.len + (in ? list[j] : 0), to = x.len + j;
        const int pf = in ? page_of(c, x.seq, from, x.cap) : -1, pt = in ? page_of(c, x.seq, to, x.cap) : -1;
        const bool go = pf >= 0 && pt >= 0 && from != to;
        const unsigned long long m = __ballot(go);
        if (go) {
          const int k = n + __popcll(m & ((1ull << tid) - 1));
          sFrom[k] = make_int2(pf, from & (c.page - 1));
          sTo[k] = make_int2(pt, to & (c.page - 1));
        }
        n += __popcll(m);
      }
      if (tid == 0) sCount = n;
    }
    __syncthreads();
    const int n = sCount;
    if (n == 0) continue;
    for (int co = blockIdx.y * per + mine; mine < per && co < combos; co += gridDim.y * per) {
      const int lh = co >> 1;
      char* base = (char*)(co & 1 ? c.v : c.k) + (size_t)chunk * 16;
      auto at = [&](int2 p) { return (u32x4*)(base + slot_elem(c, lh / c.nkv, p.x, lh % c.nkv, p.y) * esz); };
      for (int j = 0; j < n; j += 8) {
        u32x4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = *at(sFrom[j + u < n ? j + u : n - 1]);
        // (all of them read before any is written)
#pragma unroll
        for (int u = 0; u < 8; ++u) asm volatile("" : "+v"(v[u]));
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (j + u < n) __builtin_nontemporal_store(v[u], at(sTo[j + u]));
      }
    }
  }
  if (gridDim.y == 1 && tid == 0) grow(c, x, a, fine);
}

// The new lengths, a wave to an entry.
__global__ __launch_bounds__(256) void k_pages_grow(PagedCache c, PagedRows r, const int32_t* kept,
                                                    const int32_t* n_kept) {
  const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (e >= r.n_ent) return;
  const Entry x = entry_of(c, r, e);
  const int a = n_kept ? n_kept[e] : x.n;
  if (x.seq < 0) return;
  const bool count = a >= 0 && a <= x.n;
  const bool fine = __all(count && (!kept || kept_fine(kept + x.row0, x.n, a, lane, 64)));
  if (lane == 0) grow(c, x, a, fine);
}

hipError_t launch_pages_commit(const PagedCache& c, const PagedRows& r, const int32_t* kept, const int32_t* n_kept,
                               hipStream_t st) {
  if (r.n_ent <= 0) return hipSuccess;
  if (kept) {
    const int esz = c.dtype == DT_BF16 ? 2 : 4, cpr = c.hd * esz / 16, combos = 2 * c.layers * c.nkv;
    // About a column to each of 1,024 threads: one workgroup moves an entry's
    // drafts and sets its length. More: workgroups of 256, and a second launch
    // when all of them have read the old length (eight entries of 512 columns
    // 4.3 us against 5.6, 1,152 columns 5.5 / 5.7, 2,048 columns 7.1 / 5.7).
    const bool one = (long long)combos * cpr <= 1280;
    if (!launchable(r.n_ent, one ? 1024 : 256)) return GRID_FULL;
    if (one) {
      hipLaunchKernelGGL(k_pages_move, dim3(r.n_ent, 1), dim3(1024), 0, st, c, r, kept, n_kept, cpr, esz);
      return hipGetLastError();
    }
    const int per = 256 / cpr, gy = std::min((combos + per - 1) / per, 65535);
    hipLaunchKernelGGL(k_pages_move, dim3(r.n_ent, gy), dim3(256), 0, st, c, r, kept, n_kept, cpr, esz);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_pages_grow, dim3((r.n_ent + 3) / 4), dim3(256), 0, st, c, r, kept, n_kept);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// A context's prefix into a sequence
// ---------------------------------------------------------------------------

// A thread takes VEC keys by VEC head-dim elements: K's 16-byte runs lie along
// the head dim as the pages' do, V's along the keys, so V is turned in
// registers. 256 threads cover the elements of VEC keys first, so that rows are
// written in one piece. 305 rows of 256 in 18 layers, 11.2 MB: 7 us, the
// latency of its look-ups; once a frame.
template <typename T>
__global__ __launch_bounds__(256) void k_ctx_to_pages(PagedCache c, const T* k, const T* v, size_t lk, size_t lv, int nb,
                                                      int rows, int seq) {
  constexpr int VEC = El<T>::VEC, DT = sizeof(T) == 2 ? DT_BF16 : DT_F32;
  const int layer = blockIdx.y / c.nkv, j = blockIdx.y % c.nkv, chunks = c.hd / VEC;
  const int i = blockIdx.x * 256 + threadIdx.x, key0 = i / chunks * VEC, d0 = i % chunks * VEC;
  if (key0 >= rows) return;
  int h = c.held[seq], l = c.lens[seq];
  h = h < 0 ? 0 : h > c.max_pages ? c.max_pages : h;
  const int cap = h << c.page_lg;
  l = l < 0 ? 0 : l > cap ? cap : l;
  T a[VEC][VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e)
    *(u32x4*)a[e] = *(const u32x4*)(v + layer * lv + kv_vidx(DT, nb, c.hd, j, key0, d0 + e));
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int key = key0 + e;
    if (key >= rows) break;
    const int slot = l + key, page = page_of(c, seq, slot, cap);
    if (page < 0) {
      if (d0 == 0 && j == 0 && layer == 0) flag(c, PG_OUT);
      continue;
    }
    const size_t to = slot_elem(c, layer, page, j, slot & (c.page - 1)) + d0;
    T b[VEC];
#pragma unroll
    for (int t = 0; t < VEC; ++t) b[t] = a[t][e];
    *(u32x4*)((T*)c.v + to) = *(const u32x4*)b;
    *(u32x4*)((T*)c.k + to) = *(const u32x4*)(k + layer * lk + kv_kidx(DT, nb, c.hd, j, key, d0));
  }
}

hipError_t launch_ctx_to_pages(const PagedCache& c, const void* k, const void* v, size_t lk, size_t lv, int nb,
                               int rows, int seq, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  const int vec = c.dtype == DT_BF16 ? 8 : 4;
  const long long items = (long long)((rows + vec - 1) / vec) * (c.hd / vec);
  const dim3 grid((unsigned)((items + 255) / 256), (unsigned)(c.layers * c.nkv));
  if (grid.y > 65535) return GRID_FULL;
  if (c.dtype == DT_BF16)
    hipLaunchKernelGGL(k_ctx_to_pages<uint16_t>, grid, dim3(256), 0, st, c, (const uint16_t*)k, (const uint16_t*)v, lk,
                       lv, nb, rows, seq);
  else
    hipLaunchKernelGGL(k_ctx_to_pages<float>, grid, dim3(256), 0, st, c, (const float*)k, (const float*)v, lk, lv, nb,
                       rows, seq);
  return hipGetLastError();
}

}  // namespace vla
