// Kernels of the paged KV cache: per-head norms and rotation with the store
// into pages, and the pages' own book-keeping (who holds which page, copies
// on a fork, accepted drafts moved together). Attention over it is in
// tree.hip.
#include <algorithm>

#include "paged_dev.h"

namespace vla {
using namespace pg;

// ---------------------------------------------------------------------------
// RMSNorm of queries and keys per head, rotation, store
// ---------------------------------------------------------------------------

// y = R(pos) (x / sqrt(mean(x^2) + eps) * g) for every query and key head, K
// and V into the cache. A wave takes one row and 64 / LPH heads of it at a
// time; a lane holds the two 16-byte chunks that the rotation pairs (elements
// i and i + rot / 2), so the rotation needs no other lane and the mean of
// squares one butterfly over the LPH lanes of a head. Squares, mean, angles
// and rotation are fp32; the result is rounded once.
template <typename T, int LPH>
__global__ __launch_bounds__(256) void k_rope_norm(RopeNormDesc d, int parts) {
  constexpr int VEC = El<T>::VEC, HPW = 64 / LPH;
  const int lane = threadIdx.x & 63;
  const long long w = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(w / parts), part = (int)(w % parts);
  if (row >= d.r.n_rows) return;
  const int e = wave_find(d.r.start, d.r.n_ent, row);
  if (e >= d.r.n_ent) return;
  const Entry x = entry_of(d.c, d.r, e);
  const int i = row - x.row0;
  if (x.seq < 0 || i < 0 || i >= x.n) return;
  const int slot = x.len + i;
  const int pos = d.pos ? d.pos[row] : slot;
  const int half = d.rot / 2;
  if (d.rot && (pos < 0 || pos >= d.n_pos)) {
    if (part == 0 && lane == 0) flag(d.c, PG_BAD);
    return;
  }
  const int page = page_of(d.c, x.seq, slot, x.cap);
  if (page < 0 && part == 0 && lane == 0) flag(d.c, PG_OUT);
  const int at = slot & (d.c.page - 1);

  // the lane's two chunks: rotated pairs first, then the rest in neighbours
  const int sub = lane % LPH, hs = lane / LPH, np = d.c.hd / (2 * VEC), rp = half / VEC;
  const bool on = sub < np, turn = sub < rp;
  const int lo = turn ? sub * VEC : 2 * (rp * VEC) + 2 * (sub - rp) * VEC;
  const int hi = turn ? lo + half : lo + VEC;
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
  const int gq = (d.nq + HPW - 1) / HPW, gk = (d.c.nkv + HPW - 1) / HPW;
  for (int g = part; g < gq + 2 * gk; g += parts) {
    const int kind = g < gq ? 0 : g < gq + gk ? 1 : 2;
    const int head = (kind == 0 ? g : kind == 1 ? g - gq : g - gq - gk) * HPW + hs;
    const bool live = on && head < (kind == 0 ? d.nq : d.c.nkv);
    const T* src = (const T*)(kind == 0 ? d.q : kind == 1 ? d.k : d.v) +
                   (size_t)row * (size_t)(kind == 0 ? d.ldq : kind == 1 ? d.ldk : d.ldv) + (size_t)head * d.c.hd;
    uint4 ua = make_uint4(0, 0, 0, 0), ub = ua;
    if (live) {
      ua = *(const uint4*)(src + lo);
      ub = *(const uint4*)(src + hi);
    }
    T* dst;
    if (kind == 0) {
      dst = (T*)d.q_out + (size_t)row * (size_t)d.ldo + (size_t)head * d.c.hd;
    } else {
      dst = (T*)(kind == 1 ? d.c.k : d.c.v) + (page < 0 ? 0 : slot_elem(d.c, d.layer, page, head, at));
    }
    const bool put = live && (kind == 0 || page >= 0);
    if (kind < 2) {
      float a[VEC], b[VEC];
      unpack(ua, a);
      unpack(ub, b);
      const float* gp = kind == 0 ? d.q_gain : d.k_gain;
      if (gp) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) ss = __builtin_fmaf(a[j], a[j], __builtin_fmaf(b[j], b[j], ss));
#pragma unroll
        for (int m = 1; m < LPH; m *= 2) ss += __shfl_xor(ss, m);
        const float inv = 1.f / sqrtf(ss / d.c.hd + d.eps);
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
          const float u = a[j] * cs[j] - b[j] * sn[j];
          b[j] = b[j] * cs[j] + a[j] * sn[j];
          a[j] = u;
        }
      }
      ua = pack(a);
      ub = pack(b);
    }
    if (put) {
      *(uint4*)(dst + lo) = ua;
      *(uint4*)(dst + hi) = ub;
    }
  }
}

template <typename T>
static hipError_t rope_norm_t(const RopeNormDesc& d, hipStream_t st) {
  const int np = d.c.hd / (2 * El<T>::VEC);
  const int lph = np <= 2 ? 2 : np <= 4 ? 4 : np <= 8 ? 8 : 16;
  const int hpw = 64 / lph;
  const int groups = (d.nq + hpw - 1) / hpw + 2 * ((d.c.nkv + hpw - 1) / hpw);
  const int parts = groups;
  const long long wgs = ((long long)d.r.n_rows * parts + 3) / 4;
  if (wgs > 0x7FFFFFFFll) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs), block(256);
  switch (lph) {
    case 2:
      hipLaunchKernelGGL((k_rope_norm<T, 2>), grid, block, 0, st, d, parts);
      break;
    case 4:
      hipLaunchKernelGGL((k_rope_norm<T, 4>), grid, block, 0, st, d, parts);
      break;
    case 8:
      hipLaunchKernelGGL((k_rope_norm<T, 8>), grid, block, 0, st, d, parts);
      break;
    default:
      hipLaunchKernelGGL((k_rope_norm<T, 16>), grid, block, 0, st, d, parts);
  }
  return hipGetLastError();
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

constexpr int PT = 1024;  // threads of the dealing workgroup

// Exclusive prefix of x over the workgroup, and the total.
__device__ __forceinline__ int block_scan(int x, int* total) {
  __shared__ int sW[PT / 64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int s = x;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const int y = __shfl_up(s, m);
    if (lane >= m) s += y;
  }
  __syncthreads();  // the last call's sums are read
  if (lane == 63) sW[wv] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < PT / 64; ++i) {
    const int v = sW[i];
    before += i < wv ? v : 0;
    all += v;
  }
  *total = all;
  return before + s - x;
}

// The next `want` (<= PT) free pages from page *pos on, ascending, into list;
// returns how many there are and moves *pos behind the last one taken. Pages
// that this launch gave out lie before *pos, so refs may be read as it was.
__device__ int take_free(const PagedCache& c, int* pos, int want, int* list) {
  int found = 0, p0 = *pos;
  for (int base = p0 & ~7; found < want && base < c.n_pages; base += 8 * PT) {
    const int first = base + 8 * threadIdx.x;
    unsigned bits = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int p = first + j;
      if (p >= p0 && p < c.n_pages && c.refs[p] == 0) bits |= 1u << j;
    }
    int total;
    int rank = found + block_scan(__popc(bits), &total);
    for (; bits && rank < want; bits &= bits - 1, ++rank) list[rank] = first + __ffs(bits) - 1;
    found += total;
  }
  __syncthreads();
  const int got = found < want ? found : want;
  *pos = found < want ? c.n_pages : got ? list[got - 1] + 1 : p0;
  return got;
}

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
  if (wgs > 0x7FFFFFFFll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_pages_init, dim3((unsigned)wgs), dim3(256), 0, st, c);
  return hipGetLastError();
}

// Pages for len + rows slots of every entry, entries in order.
__global__ __launch_bounds__(PT) void k_pages_reserve(PagedCache c, PagedRows r) {
  __shared__ int sList[PT], sOff[PT], sSeq[PT], sHeld[PT];
  const int tid = threadIdx.x;
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
    if (need > 0)
      for (int j = 0; j < tid; ++j)
        if (sSeq[j] == seq) {
          need = 0;
          break;
        }
    int total;
    const int off = block_scan(need, &total);
    sOff[tid] = off;
    __syncthreads();
    int given = 0;
    while (given < total) {
      const int want = total - given < PT ? total - given : PT;
      const int got = take_free(c, &pos, want, sList);
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
  hipLaunchKernelGGL(k_pages_reserve, dim3(1), dim3(PT), 0, st, c, r);
  return hipGetLastError();
}

// Fork, first half: who holds what. A pair is made when both sequences are
// in range, the child was empty, no earlier pair of the call has the same
// child and the parent is no child of the call. Children are claimed by the
// lowest pair index in lens (0 for an empty sequence; claims are negative).
constexpr int CLAIM = 1 << 30;
__global__ __launch_bounds__(PT) void k_pages_fork(PagedCache c, int n, const int32_t* src, const int32_t* dst,
                                                   int32_t* made) {
  __shared__ int sList[PT], sSrc[PT], sDst[PT], sFull[PT];
  const int tid = threadIdx.x;
  auto len_of = [&](int s) { return __hip_atomic_load(c.lens + s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  for (int i = tid; i < n; i += PT) {
    const int s = src[i], t = dst[i];
    if (s < 0 || s >= c.n_seqs || t < 0 || t >= c.n_seqs || s == t || c.held[t] != 0) continue;
    if (len_of(t) <= 0) atomicMin(c.lens + t, i - CLAIM);
  }
  __syncthreads();
  for (int i = tid; i < n; i += PT) {
    const int s = src[i], t = dst[i];
    const bool in = s >= 0 && s < c.n_seqs && t >= 0 && t < c.n_seqs && s != t;
    made[i] = in && len_of(t) == i - CLAIM && len_of(s) >= 0;
  }
  __syncthreads();
  int pos = 0;
  for (int base = 0; base < n; base += PT) {
    const int i = base + tid;
    int s = -1, t = -1, len = 0, full = 0, need = 0;
    if (i < n) {
      s = src[i];
      t = dst[i];
      if (made[i]) {
        int h = c.held[s];
        h = h < 0 ? 0 : h > c.max_pages ? c.max_pages : h;
        const int l = len_of(s), cap = h << c.page_lg;
        len = l < cap ? l : cap;
        full = len >> c.page_lg;
        need = (len & (c.page - 1)) != 0;
      } else {
        if (t >= 0 && t < c.n_seqs && len_of(t) == i - CLAIM)
          __hip_atomic_store(c.lens + t, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s = t = -1;
      }
    }
    int total;
    const int rank = block_scan(need, &total);
    const int got = take_free(c, &pos, total, sList);
    if (need && rank >= got) {  // no page for its last slots: not made
      __hip_atomic_store(c.lens + t, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      made[i] = 0;
      flag(c, PG_OUT);
      s = t = -1;
    }
    if (t >= 0) {
      __hip_atomic_store(c.lens + t, len, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      c.held[t] = full + need;
      if (need) {
        const int p = sList[rank];
        c.table[(size_t)t * c.max_pages + full] = p;
        c.refs[p] = 1;
      }
    }
    sSrc[tid] = s;
    sDst[tid] = t;
    sFull[tid] = full;
    __syncthreads();
    // the full pages are shared, a wave to a pair
    for (int j = tid >> 6; j < PT && base + j < n; j += PT / 64) {
      if (sDst[j] < 0) continue;
      const int32_t* from = c.table + (size_t)sSrc[j] * c.max_pages;
      int32_t* to = c.table + (size_t)sDst[j] * c.max_pages;
      for (int k = tid & 63; k < sFull[j]; k += 64) {
        const int p = from[k];
        to[k] = p;
        if ((unsigned)p < (unsigned)c.n_pages) atomicAdd(c.refs + p, 1);
      }
    }
    __syncthreads();
  }
}

// Fork, second half: the used slots of the last page, K and V of one layer
// and KV head to a workgroup.
__global__ __launch_bounds__(256) void k_pages_copy(PagedCache c, const int32_t* src, const int32_t* dst,
                                                    const int32_t* made, int esz) {
  const int i = blockIdx.x / (c.layers * c.nkv), lh = blockIdx.x % (c.layers * c.nkv);
  if (!made[i]) return;
  const int s = src[i], t = dst[i], len = c.lens[t];
  const int part = len & (c.page - 1), cap = c.held[t] << c.page_lg;
  if (!part) return;
  const int ps = page_of(c, s, len, cap), pt = page_of(c, t, len, cap);
  if (ps < 0 || pt < 0) return;
  const size_t from = slot_elem(c, lh / c.nkv, ps, lh % c.nkv, 0) * esz;
  const size_t to = slot_elem(c, lh / c.nkv, pt, lh % c.nkv, 0) * esz;
  const int chunks = part * c.hd * esz / 16;
  const uint4 *ka = (const uint4*)((const char*)c.k + from), *va = (const uint4*)((const char*)c.v + from);
  uint4 *kb = (uint4*)((char*)c.k + to), *vb = (uint4*)((char*)c.v + to);
  for (int j = threadIdx.x; j < chunks; j += 256) {
    const uint4 a = ka[j], b = va[j];
    kb[j] = a;
    vb[j] = b;
  }
}

hipError_t launch_pages_fork(const PagedCache& c, int n, const int32_t* src, const int32_t* dst, int32_t* made,
                             hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const long long wgs = (long long)n * c.layers * c.nkv;
  if (wgs > 0x7FFFFFFFll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_pages_fork, dim3(1), dim3(PT), 0, st, c, n, src, dst, made);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)wgs), dim3(256), 0, st, c, src, dst, made,
                     c.dtype == DT_BF16 ? 2 : 4);
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
  hipLaunchKernelGGL(k_pages_release, dim3(n), dim3(256), 0, st, c, seqs);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Commit: accepted drafts move together
// ---------------------------------------------------------------------------

// Whether entry x's accepted list holds ascending drafts of it, by a whole
// workgroup of 256 (or one wave with W = 64).
template <int W>
__device__ __forceinline__ bool kept_fine(const int32_t* kept, int n, int a) {
  bool ok = true;
  for (int j = threadIdx.x % W; j < a; j += W) {
    const int k = kept[j];
    ok = ok && k >= 0 && k < n && (j == 0 || k > kept[j - 1]);
  }
  return W == 64 ? __all(ok) : __syncthreads_and(ok);
}
__device__ __forceinline__ int kept_count(const int32_t* n_kept, int e, int n) {
  return n_kept ? n_kept[e] : n;
}

// Draft kept[j] moves to the slot of draft j. A thread owns one 16-byte
// column of one layer's K or V head and takes the drafts in order: a list
// ascends, so kept[j] >= j and no draft is written over before it is read
// (groups are read whole before they are written).
constexpr int KMOVE = 256;  // drafts whose places are worked out at a time
__global__ __launch_bounds__(256) void k_pages_move(PagedCache c, PagedRows r, const int32_t* kept,
                                                    const int32_t* n_kept, int cpr, int esz) {
  __shared__ int sFrom[KMOVE], sTo[KMOVE], sFromAt[KMOVE], sToAt[KMOVE];
  const int e = blockIdx.x;
  const Entry x = entry_of(c, r, e);
  const int a = kept_count(n_kept, e, x.n);
  if (x.seq < 0 || a <= 0 || a > x.n) return;
  const int32_t* list = kept + x.row0;
  if (!kept_fine<256>(list, x.n, a)) return;
  const int per = 256 / cpr;
  const int combo = blockIdx.y * per + (int)threadIdx.x / cpr, chunk = (int)threadIdx.x % cpr;
  const bool live = (int)threadIdx.x < per * cpr && combo < 2 * c.layers * c.nkv;
  const int kv = combo & 1, lh = combo >> 1;
  char* base = (char*)(kv ? c.v : c.k) + (size_t)chunk * 16;
  const size_t lbase = live ? (size_t)(lh / c.nkv) * c.n_pages : 0;
  const int head = lh % c.nkv;
  auto at = [&](int page, int slot) {
    return (uint4*)(base + ((((lbase + page) * c.nkv + head) * c.page + slot) * c.hd) * esz);
  };
  for (int j0 = 0; j0 < a; j0 += KMOVE) {
    const int cnt = a - j0 < KMOVE ? a - j0 : KMOVE;
    __syncthreads();
    if ((int)threadIdx.x < cnt) {
      const int j = j0 + threadIdx.x, from = x.len + list[j], to = x.len + j;
      const int pf = page_of(c, x.seq, from, x.cap), pt = page_of(c, x.seq, to, x.cap);
      sFrom[threadIdx.x] = pt < 0 || from == to ? -1 : pf;
      sTo[threadIdx.x] = pt;
      sFromAt[threadIdx.x] = from & (c.page - 1);
      sToAt[threadIdx.x] = to & (c.page - 1);
    }
    __syncthreads();
    if (!live) continue;
    for (int j = 0; j < cnt; j += 8) {
      uint4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (j + u < cnt && sFrom[j + u] >= 0) v[u] = *at(sFrom[j + u], sFromAt[j + u]);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (j + u < cnt && sFrom[j + u] >= 0) *at(sTo[j + u], sToAt[j + u]) = v[u];
    }
  }
}

// The new lengths, a wave to an entry.
__global__ __launch_bounds__(256) void k_pages_grow(PagedCache c, PagedRows r, const int32_t* kept,
                                                    const int32_t* n_kept) {
  const int e = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (e >= r.n_ent) return;
  const Entry x = entry_of(c, r, e);
  const int a = kept_count(n_kept, e, x.n);
  if (x.seq < 0) return;
  const bool fine = a >= 0 && a <= x.n && (!kept || kept_fine<64>(kept + x.row0, x.n, a));
  if ((threadIdx.x & 63) != 0) return;
  if (!fine) {
    flag(c, PG_BAD);
    return;
  }
  const bool fits = x.len + a <= x.cap;
  if (!fits) flag(c, PG_OUT);
  c.lens[x.seq] = fits ? x.len + a : x.cap;
}

hipError_t launch_pages_commit(const PagedCache& c, const PagedRows& r, const int32_t* kept, const int32_t* n_kept,
                               hipStream_t st) {
  if (r.n_ent <= 0) return hipSuccess;
  if (kept) {
    const int esz = c.dtype == DT_BF16 ? 2 : 4, cpr = c.hd * esz / 16, per = 256 / cpr;
    const int combos = 2 * c.layers * c.nkv;
    const int gy = (combos + per - 1) / per;
    if (gy > 65535) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_pages_move, dim3(r.n_ent, gy), dim3(256), 0, st, c, r, kept, n_kept, cpr, esz);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_pages_grow, dim3((r.n_ent + 3) / 4), dim3(256), 0, st, c, r, kept, n_kept);
  return hipGetLastError();
}

}  // namespace vla
