// Device helpers of the paged cache's kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "deal.h"
#include "kernels.h"
#include "paged.h"

namespace vla {
namespace pg {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A lane's chunk: 16 bytes of a row, VEC elements.
template <typename T>
struct El;
template <>
struct El<float> {
  static constexpr int VEC = 4;
};
template <>
struct El<uint16_t> {
  static constexpr int VEC = 8;
};

// round to nearest, ties to even (the hardware conversion)
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
__device__ __forceinline__ void unpack(u32x4 u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack(u32x4 u, float (&x)[4]) {
  x[0] = __uint_as_float(u.x);
  x[1] = __uint_as_float(u.y);
  x[2] = __uint_as_float(u.z);
  x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
  return u32x4{bf2(x[0], x[1]), bf2(x[2], x[3]), bf2(x[4], x[5]), bf2(x[6], x[7])};
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
  return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

// Inclusive sum over the wave's lanes, by shifts inside rows of 16 lanes and
// broadcasts of their last ones (no LDS round trips).
template <int CTRL, int ROWS>
__device__ __forceinline__ void scan_step(int& v) {
  v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ void scan_step(long long& v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  v += (long long)(((unsigned long long)(uint32_t)hi << 32) | (uint32_t)lo);
}
template <typename I>
__device__ __forceinline__ I wave_scan(I v) {
  scan_step<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  scan_step<0x112, 0xf>(v);
  scan_step<0x114, 0xf>(v);
  scan_step<0x118, 0xf>(v);
  scan_step<0x142, 0xa>(v);  // row_bcast 15 to rows 1 and 3
  scan_step<0x143, 0xc>(v);  // row_bcast 31 to rows 2 and 3
  return v;
}
// The entry whose rows hold row t, by the whole wave: the largest e <= n with
// start[e] <= t (start[0] is taken to be; n: t lies behind the last entry).
// 64 entries a step, so 4,096 entries take two round trips. Every index stays
// in [1, n] whatever the values are.
__device__ __forceinline__ int wave_find(const int32_t* start, int n, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 64) {
    const int step = (len + 63) / 64;
    const int i = (lane + 1) * step;
    const int c = __popcll(__ballot(start[lo + (i < len ? i : len)] <= t));
    if (c * step >= len) return lo + len;
    lo += c * step;
    len = len - c * step < step ? len - c * step : step;
  }
  return lo + __popcll(__ballot(lane < len && start[lo + (lane < len ? lane + 1 : len)] <= t));
}

__device__ __forceinline__ Entry entry_of(const PagedCache& c, const PagedRows& r, int e) {
  // (every load is issued at once: an entry without a sequence reads the first)
  const int q = r.seqs ? r.seqs[e] : e;
  const bool in = q >= 0 && q < c.n_seqs;
  const int at = in ? q : 0;
  const int a = r.start[e], b = r.start[e + 1], h = c.held[at], l = c.lens[at];
  Entry x;
  x.seq = in ? q : -1;
  x.row0 = a < 0 ? 0 : a > r.n_rows ? r.n_rows : a;
  const int end = b > r.n_rows ? r.n_rows : b;
  x.n = in && end > x.row0 ? end - x.row0 : 0;
  x.cap = (h < 0 || !in ? 0 : h > c.max_pages ? c.max_pages : h) << c.page_lg;
  x.len = l < 0 ? 0 : l > x.cap ? x.cap : l;
  return x;
}

// The page of a slot of sequence s (-1: none).
__device__ __forceinline__ int page_of(const PagedCache& c, int s, int slot, int cap) {
  if (slot < 0 || slot >= cap) return -1;
  const int p = c.table[(size_t)s * c.max_pages + (slot >> c.page_lg)];
  return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}
// Elements before slot `at` of KV head j in page p of a layer.
__device__ __forceinline__ size_t slot_elem(const PagedCache& c, int layer, int p, int j, int at) {
  return ((((size_t)layer * c.n_pages + p) * c.nkv + j) * c.page + at) * c.hd;
}
// Exclusive prefix of x over the workgroup, and the total.
template <int PT, typename I>
__device__ __forceinline__ I block_scan(I x, I* total) {
  __shared__ I sW[PT / 64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const I s = wave_scan(x);
  __syncthreads();  // the last call's sums are read
  if (lane == 63) sW[wv] = s;
  __syncthreads();
  I before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < PT / 64; ++i) {
    const I v = sW[i];
    before += i < wv ? v : 0;
    all += v;
  }
  *total = all;
  return before + s - x;
}

// Which of the thread's eight pages of the 8 PT from `base` on are free.
__device__ __forceinline__ unsigned free_bits(const PagedCache& c, int base) {
  const int first = base + 8 * threadIdx.x;
  unsigned bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int p = first + j < c.n_pages ? first + j : c.n_pages - 1;
    if (c.refs[p] == 0 && first + j < c.n_pages) bits |= 1u << j;
  }
  return bits;
}
// The next `want` (<= PT) free pages from page *pos on, ascending, into list;
// returns how many there are and moves *pos behind the last one taken. Pages
// that this launch gave out lie before *pos, so refs may be read as it was;
// bits0 is free_bits(0), which a kernel reads while it has nothing else.
template <int PT>
__device__ __forceinline__ int take_free(const PagedCache& c, unsigned bits0, int* pos, int want, int* list) {
  int found = 0, p0 = *pos;
  for (int base = p0 & ~(8 * PT - 1); found < want && base < c.n_pages; base += 8 * PT) {
    const int first = base + 8 * threadIdx.x;
    unsigned bits = base == 0 ? bits0 : free_bits(c, base);
    if (first < p0) bits &= p0 - first < 8 ? ~0u << (p0 - first) : 0u;
    int total;
    int rank = found + block_scan<PT>((int)__popc(bits), &total);
    for (; bits && rank < want; bits &= bits - 1, ++rank) list[rank] = first + __ffs(bits) - 1;
    found += total;
  }
  __syncthreads();
  const int got = found < want ? found : want;
  *pos = found < want ? c.n_pages : got ? list[got - 1] + 1 : p0;
  return got;
}

__device__ __forceinline__ void flag(const PagedCache& c, int bit) { atomicOr(c.status, bit); }

}  // namespace pg
}  // namespace vla
