// Cutting sequences of a paged KV cache back to their weightiest slots: weights
// summed over layers and heads, the largest picked, and the kept slots' K, V and
// weights moved together in every layer.
#include <algorithm>

#include "paged_dev.h"

namespace vla {
using namespace pg;

namespace {

constexpr int PICK = 1024;   // threads that pick a sequence's slots
constexpr int MOVE = 256, U = 8;  // threads that move, and chunks that each has in flight

// What the first kernels found out about an entry.
struct Cut {
  int seq;          // -1: skipped
  int len, cap;     // slots before, and those that its pages hold
  int stay;         // slots after
  int gap;          // the first slot that goes
  int fresh;        // pages that take the place of shared ones
  int pad[2];
};

struct Ev {
  EvictDesc d;
  Cut* cut;        // [n]
  int32_t* fresh;  // [n][max_pages]: the page in place of a shared one, -1 (where an entry has any)
  double* score;   // [n][slots]
  int slots;
};

__device__ __forceinline__ Entry state_of(const PagedCache& c, int s) {
  Entry x{-1, 0, 0, 0, 0};
  if (s < 0 || s >= c.n_seqs) return x;
  const int h = c.held[s], l = c.lens[s];
  x.seq = s;
  x.cap = (h < 0 ? 0 : h > c.max_pages ? c.max_pages : h) << c.page_lg;
  x.len = l < 0 ? 0 : l > x.cap ? x.cap : l;
  return x;
}

// A slot's weight: the sum over layers and heads.
__global__ __launch_bounds__(256) void k_evict_score(Ev e) {
  const PagedCache& c = e.d.c;
  const int i = blockIdx.y, slot = blockIdx.x * 256 + threadIdx.x;
  const Entry x = state_of(c, e.d.seqs[i]);
  if (slot >= x.len || x.len <= e.d.keep[i]) return;
  const float* p = e.d.mass + (size_t)x.seq * c.nkv * e.slots + slot;
  const size_t layer = (size_t)c.n_seqs * c.nkv * e.slots;
  // (eight loads of the inner loop are out together: heads where there are as
  // many, whose rows are neighbours, else layers if there are more of them. 16
  // sequences of 3,000 slots, 28 layers: of 8 heads 27 us so and 39 the other way
  // round, of 1, 4 and 7 heads 8, 21 and 35 us, and 16, 52 and 87; 4 layers of 4
  // heads 9 and 10)
  const bool deep = c.nkv < 8 && c.layers > c.nkv;
  const int n0 = deep ? c.nkv : c.layers, n1 = deep ? c.layers : c.nkv;
  const size_t s0 = deep ? (size_t)e.slots : layer, s1 = deep ? layer : (size_t)e.slots;
  double sum = 0;
  for (int i0 = 0; i0 < n0; ++i0)
#pragma unroll 8
    for (int i1 = 0; i1 < n1; ++i1) sum += p[i0 * s0 + i1 * s1];
  e.score[(size_t)i * e.slots + slot] = sum;
}

// Which slots stay. Weights are not negative, so their bits order them: the
// keep-th largest is found eight bits at a time from counts in the LDS, and the
// kept slots are listed in order. A thread looks at neighbouring slots. Bound by
// the counts' barriers and conflicts, 1.2 us a pass, of which random weights
// take five or so: 12 us for 700 to 1,500 slots, 15 for 4,000.
__global__ __launch_bounds__(PICK) void k_evict_pick(Ev e) {
  typedef unsigned long long u64;
  const PagedCache& c = e.d.c;
  __shared__ int sHist[256], sBin, sAbove, sGap;
  const int i = blockIdx.x, tid = threadIdx.x;
  const int s = e.d.seqs[i];
  const Entry x = state_of(c, s);
  bool again = false;
  for (int j = tid; j < i; j += PICK) again = again || e.d.seqs[j] == s;
  again = __syncthreads_or(again);
  const int keep = e.d.keep[i];
  if (x.seq < 0 || again || keep < 0) {
    if (tid == 0) {
      e.cut[i].seq = -1;
      if (x.seq >= 0 && !again) flag(c, PG_BAD);
    }
    return;
  }
  int32_t* kept = e.d.kept + (size_t)i * e.slots;
  if (x.len <= keep) {
    for (int j = tid; j < x.len; j += PICK) kept[j] = j;
    if (tid == 0) e.cut[i] = Cut{x.seq, x.len, x.cap, x.len, x.len, 0};
    return;
  }
  const int per = (x.len + PICK - 1) / PICK, j0 = tid * per, j1 = min(j0 + per, x.len);
  const u64* score = (const u64*)(e.score + (size_t)i * e.slots);
  auto key = [&](int j) -> u64 {
    if (j < e.d.first || (long long)j >= (long long)x.len - e.d.last) return ~0ull;
    const u64 v = score[j];
    // (what is negative or not a number has the sign or lies above infinity)
    return v > 0x7FF0000000000000ull ? 0ull : v;
  };
  // (of up to 4,096 slots the keys stay in registers)
  constexpr int KEYS = 4;
  u64 own[KEYS];
#pragma unroll
  for (int k = 0; k < KEYS; ++k) own[k] = per <= KEYS && j0 + k < j1 ? key(j0 + k) : 0;
  auto each = [&](auto&& f) {
    if (per <= KEYS) {
#pragma unroll
      for (int k = 0; k < KEYS; ++k)
        if (j0 + k < j1) f(own[k], j0 + k);
    } else {
#pragma unroll 4
      for (int j = j0; j < j1; ++j) f(key(j), j);
    }
  };
  int want = keep;  // of those whose upper bits are `prefix`
  u64 prefix = 0, mask = 0;
  if (keep > 0)
    for (int sh = 56; sh >= 0; sh -= 8) {
      if (tid < 256) sHist[tid] = 0;
      __syncthreads();
      each([&](u64 k, int) {
        if ((k & mask) == prefix) atomicAdd(&sHist[(int)(k >> sh) & 255], 1);
      });
      __syncthreads();
      if (tid < 64) {
        // bins from the top: lane l has 255 - 4 l and the three below
        int n[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += n[k] = sHist[255 - 4 * tid - k];
        int above = wave_scan(sum) - sum;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (above < want && above + n[k] >= want) sBin = 255 - 4 * tid - k, sAbove = above;
          above += n[k];
        }
      }
      __syncthreads();
      const int bin = sBin;
      want -= sAbove;
      prefix |= (u64)bin << sh;
      mask |= 255ull << sh;
      if (sHist[bin] == want) break;  // all of them stay
      __syncthreads();
    }
  // ties go to the lower slots
  int over = 0, equal = 0;
  if (keep > 0)
    each([&](u64 k, int) {
      over += (k & mask) > prefix;
      equal += (k & mask) == prefix;
    });
  if (tid == 0) sGap = x.len;
  int all;
  const int eq0 = block_scan<PICK>(equal, &all);
  const int mine = max(0, min(equal, want - eq0));
  int at = block_scan<PICK>(over + (keep > 0 ? mine : 0), &all), left = mine, gap = x.len;
  if (keep > 0)
    each([&](u64 k, int j) {
      k &= mask;
      const bool tie = k == prefix && left > 0;
      left -= tie;
      if (k > prefix || tie) kept[at++] = j;
      else gap = min(gap, j);
    });
  else gap = 0;
  atomicMin(&sGap, gap);
  __syncthreads();
  if (tid == 0) e.cut[i] = Cut{x.seq, x.len, x.cap, keep, sGap, 0};
}

// Pages in place of shared ones that would be written to: entries in order,
// free pages lowest first. Where they do not last, the entry is not cut.
__global__ __launch_bounds__(PICK) void k_evict_pages(Ev e) {
  const PagedCache& c = e.d.c;
  __shared__ int sList[PICK];
  const int tid = threadIdx.x, lane = tid & 63;
  auto shared = [&](const Cut& x, int p) {
    const int id = c.table[(size_t)x.seq * c.max_pages + p];
    return (unsigned)id < (unsigned)c.n_pages && c.refs[id] > 1;
  };
  bool any = false;
  for (int i = tid >> 6; i < e.d.n; i += PICK / 64) {
    const Cut x = e.cut[i];
    if (x.seq < 0 || x.stay == x.len) continue;
    for (int p = (x.gap >> c.page_lg) + lane; p < (x.stay + c.page - 1) >> c.page_lg; p += 64) any = any || shared(x, p);
  }
  if (!__syncthreads_or(any)) return;
  const unsigned bits0 = free_bits(c, 0);
  int pos = 0;
  for (int i = 0; i < e.d.n; ++i) {
    const Cut x = e.cut[i];
    if (x.seq < 0 || x.stay == x.len) continue;
    const int p0 = x.gap >> c.page_lg, p1 = (x.stay + c.page - 1) >> c.page_lg;
    int32_t* to = e.fresh + (size_t)i * c.max_pages;
    int need = 0;
    for (int b = p0; b < p1; b += PICK) need += __syncthreads_count(b + tid < p1 && shared(x, b + tid));
    if (need == 0) continue;
    const int pos0 = pos;
    bool dry = false;
    for (int b = p0; b < p1 && !dry; b += PICK) {
      const bool is = b + tid < p1 && shared(x, b + tid);
      int cnt;
      const int rank = block_scan<PICK>((int)is, &cnt);
      dry = take_free<PICK>(c, bits0, &pos, cnt, sList) < cnt;
      if (b + tid < p1) to[b + tid] = is && !dry ? sList[rank] : -1;
      __syncthreads();
    }
    if (dry) {
      pos = pos0;
      int32_t* kept = e.d.kept + (size_t)i * e.slots;
      for (int j = tid; j < x.len; j += PICK) kept[j] = j;
      if (tid == 0) {
        flag(c, PG_OUT);
        e.cut[i].stay = e.cut[i].gap = x.len;
      }
    } else {
      // (a page that is given out is behind every page that is looked at as shared)
      for (int p = p0 + tid; p < p1; p += PICK)
        if (to[p] >= 0) c.refs[to[p]] = 1;
      if (tid == 0) e.cut[i].fresh = need;
    }
    __syncthreads();
  }
}

// K or V of one layer and head of an entry, rows of `width` 16-byte chunks. A
// slot never moves up, so rows go by in order: a group is read whole before any
// of it is written, and the next group, whose rows lie behind all that this one
// writes, is on its way meanwhile (32 KB each). Bound by memory: 16 sequences,
// 28 layers of 8 heads of 128, 5.9 GB in 1.20 ms, 4.9 TB/s read and written; 8
// sequences of 18 layers of one head of 256, 177 MB in 36 us.
__device__ __forceinline__ void move_rows(const Ev& e, int i, const Cut& x, int lh, bool val, int width) {
  const PagedCache& c = e.d.c;
  const int tid = threadIdx.x, G = MOVE * U / width;  // rows of a group
  const int esz = c.dtype == DT_BF16 ? 2 : 4;
  __shared__ unsigned long long sFrom[2][MOVE * U / 4], sTo[2][MOVE * U / 4];
  const int32_t *kept = e.d.kept + (size_t)i * e.slots, *table = c.table + (size_t)x.seq * c.max_pages;
  const int32_t* fresh = x.fresh ? e.fresh + (size_t)i * c.max_pages : nullptr;
  // (the first page that is replaced takes its first slots as well)
  const int g0 = x.gap >> c.page_lg;
  const int begin = fresh && fresh[g0] >= 0 ? g0 << c.page_lg : x.gap;
  char* base = (char*)(val ? c.v : c.k);
  constexpr unsigned long long NONE = ~0ull;
  auto places = [&](int r0, int b) {
    for (int k = tid; k < G; k += MOVE) {
      const int r = r0 + k;
      unsigned long long from = NONE, to = 0;
      if (r < x.stay) {
        const int old = kept[r], pf = table[old >> c.page_lg], nw = fresh ? fresh[r >> c.page_lg] : -1;
        const int pt = nw >= 0 ? nw : table[r >> c.page_lg];
        if ((unsigned)pf < (unsigned)c.n_pages && (unsigned)pt < (unsigned)c.n_pages) {
          from = slot_elem(c, lh / c.nkv, pf, lh % c.nkv, old & (c.page - 1)) * esz;
          to = slot_elem(c, lh / c.nkv, pt, lh % c.nkv, r & (c.page - 1)) * esz;
        } else {
          flag(c, PG_OUT);
        }
      }
      sFrom[b][k] = from, sTo[b][k] = to;
    }
  };
  u32x4 v[2][U];
  auto read = [&](u32x4 (&w)[U], int b) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int at = tid + k * MOVE, row = at / width;
      const unsigned long long f = row < G ? sFrom[b][row] : NONE;
      if (f != NONE) w[k] = *(const u32x4*)(base + f + (at - row * width) * 16);
    }
  };
  auto write = [&](u32x4 (&w)[U], int b) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int at = tid + k * MOVE, row = at / width;
      if (row < G && sFrom[b][row] != NONE) *(u32x4*)(base + sTo[b][row] + (at - row * width) * 16) = w[k];
    }
  };
  if (begin >= x.stay) return;
  places(begin, 0);
  __syncthreads();
  read(v[0], 0);
  for (int r0 = begin;; r0 += 2 * G) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = r0 + k * G;
      const bool more = r + G < x.stay;
      if (more) places(r + G, k ^ 1);
      // (every wave's reads of this group are here before any is written)
#pragma unroll
      for (int j = 0; j < U; ++j) asm volatile("" : "+v"(v[k][j]));
      __syncthreads();
      if (more) read(v[k ^ 1], k ^ 1);
      write(v[k], k);
      if (!more) return;
      __syncthreads();  // (this group's places are used up)
    }
  }
}

// The weights of one layer and head likewise.
__device__ __forceinline__ void move_mass(const Ev& e, int i, const Cut& x, int lh) {
  const PagedCache& c = e.d.c;
  const int tid = threadIdx.x;
  const size_t row = (((size_t)(lh / c.nkv) * c.n_seqs + x.seq) * c.nkv + lh % c.nkv) * e.slots;
  const float* from = e.d.mass + row;
  float* to = e.d.mass_out + row;
  const int32_t* kept = e.d.kept + (size_t)i * e.slots;
  for (int r0 = from == to ? x.gap : 0; r0 < x.stay; r0 += MOVE * U) {
    float v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int r = r0 + tid + k * MOVE;
      v[k] = r < x.stay ? from[kept[r]] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) asm volatile("" : "+v"(v[k]));
    __syncthreads();
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int r = r0 + tid + k * MOVE;
      if (r < x.stay) to[r] = v[k];
    }
  }
  __syncthreads();
  for (int r = x.stay + tid; r < x.cap; r += MOVE) to[r] = 0.f;
}

__global__ __launch_bounds__(MOVE) void k_evict_move(Ev e, int width) {
  const int heads = e.d.c.layers * e.d.c.nkv, i = blockIdx.x / (3 * heads), k = blockIdx.x % (3 * heads);
  const Cut x = e.cut[i];
  if (x.seq < 0) return;
  if (k >= 2 * heads) move_mass(e, i, x, k - 2 * heads);
  else if (x.stay < x.len) move_rows(e, i, x, k >> 1, k & 1, width);
}

// Tables, lengths and holders, when everything has moved.
__global__ __launch_bounds__(256) void k_evict_done(Ev e) {
  const PagedCache& c = e.d.c;
  const int i = blockIdx.x;
  const Cut x = e.cut[i];
  if (x.seq < 0 || x.stay == x.len) return;
  const int p1 = (x.stay + c.page - 1) >> c.page_lg;
  for (int p = (x.gap >> c.page_lg) + threadIdx.x; p < x.cap >> c.page_lg; p += 256) {
    int32_t* t = c.table + (size_t)x.seq * c.max_pages + p;
    const int old = *t, nw = p < p1 && x.fresh ? e.fresh[(size_t)i * c.max_pages + p] : -1;
    if (p < p1 && nw < 0) continue;
    *t = nw;
    if ((unsigned)old < (unsigned)c.n_pages) atomicSub(c.refs + old, 1);
  }
  if (threadIdx.x == 0) {
    c.lens[x.seq] = x.stay;
    c.held[x.seq] = p1;
  }
}

size_t up16(size_t x) { return (x + 15) & ~(size_t)15; }
int slots_of(const PagedCache& c) { return c.max_pages << c.page_lg; }
int width_of(const PagedCache& c) { return c.hd * (c.dtype == DT_BF16 ? 2 : 4) / 16; }

}  // namespace

size_t evict_scratch(const PagedCache& c, int n) {
  return up16((size_t)n * sizeof(Cut)) + up16((size_t)n * c.max_pages * 4) + (size_t)n * slots_of(c) * 8;
}

// Workgroups that move an entry: K, V and the weights of every layer and head.
static long long movers(const PagedCache& c) { return 3ll * c.layers * c.nkv; }
bool evict_fits(const PagedCache& c, int n) { return launchable(n * movers(c), MOVE) && n <= 65535; }

hipError_t launch_pages_evict(const EvictDesc& d, hipStream_t st) {
  const PagedCache& c = d.c;
  Ev e{d};
  e.slots = slots_of(c);
  char* p = (char*)d.scratch;
  e.cut = (Cut*)p;
  p += up16((size_t)d.n * sizeof(Cut));
  e.fresh = (int32_t*)p;
  p += up16((size_t)d.n * c.max_pages * 4);
  e.score = (double*)p;
  // (each works on what the one before left)
  hipError_t err;
  hipLaunchKernelGGL(k_evict_score, dim3((e.slots + 255) / 256, d.n), dim3(256), 0, st, e);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  hipLaunchKernelGGL(k_evict_pick, dim3(d.n), dim3(PICK), 0, st, e);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  hipLaunchKernelGGL(k_evict_pages, dim3(1), dim3(PICK), 0, st, e);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  hipLaunchKernelGGL(k_evict_move, dim3((unsigned)(d.n * movers(c))), dim3(MOVE), 0, st, e, width_of(c));
  if ((err = hipGetLastError()) != hipSuccess) return err;
  hipLaunchKernelGGL(k_evict_done, dim3(d.n), dim3(256), 0, st, e);
  return hipGetLastError();
}

}  // namespace vla
