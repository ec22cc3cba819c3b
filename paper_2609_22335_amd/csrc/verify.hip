// Verification of drafted tokens against a target's probabilities. An entry's
// walk is one workgroup's: which child of a node is kept hangs on one number of
// the target (and one of the draft's) each, and only where a child is refused,
// or the walk ends, does a row of probabilities have to be read whole.
#include <algorithm>

#include "paged_dev.h"

namespace vla {
using namespace pg;

namespace {

constexpr int VT = 1024, VW = VT / 64;  // threads and waves of a walk
constexpr int PARTS = 64, PT = 256;      // parts of a row that more workgroups than one go through, and their threads
constexpr int ROWS = 512;               // drafts whose numbers are fetched at a time
constexpr int GONE = 64;                // refused tokens of a node that the LDS holds

template <typename T>
__device__ __forceinline__ float value(const T* p) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)*p << 16);
  else return *p;
}

// A probability as it counts: 0 where it is negative or not a number. (Where
// max(p - S q, 0) is worked out q alone needs it: that is 0 for every such p.)
__device__ __forceinline__ float some(float x) { return fmaxf(x, 0.f); }

// A row's elements t0 .. t0 + VEC - 1, t0 from -VEC + 1 on: one load where all
// of them are the row's and aligned; others are 0.
template <typename T>
__device__ __forceinline__ void load_some(const T* row, int t0, int V, bool aligned, float (&x)[El<T>::VEC]) {
  constexpr int N = El<T>::VEC;
  if (aligned && t0 >= 0 && t0 + N <= V) {
    unpack(*(const u32x4*)(row + t0), x);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = t0 + i >= 0 && t0 + i < V ? value(row + t0 + i) : 0.f;
  }
}

// What is left of a node's target: max(p - sub q, 0) (drafts drawn from q, of
// which a negative one or NaN is 0), or p without the tokens that were refused
// (drafts chosen without chance).
template <typename T>
struct Left {
  const T *p, *q;  // q null: `gone` counts
  int V;
  double sub;
  const int *gone, *more;  // the first GONE refused tokens, and all others
  int n_gone;
  bool qa;   // q's row lies as p's does, so that both are loaded in groups
  int skew;  // elements by which p's row is behind 16 bytes

  __device__ __forceinline__ void set(const T* p_, const T* q_, int V_) {
    constexpr int N = El<T>::VEC;
    p = p_, q = q_, V = V_;
    sub = 0, n_gone = 0;
    skew = (int)(((uintptr_t)p / sizeof(T)) % N);
    qa = q && ((uintptr_t)q / sizeof(T)) % N == (unsigned)skew;
  }
  __device__ __forceinline__ int refused(int j) const { return j < GONE ? gone[j] : more[j]; }
  // groups of VEC elements; group k has elements VEC k - skew on
  __device__ __forceinline__ int groups() const { return (V + skew + El<T>::VEC - 1) / El<T>::VEC; }
  // groups first .. last - 1 can be loaded whole
  __device__ __forceinline__ int first() const { return skew > 0; }
  __device__ __forceinline__ int last() const { return !q || qa ? (V + skew) / El<T>::VEC : 0; }
  __device__ __forceinline__ void rest(int t0, const float (&x)[El<T>::VEC], const float (&y)[El<T>::VEC],
                                       double (&r)[El<T>::VEC]) const {
    constexpr int N = El<T>::VEC;
    if (q) {
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = fmax((double)x[i] - sub * (double)some(y[i]), 0.0);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = fmax((double)x[i], 0.0);
      for (int j = 0; j < n_gone; ++j) {
        const int at = refused(j) - t0;
        if ((unsigned)at < (unsigned)N) {
#pragma unroll
          for (int i = 0; i < N; ++i) r[i] = at == i ? 0.0 : r[i];
        }
      }
    }
  }
  __device__ __forceinline__ void get(int k, double (&r)[El<T>::VEC]) const {
    constexpr int N = El<T>::VEC;
    const int t0 = k * N - skew;
    float x[N], y[N];
    load_some(p, t0, V, true, x);
    if (q) load_some(q, t0, V, qa, y);
    rest(t0, x, y, r);
  }
  // the sum of the groups that this lane has of k0 .. k1 - 1
  __device__ __forceinline__ double sum(int k0, int k1) const {
    constexpr int N = El<T>::VEC, U = sizeof(T) == 4 ? 3 : 2;
    const int lane = threadIdx.x & 63, a = max(k0, first()), b = min(k1, last());
    double s[2] = {0, 0};
    auto add = [&](const double (&r)[N]) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i & 1] += r[i];
    };
    int k = k0;
    if (a < b) {
      if (k0 + lane < a) {
        double r[N];
        get(k0 + lane, r);
        add(r);
      }
      k = a;
      // (the next loads are out while these are added up)
      u32x4 u[2][U], w[2][U];
      auto fetch = [&](int at, int e) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int t0 = (at + 64 * i + lane) * N - skew;
          u[e][i] = *(const u32x4*)(p + t0);
          if (q) w[e][i] = *(const u32x4*)(q + t0);
        }
      };
      auto work = [&](int at, int e) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          float x[N], y[N];
          double r[N];
          unpack(u[e][i], x);
          if (q) unpack(w[e][i], y);
          rest((at + 64 * i + lane) * N - skew, x, y, r);
          add(r);
        }
      };
      if (k + 64 * U <= b) fetch(k, 0);
      while (k + 64 * U <= b) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool more = k + 128 * U <= b;
          if (more) fetch(k + 64 * U, e ^ 1);
          __builtin_amdgcn_sched_barrier(0);
          work(k, e);
          k += 64 * U;
          if (!more) break;
        }
      }
    }
    for (k += lane; k < k1; k += 64) {
      double r[N];
      get(k, r);
      add(r);
    }
    return s[0] + s[1];
  }
};

// Groups of one of `parts` parts.
__device__ __forceinline__ int part_of(int groups, int parts = VW) { return ((groups + parts - 1) / parts + 63) & ~63; }

// Sums over the wave by shifts inside rows of 16 lanes and broadcasts of their
// last ones, as wave_scan (an LDS round trip a step took 0.6 us each).
template <int CTRL, int ROWS>
__device__ __forceinline__ void sum_step(double& x) {
  const long long v = __builtin_bit_cast(long long, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  x += __builtin_bit_cast(double, (long long)(((unsigned long long)hi << 32) | lo));
}
__device__ __forceinline__ double scan_sum(double x) {  // inclusive over the lanes
  sum_step<0x111, 0xf>(x);
  sum_step<0x112, 0xf>(x);
  sum_step<0x114, 0xf>(x);
  sum_step<0x118, 0xf>(x);
  sum_step<0x142, 0xa>(x);
  sum_step<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ double wave_sum(double x) {
  const long long v = __builtin_bit_cast(long long, scan_sum(x));
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, 63), hi = __builtin_amdgcn_readlane((int)(v >> 32), 63);
  return __builtin_bit_cast(double, (long long)(((unsigned long long)hi << 32) | lo));
}
// of n <= 64 values, a lane to each
__device__ __forceinline__ double sum_of(const double* part, int n) {
  const int lane = threadIdx.x & 63;
  return wave_sum(lane < n ? part[lane] : 0.0);
}

// Sums of the groups [k0, k1), a wave to each of VW equal parts: into part[],
// and their sum (the same in every thread).
template <typename T>
__device__ __forceinline__ double sum_parts(const Left<T>& l, int k0, int k1, double* part) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int per = part_of(k1 - k0), a = k0 + wv * per, b = min(a + per, k1);
  const double s = wave_sum(a < b ? l.sum(a, b) : 0.0);
  __syncthreads();  // the last sums are read
  if (lane == 0) part[wv] = s;
  __syncthreads();
  return sum_of(part, VW);
}

// The first token whose running sum passes u times the total, whose `n` parts
// (at most PARTS) are in part[]: the part that holds it, a sixteenth of that
// while it has more groups than there are threads, and there element by element.
// -1 where the total is 0 or not finite. (Should roundings leave none, the last
// token with anything.)
template <typename T>
__device__ __forceinline__ int draw(const Left<T>& l, double u, double total, int n, double* part, int* out) {
  constexpr int N = El<T>::VEC;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if (!(total > 0) || !(total < INFINITY)) return -1;
  const double want = u * total;
  int k0 = 0, k1 = l.groups();
  double before = 0;
  auto choose = [&](int parts) {
    const int per = part_of(k1 - k0, parts);
    const double x = lane < parts ? part[lane] : 0.0, run = before + scan_sum(x);
    const unsigned long long some = __ballot(x > 0), past = __ballot(x > 0 && run > want);
    const int pick = past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : 0;
    const double below = __shfl(run - x, pick);
    k0 += pick * per;
    k1 = min(k0 + per, k1);
    before = below;
  };
  if (k1 > VT) choose(n);
  while (k1 - k0 > VT) {
    sum_parts(l, k0, k1, part);
    choose(VW);
  }
  // a group to a thread
  double r[N], s = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = 0;
  if (k0 + tid < k1) l.get(k0 + tid, r);
#pragma unroll
  for (int i = 0; i < N; ++i) s += r[i];
  double run = scan_sum(s);
  __syncthreads();
  if (lane == 63) part[wv] = run;
  if (tid == 0) out[0] = 0x7FFFFFFF, out[1] = -1;
  __syncthreads();
  run = before + (sum_of(part, wv) + (run - s));
  int hit = 0x7FFFFFFF, last = -1;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    run += r[i];
    const int t = (k0 + tid) * N - l.skew + i;
    if (r[i] > 0) {
      last = t;
      if (run > want && hit == 0x7FFFFFFF) hit = t;
    }
  }
  if (hit != 0x7FFFFFFF) atomicMin(&out[0], hit);
  if (last >= 0) atomicMax(&out[1], last);
  __syncthreads();
  return out[0] == 0x7FFFFFFF ? out[1] : out[0];
}

// The likeliest token of every row (the lowest, where several are); -1: none.
template <typename T>
__global__ __launch_bounds__(256) void k_likeliest(DraftsDesc d) {
  constexpr int N = El<T>::VEC;
  __shared__ float sV[4];
  __shared__ int sI[4];
  const int row = blockIdx.x, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const T* p = (const T*)d.probs + (size_t)row * d.ldp;
  const int skew = (int)(((uintptr_t)p / sizeof(T)) % N), groups = (d.vocab + skew + N - 1) / N;
  float best = -INFINITY;
  int at = 0x7FFFFFFF;
#pragma unroll 4
  for (int k = threadIdx.x; k < groups; k += 256) {
    float x[N];
    const int t0 = k * N - skew;
    load_some(p, t0, d.vocab, true, x);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (x[i] > best && t0 + i >= 0 && t0 + i < d.vocab) best = x[i], at = t0 + i;
  }
  auto join = [&](float v, int i) {
    if (v > best || (v == best && i < at)) best = v, at = i;
  };
#pragma unroll
  for (int s = 32; s; s /= 2) {
    const float v = __shfl_xor(best, s);
    const int i = __shfl_xor(at, s);
    join(v, i);
  }
  if (lane == 0) sV[wv] = best, sI[wv] = at;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) join(sV[w], sI[w]);
    d.best[row] = at == 0x7FFFFFFF ? -1 : at;
  }
}

// A walk up to the first sum over a row that it needs, by PARTS / 4 workgroups
// an entry, and that sum in parts.
struct Pre {
  double sum[PARTS];
  double sub;
  int node, count;
  int at;  // the draft to go on with (0: nothing of this counts)
  int n_gone, gone[GONE];
};

// The walk. Drafts come by in their order; one whose parent is the node that
// the walk is at is tried, and taken or refused. (A node's children stand
// behind it, so none is passed by.)
//
// One CU reads 50 GB/s from the HBM, so where rows are long and entries few,
// PARTS / 4 workgroups of four waves (PRE) walk an entry up to the first sum
// over a row that it needs and work out a part of it with each wave; the walk
// proper goes on from there. 64 chains over 131,072 tokens: 19 us (67 MB, 3.5
// TB/s) and 8 in turn, against 33 without; over 50,001 tokens a CU's pass takes 3
// us, no more than the second launch. Later sums of an entry are one CU's however
// long the rows are: eight trees of 24 to 40 drafts take 33 us over 50,001 tokens
// and 59 over 131,072.
template <typename T, int NT, bool PRE>
__global__ __launch_bounds__(NT) void k_verify(DraftsDesc d) {
  __shared__ int sPar[ROWS], sTok[ROWS];
  __shared__ float sU[ROWS], sP[ROWS], sQ[ROWS];
  __shared__ double sPart[PARTS];
  __shared__ int sGone[GONE], sOut[2];
  constexpr int WGS = PARTS / 4;
  const int e = PRE ? blockIdx.x / WGS : blockIdx.x, part = PRE ? blockIdx.x % WGS : 0, tid = threadIdx.x;
  // (as entry_of, without the sequence's state)
  const int seq = d.r.seqs ? d.r.seqs[e] : e, first = d.r.start[e], end = d.r.start[e + 1];
  if (seq < 0 || seq >= d.c.n_seqs) return;
  const int row0 = min(max(first, 0), d.r.n_rows), n = max(min(end, d.r.n_rows) - row0, 0);
  if (n == 0) {
    if (!PRE && tid == 0) d.n_kept[e] = 0, d.next[e] = -1;
    return;
  }
  const T *P = (const T*)d.probs + (size_t)row0 * d.ldp, *Q = (const T*)d.drafted;
  if (Q) Q += (size_t)row0 * d.ldq;
  const bool greedy = !d.uniform;
  int32_t *kept = d.kept + row0, *gone = d.best + row0;  // (not used for likeliest tokens then)
  Pre* pre = d.pre ? (Pre*)d.pre + e : nullptr;
  Left<T> left;
  left.gone = sGone, left.more = gone;
  int node = 0, count = 1, at = 1, parts = VW;
  double z = 1;         // what is left of the node's target
  bool summed = false;  // z is the sum of what is left, its parts in sPart
  bool odd = false;
  if (!PRE && pre && pre->at > 0) {
    node = pre->node, count = pre->count, at = pre->at;
    left.set(P + (size_t)node * d.ldp, Q ? Q + (size_t)node * d.ldq : nullptr, d.vocab);
    left.sub = pre->sub, left.n_gone = pre->n_gone;
    if (tid < PARTS) sPart[tid] = pre->sum[tid];
    if (tid < GONE) sGone[tid] = pre->gone[tid];
    __syncthreads();
    parts = PARTS, summed = true;
    z = sum_of(sPart, PARTS);
    if (!d.parent && n <= ROWS) at = n;  // (a chain's node has one draft, and all have been looked at)
  } else {
    left.set(P, Q, d.vocab);
    if (part == 0 && tid == 0) kept[0] = 0;
  }
  // Where no draft was refused (S is 0) all of the target is left, whatever q holds.
  auto untouched = [&] {
    if (!(left.sub > 0)) left.q = nullptr;
  };
  // PRE: this wave's part of what is left, and where the walk is
  auto leave = [&](int next) {
    untouched();
    const int wv = tid >> 6, mine = part * 4 + wv, groups = left.groups(), per = part_of(groups, PARTS);
    const int a = min(mine * per, groups), b = min(a + per, groups);
    const double s = wave_sum(a < b ? left.sum(a, b) : 0.0);
    if ((tid & 63) == 0) pre->sum[mine] = s;
    if (part == 0) {
      if (tid < left.n_gone) pre->gone[tid] = sGone[tid];
      if (tid == 0) pre->sub = left.sub, pre->node = node, pre->count = count, pre->at = next, pre->n_gone = left.n_gone;
    }
  };
  for (int c0 = at; c0 < n; c0 += ROWS) {
    const int m = min(ROWS, n - c0);
    __syncthreads();
    for (int k = tid; k < m; k += NT) {
      const int i = c0 + k, row = row0 + i;
      int par = d.parent ? d.parent[row] : i - 1;
      const int tok = d.tokens[row];
      if (par < 0 || par >= i) par = -1;
      const bool in = par >= 0 && tok >= 0 && tok < d.vocab;
      odd = odd || !in;
      sPar[k] = par;
      sTok[k] = in ? tok : -1;
      if (greedy) {
        sP[k] = in && d.best[row0 + par] == tok ? 1.f : 0.f;
      } else {
        sU[k] = d.uniform[row];
        sP[k] = in ? some(value(P + (size_t)par * d.ldp + tok)) : 0.f;
        sQ[k] = in && Q ? some(value(Q + (size_t)par * d.ldq + tok)) : 0.f;
      }
      if (part == 0 && (PRE || !pre || at == 1)) kept[i] = -1;
    }
    __syncthreads();
    for (int k = 0; k < m; ++k) {
      if (sPar[k] != node || sTok[k] < 0) continue;
      bool yes;
      double mine = 0;
      if (greedy) {
        yes = sP[k] > 0.f;
      } else if (Q) {
        mine = fmax((double)sP[k] - left.sub * (double)sQ[k], 0.0);
        yes = (double)sU[k] * (double)sQ[k] * z < mine;
      } else {
        mine = sP[k];
        for (int j = 0; j < left.n_gone; ++j) mine = left.refused(j) == sTok[k] ? 0.0 : mine;
        yes = (double)sU[k] * z < mine;
      }
      if (yes) {
        node = c0 + k;
        left.set(P + (size_t)node * d.ldp, Q ? Q + (size_t)node * d.ldq : nullptr, d.vocab);
        z = 1, summed = false;
        if (part == 0 && tid == 0) kept[count] = node;
        ++count;
      } else if (!greedy) {
        if (Q) {
          left.sub += z;
          if constexpr (PRE) {
            if (odd) flag(d.c, PG_BAD);
            leave(c0 + k + 1);
            // (drafts behind these rows are not kept either)
            if (part == 0)
              for (int i = c0 + m + tid; i < n; i += NT) kept[i] = -1;
            return;
          }
          z = sum_parts(left, 0, left.groups(), sPart);
          parts = VW, summed = true;
        } else if (mine > 0) {
          z -= mine;
          summed = false;
          if (PRE && left.n_gone == GONE) {  // (more than the LDS holds)
            if (part == 0 && tid == 0) pre->at = 0;
            return;
          }
          __syncthreads();
          if (tid == 0) {
            if (left.n_gone < GONE) sGone[left.n_gone] = sTok[k];
            else gone[left.n_gone] = sTok[k];
          }
          __syncthreads();
          ++left.n_gone;
        }
      }
    }
  }
  if constexpr (PRE) {
    if (odd) flag(d.c, PG_BAD);
    leave(n);
    return;
  }
  int token;
  if (greedy) {
    token = d.best[row0 + node];
  } else {
    const double u = d.uniform[row0];
    untouched();
    if (!summed) z = sum_parts(left, 0, left.groups(), sPart), parts = VW;
    token = draw(left, u, z, parts, sPart, sOut);
    if (token < 0 && (left.sub > 0 || left.n_gone)) {  // nothing is left: all of the target
      left.sub = 0, left.n_gone = 0, left.q = nullptr;
      z = sum_parts(left, 0, left.groups(), sPart);
      token = draw(left, u, z, VW, sPart, sOut);
    }
  }
  odd = odd || token < 0;
  if (odd) flag(d.c, PG_BAD);
  if (tid == 0) d.n_kept[e] = count, d.next[e] = token;
}

template <typename T>
hipError_t verify(const DraftsDesc& d, hipStream_t st) {
  if (!d.uniform && d.r.n_rows > 0) {
    hipLaunchKernelGGL(k_likeliest<T>, dim3(d.r.n_rows), dim3(256), 0, st, d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (d.pre) {
    hipLaunchKernelGGL((k_verify<T, PT, true>), dim3(d.r.n_ent * (PARTS / 4)), dim3(PT), 0, st, d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_verify<T, VT, false>), dim3(d.r.n_ent), dim3(VT), 0, st, d);
  return hipGetLastError();
}

}  // namespace

// Where PARTS / 4 workgroups to an entry begin the walk: rows too long for one CU, and
// CUs that would be idle.
static bool verify_pre(const DraftsDesc& d) { return d.vocab >= 65536 && d.r.n_ent <= 128; }
static size_t best_bytes(const DraftsDesc& d) { return ((size_t)d.r.n_rows * 4 + 15) & ~(size_t)15; }
size_t verify_scratch(const DraftsDesc& d) {
  return best_bytes(d) + (verify_pre(d) ? (size_t)d.r.n_ent * sizeof(Pre) : 0);
}
bool verify_fits(const DraftsDesc& d) { return launchable(d.r.n_rows, 256) && launchable(d.r.n_ent, VT); }

hipError_t launch_verify(const DraftsDesc& x, hipStream_t st) {
  if (x.r.n_ent <= 0) return hipSuccess;
  DraftsDesc d = x;
  d.best = (int32_t*)d.scratch;
  // (a batch without rows has entries to answer all the same, and no scratch)
  if (d.uniform && d.r.n_rows > 0 && verify_pre(d)) d.pre = (void*)((char*)d.scratch + best_bytes(d));
  return d.dtype == DT_BF16 ? verify<uint16_t>(d, st) : verify<float>(d, st);
}

}  // namespace vla
