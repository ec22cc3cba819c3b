// Internal interface between the host runtime and the kernels of the paged
// KV cache. Not part of the C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vla {

// A paged cache (vla_pages of the ABI, checked) and a batch of rows over it.
struct PagedCache {
  int dtype = 0;  // DT_F32 or DT_BF16
  int layers = 0, nkv = 0, hd = 0;
  int page = 0, page_lg = 0;  // slots of a page and its logarithm
  int n_pages = 0, n_seqs = 0, max_pages = 0;
  void* k = nullptr;  // [layers][n_pages][nkv][page][hd]
  void* v = nullptr;
  int32_t* table = nullptr;  // [n_seqs][max_pages], -1: no page
  int32_t* lens = nullptr;   // [n_seqs] committed slots
  int32_t* held = nullptr;   // [n_seqs] pages in the table
  int32_t* refs = nullptr;   // [n_pages] sequences that hold the page; 0: free
  int32_t* status = nullptr;
};
struct PagedRows {
  int n_rows = 0, n_ent = 0;
  const int32_t* start = nullptr;  // [n_ent + 1]
  const int32_t* seqs = nullptr;   // [n_ent] or null
};

// A grid holds fewer than 2^32 threads in each direction. What the launches
// below return where they would need more: a value that the runtime has no
// meaning for, so that its own errors stay apart from it.
inline bool launchable(long long wgs, int threads) { return wgs * threads < (1ll << 32); }
constexpr hipError_t GRID_FULL = (hipError_t)2000;

// status bits
enum { PG_OUT = 1, PG_BAD = 2 };

struct RopeNormDesc {
  PagedCache c;
  PagedRows r;
  int layer = 0, nq = 0;
  const void *q = nullptr, *k = nullptr, *v = nullptr;
  long long ldq = 0, ldk = 0, ldv = 0, ldo = 0;
  void* q_out = nullptr;
  const float *q_gain = nullptr, *k_gain = nullptr;
  int gain_plus_one = 0;
  float eps = 0.f;
  const float *cs = nullptr, *sn = nullptr;  // [n_pos][rot / 2]
  int n_pos = 0, rot = 0;
  const int32_t* pos = nullptr;
};
bool rope_norm_fits(const RopeNormDesc& d);  // (a grid holds it)
hipError_t launch_rope_norm(const RopeNormDesc& d, hipStream_t st);

struct TreeAttnDesc {
  PagedCache c;
  PagedRows r;
  int layer = 0, nq = 0;
  const void* q = nullptr;
  void* out = nullptr;
  long long ldq = 0, ldo = 0;
  const uint32_t* mask = nullptr;  // [n_rows][mask_words] or null: causal
  int mask_words = 0;
  float scale = 0.f;
  void* scratch = nullptr;
  int cus = 256;
};
size_t tree_attn_scratch(const TreeAttnDesc& d);
hipError_t launch_tree_attn(const TreeAttnDesc& d, hipStream_t st);

hipError_t launch_pages_init(const PagedCache& c, hipStream_t st);
hipError_t launch_pages_reserve(const PagedCache& c, const PagedRows& r, hipStream_t st);
bool fork_fits(const PagedCache& c, int n);
hipError_t launch_pages_fork(const PagedCache& c, int n, const int32_t* src, const int32_t* dst, int32_t* made,
                             hipStream_t st);
hipError_t launch_pages_commit(const PagedCache& c, const PagedRows& r, const int32_t* kept, const int32_t* n_kept,
                               hipStream_t st);
hipError_t launch_pages_release(const PagedCache& c, int n, const int32_t* seqs, hipStream_t st);

// The prefix rows 0 .. rows - 1 of a context (K and V in the KV-cache layout,
// nb 32-key blocks per KV head, layers lk / lv elements apart) to the slots
// behind sequence seq's committed ones, in every layer.
hipError_t launch_ctx_to_pages(const PagedCache& c, const void* k, const void* v, size_t lk, size_t lv, int nb,
                               int rows, int seq, hipStream_t st);

}  // namespace vla
