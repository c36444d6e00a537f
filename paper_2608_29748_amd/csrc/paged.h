// Operators over the paged KV cache: appending rows, attention with a sliding window and
// sinks, attention of a batch whose sequences share a prefix.
#pragma once
#include "common.h"

namespace rt {

// One cache and the rows of a call, as the kernels see them.  Sequence s has the rows
// row_start[s] .. row_start[s + 1] - 1 (row_start null: rows_each rows each) and
// kv_len[s * kv_stride] + kv_add keys, its rows' own among them: row i is at position
// keys - rows + i.  Nothing on the device is trusted to be in range: rows are clamped to
// n_rows, keys to the page table's width, and pages outside [0, n_pages) hold no keys.
struct PagedRows {
  void* k; void* v;              // K pages [page][kv head][16][hd], V pages [page][kv head][hd][16]
  const int32_t* page_table;     // [n_seqs][max_pages]
  int max_pages, n_pages;
  int n_q_heads, n_kv_heads, head_dim;
  int n_seqs, n_rows, rows_each;
  const int32_t* row_start;
  const int32_t* kv_len; int kv_stride, kv_add;
};

struct AppendArgs {
  PagedRows r;
  const void* q; const void* ks; const void* vs;   // source rows, head h at column h * head_dim
  long ldq, ldk, ldv;
  void* q_out; long ldqo;                          // storage type; q null: no queries
  const float* cos; const float* sin;              // [position][rot_dim / 2]; null: no rotation
  int rot_dim;
  const void* q_norm; const void* k_norm; float eps;   // per-head RMSNorm weights (storage type), may be null
};
// T: storage type of the cache, S: type of the source rows (T or float).
template <typename T, typename S>
hipError_t paged_append(const AppendArgs& a, hipStream_t s);

struct PagedAttnArgs {
  PagedRows r;
  const void* q; long ldq;       // storage type, head h at column h * head_dim
  void* out; long ldo;           // the same; packed: GEMM-operand layout with group stride ldo
  int packed;
  float scale;
  int window, sinks;             // key j of the row at position p: j > p - window or j < sinks
  int prefix;                    // keys 0 .. prefix-1 lie in the same pages of every sequence (a
                                 // multiple of 16; those of sequence 0's table are read)
  int max_rows, max_kv;          // expected longest sequence of rows and of keys (choices only)
  float* part_o; float* part_ml; // split partials, see paged_attn.hip
};
// Key splits of a call.
struct PagedPlan {
  int splits;                    // of the sequences' own keys
  int shared;                    // of the shared prefix (0: no pass of its own)
  // partial results per row, those of the prefix first (0: rows are finished in one go)
  int parts() const { return shared || splits > 1 ? shared + splits : 0; }
  int launches() const { return parts() ? 2 : 1; }      // the passes, the merge
};
PagedPlan paged_plan(const PagedAttnArgs& a, int elem_bytes);
// The kernel of a call's passes (RT_A_KERNEL's values), with pages by non-temporal loads or not, and
// the workgroups of the prefix's pass and of the sequences' own.
struct PagedChoice { int kernel; bool streamed; long g0, g1; };
PagedChoice paged_choice(const PagedAttnArgs& a, const PagedPlan& p, int elem_bytes);
// Floats of part_o (returned) and part_ml.
size_t paged_part_floats(const PagedAttnArgs& a, const PagedPlan& p, size_t* ml);
// Launch i (0 .. p.launches() - 1, in order) of a call.
template <typename T>
hipError_t paged_launch(const PagedAttnArgs& a, const PagedPlan& p, int i, hipStream_t s);

constexpr long kMaxGrid = 0xffffffffl / 256;      // workgroups of a launch: 32 bits count its threads

#ifdef __HIPCC__
// Rows a .. a + n - 1 and key count of sequence s, as clamped.
struct SeqRows { int a, n, keys; };
__device__ __forceinline__ SeqRows seq_rows(const PagedRows& r, int s) {
  SeqRows q;
  if (r.row_start) {
    q.a = min(max(r.row_start[s], 0), r.n_rows);
    q.n = min(max(r.row_start[s + 1], q.a), r.n_rows) - q.a;
  } else {
    q.a = s * r.rows_each;
    q.n = r.rows_each;
  }
  q.keys = r.kv_len[(size_t)s * r.kv_stride] + r.kv_add;
  return q;
}
// Sequence of row t (n_seqs: none), for every lane of a wave the same t: the number of
// sequences whose rows end at or before t.
__device__ __forceinline__ int row_seq(const PagedRows& r, int t) {
  if (!r.row_start) return t / r.rows_each;
  const int lane = threadIdx.x & 63;
  int s = 0;
  for (int s0 = 0; s0 < r.n_seqs; s0 += 64)
    s += (int)__popcll(__ballot(s0 + lane < r.n_seqs && r.row_start[min(s0 + lane, r.n_seqs - 1) + 1] <= t));
  return s;
}
// Item `blk` of the sequences' items laid end to end, f(s) of them for sequence s: item `in` of
// sequence s (false: there are fewer).  All 64 lanes must be active.
template <typename F>
__device__ __forceinline__ bool find_block(int n_seqs, int blk, F&& f, int& s, int& in) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int s0 = 0; s0 < n_seqs; s0 += 64) {
    int inc = s0 + lane < n_seqs ? f(s0 + lane) : 0;
    const int own = inc;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int t = __shfl_up(inc, o, 64);
      if (lane >= o) inc += t;
    }
    const unsigned long long m = __ballot(base + inc > blk);
    if (m) {
      const int l = __builtin_ctzll(m);
      s = s0 + l;
      in = blk - base - __builtin_amdgcn_readlane(inc - own, l);
      return (unsigned)in < (unsigned)__builtin_amdgcn_readlane(own, l);   // (not of sums past 32 bits)
    }
    base += __builtin_amdgcn_readlane(inc, 63);
  }
  return false;
}
#endif

}  // namespace rt
