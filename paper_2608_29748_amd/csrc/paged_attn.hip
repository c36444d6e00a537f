// Attention over the paged KV cache with a sliding window and sinks, and of batches whose
// sequences share a prefix.
//
// For the row at position p of a sequence, with s_j = scale q . k_j over its visible keys,
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   m = max_j s_j  (zeros: no visible key).
// The keys are walked once with a running maximum and sum; several walks over parts of the
// keys (waves, key splits, the shared prefix) are joined by the same rule, each weighted with
// exp(its maximum - the largest).
//
// Visible keys of a row: [lo, hi) and the sinks [0, snk), snk <= lo:
//   window      hi = p + 1, lo = p - window + 1, snk = sinks
//   prefix      where it pays, keys [0, prefix) in a pass over the rows of all sequences, whose
//               tiles so fill with rows that read the same pages, and beside it [prefix, p]
//               sequence by sequence; a merge joins them.
#include "../../include/retrace.h"
#include "paged.h"

namespace rt {

typedef __attribute__((address_space(4))) const int32_t const_i32_t;

constexpr int kStep = 32;                  // keys per step of a wave: two pages
constexpr int kMaxParts = 32;              // key splits of a pass, where the other may have as many
constexpr int kMaxMerge = 64;              // partial results of a row: one a lane of the merge
constexpr float kMrefInit = -1.0e30f;      // running maximum before any visible key (log2 units)

// A pass of a call: over the shared prefix, or over the sequences' own keys (all of them where no
// pass is made over the prefix).  Both go out in one launch, the prefix's workgroups first.
struct PagedPass {
  int shared;       // 1: the rows of all sequences over the prefix
  int first;        // key from which on the sequences' own pass works (0, or the prefix)
  int splits;
  int z0;           // partial results go to parts z0 .. z0 + splits - 1; -1: rows are finished here
  int groups;       // workgroups
};

struct RowRange { int lo, hi, snk; };
__device__ __forceinline__ RowRange row_range(const PagedAttnArgs& a, const PagedPass& ps, long pos) {
  const long cap = (long)a.r.max_pages * kPage;
  const long hi = max(0l, min(pos + 1, ps.shared ? min(cap, (long)a.prefix) : cap));
  long lo = ps.first;
  if (a.window > 0) lo = max(lo, pos - a.window + 1);
  lo = min(max(lo, 0l), hi);
  return RowRange{(int)lo, (int)hi, (int)min((long)a.sinks, lo)};
}

// Steps of STEP keys over the keys [0, snk) and [lo, hi), those of the sinks first.
template <int STEP>
struct Steps {
  int n_snk, first, n;
  __device__ __forceinline__ Steps(int snk, int lo, int hi) {
    const int last = (hi + STEP - 1) / STEP;
    first = min(lo / STEP, last);
    n_snk = min((snk + STEP - 1) / STEP, first);
    n = n_snk + last - first;
  }
  __device__ __forceinline__ int key(int i) const { return (i < n_snk ? i : first + (i - n_snk)) * STEP; }
};

// What the row (of the call) tok sees; sr: its sequence, where the block has one.
__device__ __forceinline__ RowRange lane_range(const PagedAttnArgs& a, const PagedPass& ps, const SeqRows& sr, int tok) {
  const PagedRows& r = a.r;
  SeqRows q = sr;
  if (ps.shared) {
    int sq = tok;
    if (r.row_start) {            // the last sequence that starts at or before the row
      int b = 0, e = r.n_seqs;
      while (e - b > 1) {
        const int m = (b + e) >> 1;
        if (r.row_start[m] <= tok) b = m; else e = m;
      }
      sq = b;
    } else {
      sq = tok / r.rows_each;
    }
    q = seq_rows(r, sq);
    if (tok < q.a || tok >= q.a + q.n) return RowRange{0, 0, 0};     // a row of no sequence
  }
  return row_range(a, ps, (long)q.keys - q.n + (tok - q.a));
}
// Which of the eight keys from key b on a row does not see, a bit each; and the score of key x of
// such a set, minus infinity where its bit is set.
__device__ __forceinline__ uint32_t hidden8(const RowRange& r, int b) {
  auto below = [&](int x) { return (1u << min(max(x - b, 0), 8)) - 1; };
  return 0xffu & ~(below(r.hi) & (~below(r.lo) | below(r.snk)));
}
__device__ __forceinline__ float hide(float s, uint32_t hidden, int x) {
  const uint32_t m = (uint32_t)((int)(hidden << (31 - x)) >> 31);
  return __uint_as_float((m & 0xff800000u) | (~m & __float_as_uint(s)));
}
// Whether any element that the wave holds is infinite or NaN: the largest exponent, by integer maxima.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
struct Finite {
  u16x2 top16 = {0, 0};
  uint32_t top32 = 0;
  __device__ __forceinline__ void add(const Frag<bf16_t>& f) { add(f.v); }
  __device__ __forceinline__ void add(const bf16x8& v) {
    const u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) top16 = __builtin_elementwise_max(top16, __builtin_bit_cast(u16x2, u[i] & 0x7fff7fffu));
  }
  __device__ __forceinline__ void add(const Frag<float>& f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top32 = max(top32, __float_as_uint(f.get(i)) & 0x7fffffffu);
  }
  __device__ __forceinline__ bool all() const {
    return __ballot(max(top16[0], top16[1]) >= 0x7f80 || top32 >= 0x7f800000u) == 0;
  }
};
// Sequence and row block of block blk, of `per` (token, head) rows each; false: none.  A sequence's
// last rows come first: they see the most keys, and short blocks fill the end of a launch (causal prompts, 32 heads
// over 8 of 128: 4096 tokens 243 -> 219 us, 4 of 2048 247 -> 231).  The results are the same for every lane and
// made scalar, so that page ids come by scalar loads.
__device__ __forceinline__ bool block_rows(const PagedAttnArgs& a, bool shared, int blk, int per, int& s, int& rb,
                                           SeqRows& sr) {
  const PagedRows& r = a.r;
  const int G = r.n_q_heads / r.n_kv_heads;
  int s_ = 0, rb_ = blk;
  SeqRows q{0, r.n_rows, 0};
  if (!shared) {
    if (r.row_start) {
      if (!find_block(r.n_seqs, blk, [&](int i) { return (seq_rows(r, i).n * G + per - 1) / per; }, s_, rb_)) return false;
    } else {
      const int n = (r.rows_each * G + per - 1) / per;
      s_ = blk / n;
      rb_ = blk % n;
    }
    q = seq_rows(r, __builtin_amdgcn_readfirstlane(s_));
    rb_ = (q.n * G + per - 1) / per - 1 - rb_;
  }
  s = __builtin_amdgcn_readfirstlane(s_);
  rb = __builtin_amdgcn_readfirstlane(rb_);
  sr = SeqRows{__builtin_amdgcn_readfirstlane(q.a), __builtin_amdgcn_readfirstlane(q.n),
               __builtin_amdgcn_readfirstlane(q.keys)};
  return true;
}

// The pages of sequence s (the same for every lane; scalar loads for scalar indexes): those of the
// shared prefix through the first sequence's row of the table.
struct TableRow {
  const_i32_t* own;
  const_i32_t* first;
  int n_first;
  __device__ __forceinline__ TableRow(const PagedAttnArgs& a, int s) {
    const uint64_t p = (uint64_t)(a.r.page_table + (size_t)s * a.r.max_pages);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
    own = (const_i32_t*)((uint64_t)hi << 32 | lo);
    first = (const_i32_t*)a.r.page_table;
    n_first = a.prefix / kPage;
  }
  __device__ __forceinline__ int page(int j) const { return (j < n_first ? first : own)[j]; }
};
// wave-wide integer reductions of the ROCm device library (DPP based), in a scalar register
extern "C" __device__ int __ockl_wfred_min_i32(int);
extern "C" __device__ int __ockl_wfred_max_i32(int);
__device__ __forceinline__ int wave_min(int v) { return __builtin_amdgcn_readfirstlane(__ockl_wfred_min_i32(v)); }
__device__ __forceinline__ int wave_max(int v) { return __builtin_amdgcn_readfirstlane(__ockl_wfred_max_i32(v)); }

// Rows kernel: one workgroup of NW waves per block of 16 NT (token, head) rows, KV head and key
// split.  Every wave takes every NW-th step of 32 keys of the split straight from memory into
// registers in MFMA operand order (S^T = K Q^T, O^T = V^T P^T; the K rows of a 16-row tile are
// the keys 8(r/4) + 4 tile + r%4, so that a lane ends up with eight consecutive keys of its
// query, whose V^T fragment is one contiguous read); the waves' results meet in LDS.  Bound by
// memory: two waves per SIMD with one step of 16 KB (bf16, head_dim 128) each under way, and pages
// that only this workgroup reads come by non-temporal loads (NTL).  64 steps over 4100 keys, 40 heads
// (1.08 GB): 165 us (6.5 TB/s); with plain loads 185, with three waves per SIMD 197, with a second set
// of registers for the next step's keys 208.
template <int HD, int NT, int NW>
struct RowsLds {
  float o[NW][16 * NT][HD + 4];                            // results of the waves
  float ml[NW][16 * NT][2];
  float p[NW][kStep][16];                                  // one tile's weights (non-finite V only)
};
template <typename T, int HD, int NT, int NW, bool NTL>
__device__ __forceinline__ void rows_body(const PagedAttnArgs& a, const PagedPass& ps, int group, RowsLds<HD, NT, NW>& lds) {
  constexpr int NHT = HD / 16, NKS = HD / 32;
  constexpr int RB = 16 * NT;
  auto& sO = lds.o;
  auto& sML = lds.ml;
  auto& sP = lds.p;
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 63, g4 = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = group % r.n_kv_heads, split = group / r.n_kv_heads % ps.splits;
  const int blk = group / (r.n_kv_heads * ps.splits);
  const int G = r.n_q_heads / r.n_kv_heads;
  int s, rb;
  SeqRows sr;
  if (!block_rows(a, ps.shared, blk, RB, s, rb, sr)) return;
  const int nrows = sr.n * G, row0 = rb * RB;
  if (row0 >= nrows) return;

  // this lane's rows and what they see
  RowRange rg[NT];
  Frag<T> qf[NT][NKS];
  int all_lo = 0x7fffffff, all_hi = 0, all_snk = 0, min_hi = 0x7fffffff, max_lo = 0, min_snk = 0x7fffffff;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int rr = min(row0 + t * 16 + c16, nrows - 1);
    const int tok = sr.a + rr / G;
    rg[t] = lane_range(a, ps, sr, tok);
    const T* qp = (const T*)a.q + (size_t)tok * a.ldq + (size_t)(kvh * G + rr % G) * HD;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[t][ks].load(qp + ks * 32 + g4 * 8);
    all_lo = min(all_lo, rg[t].lo);
    max_lo = max(max_lo, rg[t].lo);
    all_hi = max(all_hi, rg[t].hi);
    min_hi = min(min_hi, rg[t].hi);
    all_snk = max(all_snk, rg[t].snk);
    min_snk = min(min_snk, rg[t].snk);
  }
  all_lo = wave_min(all_lo);
  max_lo = wave_max(max_lo);
  all_hi = wave_max(all_hi);
  min_hi = wave_min(min_hi);
  all_snk = wave_max(all_snk);
  min_snk = wave_min(min_snk);
  const Steps<kStep> st(all_snk, all_lo, all_hi);
  const int per = (st.n + ps.splits - 1) / ps.splits;
  const int i_beg = split * per + w, i_end = min(st.n, (split + 1) * per);
  const int n = i_end > i_beg ? (i_end - i_beg + NW - 1) / NW : 0;      // this wave's steps

  const TableRow pt(a, s);
  const int last_page = max(0, (all_hi - 1) / kPage);
  const float sl2 = a.scale * 1.4426950408889634f;
  float mref[NT], lsum[NT];
  f32x4 o[NT][NHT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    mref[t] = kMrefInit;
    lsum[t] = 0.f;
#pragma unroll
    for (int h = 0; h < NHT; ++h) o[t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const size_t PE = (size_t)kPage * HD;
  const int ko = (8 * ((c16 >> 2) & 1) + (c16 & 3)) * HD + g4 * 8, vo = c16 * kPage + (g4 & 1) * 8;
  struct Keys {
    Frag<T> k[2][NKS], v[NHT];
    size_t b0, b1;                      // the two pages
    int k0;
    bool ok0, ok1;
  };
  // page ids of 32 steps at a time, a lane each
  int ids = 0;
  auto fetch = [&](Keys& f, int t) {    // this wave's step t
    if ((t & 31) == 0) ids = pt.page(min(st.key(i_beg + min(t + (lane >> 1), n - 1) * NW) / kPage + (lane & 1), last_page));
    const int p0 = __builtin_amdgcn_readlane(ids, 2 * (t & 31)), p1 = __builtin_amdgcn_readlane(ids, 2 * (t & 31) + 1);
    f.k0 = st.key(i_beg + t * NW);
    f.ok0 = p0 >= 0 && p0 < r.n_pages;
    f.ok1 = p1 >= 0 && p1 < r.n_pages;
    f.b0 = ((size_t)(f.ok0 ? p0 : 0) * r.n_kv_heads + kvh) * PE;
    f.b1 = ((size_t)(f.ok1 ? p1 : 0) * r.n_kv_heads + kvh) * PE;
    const T* kp = (const T*)r.k + ((c16 >> 3) ? f.b1 : f.b0) + ko;
    const T* vp = (const T*)r.v + ((g4 >> 1) ? f.b1 : f.b0) + vo;
#pragma unroll
    for (int ta = 0; ta < 2; ++ta)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        if constexpr (NTL) f.k[ta][ks].load_stream(kp + ta * 4 * HD + ks * 32);
        else f.k[ta][ks].load(kp + ta * 4 * HD + ks * 32);
      }
#pragma unroll
    for (int h = 0; h < NHT; ++h) {
      if constexpr (NTL) f.v[h].load_stream(vp + h * 16 * kPage);
      else f.v[h].load(vp + h * 16 * kPage);
    }
  };
  auto use = [&](Keys& f) {
    const int k0 = f.k0;
    const bool whole = f.ok0 && f.ok1 && k0 + kStep <= min_hi && (k0 >= max_lo || k0 + kStep <= min_snk);
    // keys (of the 32) with a non-finite V element somewhere: a weight of zero must not meet
    // them in a product, so where rows differ in what they see they are added one by one
    uint32_t bad = 0;
    if (!whole) {
      Finite fin;
#pragma unroll
      for (int h = 0; h < NHT; ++h) fin.add(f.v[h]);
      if (!fin.all()) {
        uint32_t mine = 0;
#pragma unroll
        for (int h = 0; h < NHT; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) mine |= (__builtin_isfinite(f.v[h].get(e)) ? 0u : 1u) << e;
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) mine |= __shfl_xor((int)mine, x, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (mine >> e & 1)
#pragma unroll
            for (int h = 0; h < NHT; ++h) f.v[h].set(e, 0.f);
#pragma unroll
        for (int x = 0; x < 4; ++x) bad |= (uint32_t)__builtin_amdgcn_readlane((int)mine, 16 * x) << (8 * x);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4 sc[2];
      sc[0] = sc[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        mma(sc[0], f.k[0][ks], qf[t][ks]);
        mma(sc[1], f.k[1][ks], qf[t][ks]);
      }
      if (!whole) {
        const uint32_t hid = (g4 < 2 ? f.ok0 : f.ok1) ? hidden8(rg[t], k0 + 8 * g4) : 0xffu;
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] = hide(sc[e >> 2][e & 3], hid, e);
      }
      float mx = sc[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = __builtin_elementwise_maximum(mx, sc[e >> 2][e & 3]);
      mx = group4_max(mx) * sl2;
      // the reference is raised only when a score exceeds it by more than 2^8
      if (__ballot(mx > mref[t] + 8.f)) {
        const float mn = fmaxf(mref[t], mx), al = __builtin_amdgcn_exp2f(mref[t] - mn);
#pragma unroll
        for (int h = 0; h < NHT; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][h][e] *= al;
        lsum[t] *= al;
        mref[t] = mn;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(sc[e >> 2][e & 3], sl2, -mref[t]));
        lsum[t] += p[e];
      }
      // weights of 16 bits: the rounding of each and the rounding of what that left over, two
      // products, 2^-16 of the weight (the matrix units have nothing else to do while the keys come in)
      Frag<T> ph, pl;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ph.set(e, p[e]);
        if constexpr (sizeof(T) == 2) pl.set(e, p[e] - ph.get(e));
      }
#pragma unroll
      for (int h = 0; h < NHT; ++h) {
        mma(o[t][h], f.v[h], ph);
        if constexpr (sizeof(T) == 2) mma(o[t][h], f.v[h], pl);
      }
      if (bad) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sP[w][8 * g4 + e][c16] = p[e];
        wait_lds();
        for (uint32_t m = bad; m; m &= m - 1) {
          const int j = __builtin_ctz(m);
          const float pj = *(volatile float*)&sP[w][j][c16];
          const T* vj = (const T*)r.v + (j < 16 ? f.b0 : f.b1) + (j & 15) + (size_t)(4 * g4) * kPage;
#pragma unroll
          for (int h = 0; h < NHT; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[t][h][e] += pj != 0.f ? pj * Elem<T>::to_f32(vj[(h * 16 + e) * kPage]) : 0.f;
        }
      }
    }
  };
  for (int t = 0; t < n; ++t) {
    Keys f;
    fetch(f, t);
    use(f);
  }
  // join the waves: thread i takes eight elements of a row
  constexpr int RUNS = HD / 8;
  static_assert(RB * RUNS <= 64 * NW, "a thread per item");
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float l = group4_sum(lsum[t]);
#pragma unroll
    for (int h = 0; h < NHT; ++h)
      *reinterpret_cast<f32x4*>(&sO[w][t * 16 + c16][h * 16 + 4 * g4]) = o[t][h];
    if (g4 == 0) {
      sML[w][t * 16 + c16][0] = mref[t];
      sML[w][t * 16 + c16][1] = l;
    }
  }
  __syncthreads();
  const int items = min(RB, nrows - row0) * RUNS;
  const size_t zst = (size_t)r.n_rows * r.n_q_heads;
  if ((int)threadIdx.x >= items) return;
  const int it = threadIdx.x;
  const int rl = it / RUNS, d = it % RUNS * 8, rr = row0 + rl;
  const int tok = sr.a + rr / G, h = kvh * G + rr % G;
  const size_t rh = (size_t)tok * r.n_q_heads + h;
  float M = sML[0][rl][0], L = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 1; u < NW; ++u) M = fmaxf(M, sML[u][rl][0]);
#pragma unroll
  for (int u = 0; u < NW; ++u) {
    const float f = __builtin_amdgcn_exp2f(sML[u][rl][0] - M);
    L += f * sML[u][rl][1];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += f * sO[u][rl][d + e];
  }
  if (ps.z0 >= 0) {
    const size_t row = (ps.z0 + split) * zst + rh;
    float* op = a.part_o + row * HD + d;
    *reinterpret_cast<float4*>(op) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(op + 4) = make_float4(v[4], v[5], v[6], v[7]);
    *reinterpret_cast<float2*>(a.part_ml + row * 2) = make_float2(M, L);      // (the same from every lane of the row)
    return;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;       // (NaN stays NaN)
  Frag<T> f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f.set(e, L == 0.f ? 0.f : v[e] * inv);
  const size_t at = a.packed ? pa_index(tok, h * HD + d, (size_t)a.ldo) : (size_t)tok * a.ldo + (size_t)h * HD + d;
  f.store((T*)a.out + at);
}

// Tile kernel (bf16, many rows per page): one workgroup of four waves per block of 128 (token,
// head) rows, KV head and key split.  A wave owns 32 rows, one per column of 32x32x16 MFMAs; chunks of
// 64 keys (four pages of K, four of V, one of each copied by every wave straight into LDS) pass
// through two LDS stages, the copies of the next chunk in flight while one is used, one barrier a
// chunk.  S^T = K Q^T with the K rows of a page taken in the order that swaps bits 2 and 3 of the
// row, so that a lane's eight scores of a page belong to eight consecutive keys, which is the
// B operand of O^T = V^T P^T as it stands, and V^T's fragments are contiguous 1 KiB reads.  K rows
// lie in LDS with their 16-byte pieces permuted by the row (the copies' source addresses are), so
// that the lanes of a K fragment, a row apart, fall on different banks.
// Weights meet V in two bf16 parts, as in the rows kernel, so that a call's outputs are as exact by either: one
// part, an error of 2^-9 of every weight, made the outputs' error 1.4 times that of their own rounding.  A
// prompt of 16384 tokens with a window of 4096, 32 heads of 128 (963 GFLOP, half as many again with the second
// part), takes 1.33 ms (725 TFLOP/s; 1.09 PFLOP/s of matrix instructions), with one part 1.01.  Head_dim 64 keeps
// three workgroups a compute unit for 16 bytes of scratch (8192 tokens, window 2048: 221 us, with two 236).
// Four stages were no faster where a workgroup has a compute unit to itself (32 heads over 8 of 128: 16 rows over
// 16400 keys 27.5 us, with four 29.6; 64 over 2000 19.7, 20.7; 128 over 8000 42.4, 42.3).
constexpr int kTileRows = 128;
constexpr int kChunkT = 64;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));

// Wave-wide copies of a page of N KiB at src (the same for every lane) into LDS at dst: copy j brings
// the 16 bytes at off[j] + j * step of every lane to dst + 1024 j + 16 lane.  Buffer copies: after a
// global one, which counts as flat, every wait for LDS reads would be a full one.
template <int N>
__device__ __forceinline__ void copy_page(const char* src, char* dst, const int* off, int step) {
  const __amdgpu_buffer_rsrc_t b = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(src), 0, N * 1024, 0x00027000);
#pragma unroll
  for (int j = 0; j < N; ++j)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (lds_void_t*)(dst + j * 1024), 16, off[j], j * step, 0, 0);
}

template <int HD>
struct TileLds {
  char stage[2 * 2 * (kChunkT / kPage) * kPage * HD * 2];
};
template <int HD>
__device__ __forceinline__ void tile_body(const PagedAttnArgs& a, const PagedPass& ps, int group, TileLds<HD>& lds) {
  constexpr int ROWB = HD * 2, NP = ROWB / 16, PGB = kPage * ROWB, NLD = PGB / 1024;
  constexpr int PAGES = kChunkT / kPage, STG = 2 * PAGES * PGB;
  constexpr int NKS = HD / 16, NDT = HD / 32;
  constexpr int OPB = ROWB + 16;                       // pitch of a finished row in LDS
  static_assert(2 * STG >= kTileRows * OPB, "finished rows fit the stages");
  static_assert(sizeof(lds.stage) == 2 * STG, "stages");
  char* const smem = lds.stage;
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 63, g = lane >> 5, c32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = group % r.n_kv_heads, split = group / r.n_kv_heads % ps.splits;
  const int blk = group / (r.n_kv_heads * ps.splits);
  const int G = r.n_q_heads / r.n_kv_heads;
  int s, rb;
  SeqRows sr;
  if (!block_rows(a, ps.shared, blk, kTileRows, s, rb, sr)) return;
  const int nrows = sr.n * G, row0 = rb * kTileRows;
  if (row0 >= nrows) return;

  // the keys that any row of the block sees: its first and last rows span them, except over the
  // rows of several sequences, whose prefix passes take all of the prefix
  const int first_tok = sr.a + row0 / G, last_tok = sr.a + (min(nrows, row0 + kTileRows) - 1) / G;
  const RowRange rf = ps.shared ? RowRange{0, min(a.prefix, r.max_pages * kPage), 0} : lane_range(a, ps, sr, first_tok);
  const RowRange rl = ps.shared ? rf : lane_range(a, ps, sr, last_tok);
  const int all_hi = __builtin_amdgcn_readfirstlane(max(rf.hi, rl.hi));
  const Steps<kChunkT> st(__builtin_amdgcn_readfirstlane(max(rf.snk, rl.snk)),
                          __builtin_amdgcn_readfirstlane(min(rf.lo, rl.lo)), all_hi);
  const int per = (st.n + ps.splits - 1) / ps.splits;
  const int i_beg = split * per, i_end = min(st.n, i_beg + per);

  // source offsets of this wave's copies (LDS slot j * 64 + lane of its page)
  auto swz = [](int row) { return NP == 16 ? row : row >> 1; };
  int koff[NLD], voff[NLD];
#pragma unroll
  for (int j = 0; j < NLD; ++j) {
    const int sl = j * 64 + lane, row = sl / NP, pc = sl % NP;
    koff[j] = row * ROWB + (pc ^ swz(row)) * 16;
    voff[j] = lane * 16;
  }
  const TableRow pt(a, s);
  const int last_page = max(0, (all_hi - 1) / kPage);
  struct Pages { int id[PAGES], own; };              // own: the page that this wave copies
  auto pages_at = [&](int i) {
    Pages p;
    const int pg = st.key(i) / kPage;
#pragma unroll
    for (int u = 0; u < PAGES; ++u) p.id[u] = pt.page(min(pg + u, last_page));
    p.own = pt.page(min(pg + w, last_page));
    return p;
  };
  auto ok_page = [&](int id) { return id >= 0 && id < r.n_pages; };
  auto issue = [&](const Pages& p, int stage) {
    const size_t at = ((size_t)(ok_page(p.own) ? p.own : 0) * r.n_kv_heads + kvh) * PGB;
    char* l = smem + stage + w * PGB;
    copy_page<NLD>((const char*)r.k + at, l, koff, 0);
    copy_page<NLD>((const char*)r.v + at, l + PAGES * PGB, voff, 1024);
  };
  // page ids of the chunk in use and of the next two: the last are asked for at the end of a step
  // (a scalar load under way would make every LDS wait a full one)
  Pages ids[3] = {};
  if (i_beg < i_end) {
#pragma unroll
    for (int x = 0; x < 3; ++x) ids[x] = pages_at(min(i_beg + x, i_end - 1));
    issue(ids[0], 0);
  }
  // this lane's row
  const int wrow = row0 + w * 32;
  const bool live = wrow < nrows;                       // this wave has rows
  const int rr = min(wrow + c32, nrows - 1);
  const int tok = sr.a + rr / G, head = kvh * G + rr % G;
  const RowRange rg = lane_range(a, ps, sr, tok);
  const int min_hi = wave_min(rg.hi), max_lo = wave_max(rg.lo), min_snk = wave_min(rg.snk);
  const int max_hi = wave_max(rg.hi), min_lo = wave_min(rg.lo), max_snk = wave_max(rg.snk);
  Frag<bf16_t> qf[NKS];
  {
    const bf16_t* qp = (const bf16_t*)a.q + (size_t)tok * a.ldq + (size_t)head * HD + g * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks].load(qp + ks * 16);
  }

  // read offsets: K fragment ks of the tile's rows, V fragments
  const int krow = (c32 & 16) * 1 + ((c32 & 4) << 1) + ((c32 & 8) >> 1) + (c32 & 3);   // bits 2 and 3 swapped
  // (piece 2 ks + g of the row, permuted: the pieces of ks differ from those of 0 in bits alone)
  const int kad = (krow >> 4) * PGB + (krow & 15) * ROWB + (g ^ swz(krow & 15)) * 16;
  const int vad = PAGES * PGB + c32 * 32 + g * 16;

  const float sl2 = a.scale * 1.4426950408889634f;
  float mref = kMrefInit, lsum = 0.f;
  f32x16 o[NDT];
#pragma unroll
  for (int d = 0; d < NDT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;

  int stage = 0;
  for (int i = i_beg; i < i_end; ++i) {
    wait_vm<0>();      // this wave's copies of chunk i have landed
    lds_barrier();     // everyone's have; chunk i-1's stage is free
    const Pages here = ids[0];
    if (i + 1 < i_end) issue(ids[1], stage ^ STG);
    ids[0] = ids[1];
    ids[1] = ids[2];
    auto next_pages = [&]() { ids[2] = pages_at(min(i + 3, i_end - 1)); };
    const int k0 = st.key(i);
    const char* sm = smem + stage;
    stage ^= STG;
    // (a wave none of whose rows sees the chunk passes it by)
    if (!live || !((k0 < max_hi && k0 + kChunkT > min_lo) || k0 < max_snk)) {
      next_pages();
      continue;
    }
    // all of the chunk's K fragments are asked for before the first product, and V fragments
    // before the softmax, whose arithmetic covers their way
    f32x16 sc[2];
    bf16x8 kf[2][NKS], vf[PAGES][NDT];
    auto late_v = [&]() {          // (the registers of the scores are free by then)
#pragma unroll
      for (int pg = PAGES / 2; pg < PAGES; ++pg)
#pragma unroll
        for (int d = 0; d < NDT; ++d) vf[pg][d] = *reinterpret_cast<const bf16x8*>(sm + vad + pg * PGB + d * 1024);
    };
    const int ka = (int)(sm - smem) + kad;
    wait_lds();                    // (the page ids are here: from now on LDS reads alone are waited for)
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t) kf[t][ks] = *reinterpret_cast<const bf16x8*>(smem + (ka ^ (32 * ks)) + t * 2 * PGB);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[t][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t][ks], qf[ks].v, sc[t], 0, 0, 0);
#pragma unroll
    for (int pg = 0; pg < PAGES / 2; ++pg)
#pragma unroll
      for (int d = 0; d < NDT; ++d) vf[pg][d] = *reinterpret_cast<const bf16x8*>(sm + vad + pg * PGB + d * 1024);
    __builtin_amdgcn_sched_barrier(0);
    bool pages_ok = true;
#pragma unroll
    for (int u = 0; u < PAGES; ++u) pages_ok = pages_ok && ok_page(here.id[u]);
    const bool whole = pages_ok && k0 + kChunkT <= min_hi && (k0 >= max_lo || k0 + kChunkT <= min_snk);
    unsigned bad = 0;                                   // bit 8 page + e: key 16 page + 8 g + e
    if (!whole) {
      uint32_t hid = 0;
#pragma unroll
      for (int u = 0; u < PAGES; ++u)
        hid |= (ok_page(here.id[u]) ? hidden8(rg, k0 + u * kPage + 8 * g) : 0xffu) << (8 * u);
#pragma unroll
      for (int x = 0; x < 32; ++x) sc[x >> 4][x & 15] = hide(sc[x >> 4][x & 15], hid, x);
      // keys with a non-finite V element somewhere: a weight of zero must not meet them in a
      // product, so where rows differ in what they see they are added one by one
      Finite fin;
#pragma unroll 1
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int pg = 0; pg < PAGES; ++pg) fin.add(*reinterpret_cast<const bf16x8*>(sm + vad + pg * PGB + d * 1024));
      if (!fin.all()) {
#pragma unroll 1
        for (int d = 0; d < NDT; ++d)
#pragma unroll
          for (int pg = 0; pg < PAGES; ++pg) {
            const bf16x8 v = *reinterpret_cast<const bf16x8*>(sm + vad + pg * PGB + d * 1024);
#pragma unroll
            for (int e = 0; e < 8; ++e) bad |= ((v[e] & 0x7f80) == 0x7f80 ? 1u : 0u) << (8 * pg + e);
          }
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) bad |= (unsigned)__shfl_xor((int)bad, x, 64);
      }
    }
    float m4[4], mx;
#pragma unroll
    for (int x = 0; x < 4; ++x) m4[x] = sc[x >> 1][8 * (x & 1)];
#pragma unroll
    for (int y = 1; y < 8; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x) m4[x] = __builtin_elementwise_maximum(m4[x], sc[x >> 1][8 * (x & 1) + y]);
    mx = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m4[0], m4[1]), __builtin_elementwise_maximum(m4[2], m4[3]));
    {
      const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = __builtin_elementwise_maximum(__uint_as_float(h[0]), __uint_as_float(h[1])) * sl2;
    }
    if (__ballot(mx > mref + 8.f)) {                    // the reference rises by 2^8 or more, or not at all
      const float mn = fmaxf(mref, mx), al = __builtin_amdgcn_exp2f(mref - mn);
#pragma unroll
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= al;
      lsum *= al;
      mref = mn;
    }
    // weights of a page's eight keys, in two parts as the rows kernel's: their bf16 rounding and
    // that of what it left over
    u32x4 pf[PAGES], pl[PAGES];
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[x >> 4][x & 15], sl2, -mref));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[(x + 1) >> 4][(x + 1) & 15], sl2, -mref));
      lsum += p0 + p1;
      const unsigned ph = __builtin_bit_cast(unsigned, bf2{(__bf16)p0, (__bf16)p1});
      const bf2 pr = {(__bf16)(p0 - __uint_as_float(ph << 16)), (__bf16)(p1 - __uint_as_float(ph & 0xffff0000u))};
      pf[x >> 3][x >> 1 & 3] = ph;
      pl[x >> 3][x >> 1 & 3] = __builtin_bit_cast(unsigned, pr);
    }
    late_v();
    const bool any_bad = __ballot(bad != 0) != 0;
    if (any_bad) {                                      // the product without those keys
#pragma unroll
      for (int pg = 0; pg < PAGES; ++pg) {
        u32x4 keep;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          keep[e] = (bad >> (8 * pg + 2 * e) & 1 ? 0u : 0xffffu) | (bad >> (8 * pg + 2 * e + 1) & 1 ? 0u : 0xffff0000u);
#pragma unroll
        for (int d = 0; d < NDT; ++d) vf[pg][d] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, vf[pg][d]) & keep);
      }
    }
#pragma unroll
    for (int pg = 0; pg < PAGES; ++pg) {
#pragma unroll
      for (int d = 0; d < NDT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[pg][d], __builtin_bit_cast(bf16x8, pf[pg]), o[d], 0, 0, 0);
#pragma unroll
      for (int d = 0; d < NDT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[pg][d], __builtin_bit_cast(bf16x8, pl[pg]), o[d], 0, 0, 0);
    }
    wait_lds();                    // (this wave's reads of the stage end before the barrier that gives it away)
    next_pages();
    if (!any_bad) continue;
#pragma unroll 1
    for (int gg = 0; gg < 2; ++gg) {
#pragma unroll 1
      for (unsigned m = __builtin_amdgcn_readlane((int)bad, 32 * gg); m; m &= m - 1) {
        const int x = __builtin_ctz(m);                 // key 16 (x / 8) + 8 gg + x % 8
        unsigned u = pf[0][0], r = pl[0][0];
#pragma unroll
        for (int y = 1; y < 16; ++y) {
          u = (x >> 1) == y ? pf[y >> 2][y & 3] : u;
          r = (x >> 1) == y ? pl[y >> 2][y & 3] : r;
        }
        const float pm = __uint_as_float(x & 1 ? u & 0xffff0000u : u << 16) +
                         __uint_as_float(x & 1 ? r & 0xffff0000u : r << 16);
        const float pj = __shfl(pm, c32 + 32 * gg, 64);
        const bf16_t* vj = reinterpret_cast<const bf16_t*>(sm + PAGES * PGB + (x >> 3) * PGB) + 8 * gg + (x & 7);
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            const float v = bf16_to_f32(vj[(32 * d + 8 * (y >> 2) + 4 * g + (y & 3)) * kPage]);
            o[d][y] += pj != 0.f ? pj * v : 0.f;
          }
      }
    }
    wait_lds();
  }
  {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(lsum), __float_as_uint(lsum), false, false);
    lsum = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  }
  const bool row_ok = wrow + c32 < nrows;
  const size_t rh = (size_t)tok * r.n_q_heads + head, zst = (size_t)r.n_rows * r.n_q_heads;
  if (ps.z0 >= 0) {
    if (!row_ok) return;
    const size_t row = (ps.z0 + split) * zst + rh;
    float* op = a.part_o + row * HD;
#pragma unroll
    for (int d = 0; d < NDT; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<float4*>(op + d * 32 + 8 * b + 4 * g) =
            make_float4(o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]);
    if (g == 0) {
      a.part_ml[row * 2] = mref;
      a.part_ml[row * 2 + 1] = lsum;
    }
    return;
  }
  // finished rows through LDS, so that they leave 16 bytes a lane along the row
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  lds_barrier();
  char* mine = smem + (size_t)w * 32 * OPB;
#pragma unroll
  for (int d = 0; d < NDT; ++d)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      uint2 u;
      bf16_t h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = lsum == 0.f ? (bf16_t)0 : f32_to_bf16(o[d][4 * b + e] * inv);
      u.x = h[0] | (unsigned)h[1] << 16;
      u.y = h[2] | (unsigned)h[3] << 16;
      *reinterpret_cast<uint2*>(mine + c32 * OPB + (d * 32 + 8 * b + 4 * g) * 2) = u;
    }
  wait_lds();
  for (int x = lane; x < 32 * NP; x += 64) {
    const int rl = x / NP, pc = x % NP, rw = wrow + rl;
    if (rw >= nrows) break;
    const int tk = sr.a + rw / G, col = (kvh * G + rw % G) * HD + pc * 8;
    const uint4 u = *reinterpret_cast<const uint4*>(mine + rl * OPB + pc * 16);
    const size_t at = a.packed ? pa_index(tk, col, (size_t)a.ldo) : (size_t)tk * a.ldo + col;
    *reinterpret_cast<uint4*>((bf16_t*)a.out + at) = u;
  }
}

// The launches: workgroups below p0.groups work on the first pass, the others on the second.
template <typename T, int HD, int NT, int NW, bool NTL>
__global__ __launch_bounds__(64 * NW, 2) void paged_rows_kernel(PagedAttnArgs a, PagedPass p0, PagedPass p1) {
  __shared__ __attribute__((aligned(16))) RowsLds<HD, NT, NW> lds;
  const bool first = (int)blockIdx.x < p0.groups;
  rows_body<T, HD, NT, NW, NTL>(a, first ? p0 : p1, blockIdx.x - (first ? 0 : p0.groups), lds);
}
template <int HD>
__global__ __launch_bounds__(256, HD == 64 ? 3 : 2) void paged_tile_kernel(PagedAttnArgs a, PagedPass p0, PagedPass p1) {
  __shared__ __attribute__((aligned(1024))) TileLds<HD> lds;
  const bool first = (int)blockIdx.x < p0.groups;
  tile_body<HD>(a, first ? p0 : p1, blockIdx.x - (first ? 0 : p0.groups), lds);
}
// The prefix in tiles, the sequences' own keys by rows: the first is bound by arithmetic, the second
// by memory, and a compute unit runs one of each (64 tokens behind 8192 shared and up to 1024 own keys: 48 us with
// the merge, 63 as two launches).
template <int HD, bool NTL>
__global__ __launch_bounds__(256, 2) void paged_both_kernel(PagedAttnArgs a, PagedPass p0, PagedPass p1) {
  union Lds {
    TileLds<HD> t;
    RowsLds<HD, 1, 4> r;
  };
  __shared__ __attribute__((aligned(1024))) char lds[sizeof(Lds)];
  if ((int)blockIdx.x < p0.groups) tile_body<HD>(a, p0, blockIdx.x, reinterpret_cast<Lds*>(lds)->t);
  else rows_body<bf16_t, HD, 1, 4, NTL>(a, p1, blockIdx.x - p0.groups, reinterpret_cast<Lds*>(lds)->r);
}

// Joins the zs partial results of every (row, head), one wave each: sums and weights over the
// lanes, a part each, then the parts' elements, four a lane, 256 / HD parts at a time, four such loads
// under way (10240 rows of 128, seven parts, 37 MB: 8.8 us).
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a, int zs) {
  constexpr int LPR = HD / 4, ZG = 64 / LPR;              // lanes of a part, parts at a time
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 63, zg = lane / LPR, d = lane % LPR * 4;
  const long rh = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rh >= (long)r.n_rows * r.n_q_heads) return;
  const int tok = (int)(rh / r.n_q_heads), h = (int)(rh % r.n_q_heads);
  const size_t zst = (size_t)r.n_rows * r.n_q_heads;
  float2 ml = make_float2(kMrefInit, 0.f);
  if (lane < zs) ml = *reinterpret_cast<const float2*>(a.part_ml + (lane * zst + rh) * 2);
  const int s = row_seq(r, tok);
  if (s >= r.n_seqs) return;               // a row behind the last sequence: left as it was
  const SeqRows sr = seq_rows(r, s);
  if (tok < sr.a || tok >= sr.a + sr.n) return;
  const float M = warp_max(ml.x);
  const float f = lane < zs ? __builtin_amdgcn_exp2f(ml.x - M) : 0.f;
  const float L = warp_sum(f * ml.y);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  const float* op = a.part_o + rh * HD + d;
  for (int z0 = 0; z0 < zs; z0 += 4 * ZG) {
    float4 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int z = z0 + u * ZG + zg;
      p[u] = z < zs ? *reinterpret_cast<const float4*>(op + z * zst * HD) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int z = z0 + u * ZG + zg;
      const float fz = __shfl(f, z & 63, 64);
      if (z >= zs) continue;
      v[0] += fz * p[u].x; v[1] += fz * p[u].y; v[2] += fz * p[u].z; v[3] += fz * p[u].w;
    }
  }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], o, 64);
  if (zg) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int col = h * HD + d;
  T* out = (T*)a.out + (a.packed ? pa_index(tok, col, (size_t)a.ldo) : (size_t)tok * a.ldo + col);
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = Elem<T>::from_f32(L == 0.f ? 0.f : v[e] * inv);
}

// ------------------------------------------------------------------ host
static long row_blocks(const PagedAttnArgs& a, bool shared, int rb) {
  const PagedRows& r = a.r;
  const int G = r.n_q_heads / r.n_kv_heads;
  if (shared) return ((long)r.n_rows * G + rb - 1) / rb;
  if (r.row_start) return (long)r.n_rows * G / rb + r.n_seqs;
  return (long)r.n_seqs * (((long)r.rows_each * G + rb - 1) / rb);
}
// (token, head) rows for a KV head: of all sequences over the prefix, else of a sequence on the average over
// as many as can have any.  (Not of the longest: one prompt among single tokens does not fill their tiles.)
static long rows_of(const PagedAttnArgs& a, bool shared) {
  const PagedRows& r = a.r;
  const long n = shared ? 1 : r.n_seqs < r.n_rows ? r.n_seqs : r.n_rows;
  return (r.n_rows + n - 1) / n * (r.n_q_heads / r.n_kv_heads);
}
// Keys that `tokens` consecutive rows of a sequence read in a pass from key `first` on, as far as
// the host knows.
static long keys_of(const PagedAttnArgs& a, long first, long tokens) {
  const long keys = a.max_kv - first, seen = (long)a.window + a.sinks + (tokens < a.max_rows ? tokens : a.max_rows);
  return a.window > 0 && keys > seen ? seen : keys < 0 ? 0 : keys;
}
// Query tiles of a wave of the rows kernel: two where blocks of one tile are more than the 256 compute units and
// read more than 28 steps of keys, each page then being read half as often.  One tile, two, us: 16 rows a sequence of 4
// heads of 64 over 2 behind 1000 keys 320 blocks 36.0 27.2, 640 54.9 47.0, 1400 109 95; behind 2000 400 65.5 51.6,
// 640 105 90.  32 heads over 8: behind 1000 320 blocks 29.2 26.1, 512 30.0 32.6, 768 42.3 45.4, 1024 53.3 46.4; behind
// 2000 320 49.9 38.1, 768 74.8 81.5, 1024 99.9 83.1.  Fewer blocks or keys gain less than they lose: behind
// 1000 192 21.1 19.3, 256 22.4 21.5; behind 700 320 22.6 25.4, 640 31.6 34.9, 1024 41.2 35.9; behind 300 256 10.1
// 13.6, 512 14.4 13.7, 768 18.9 21.1; a window of 128 320 11.5 11.6, 640 14.2 16.2, 800 18.1 16.2.  Head_dim 128 would
// not leave the registers for it.
static int rows_nt(const PagedAttnArgs& a, int elem_bytes) {
  const PagedRows& r = a.r;
  return elem_bytes == 4 && r.head_dim == 64 && rows_of(a, false) > 16 &&
                 row_blocks(a, false, 16) * r.n_kv_heads > 256 && keys_of(a, 0, 16) > 28 * kStep ? 2 : 1;
}
// Whether a pass (the sequences' own: from key `first` on) takes the tile kernel: bf16 rows that on the average
// fill more than one block of 16 and, of the own pass, whose blocks would read more than 160 MB of
// pages between them (40e6 places of K and V).  Below that the rows kernel, whose waves share a block's
// keys, ends sooner.  Rows against tiles, us, 32 heads over 8 of 128: blocks of 16 tokens, 16 sequences behind 300
// keys (21e6) 11.6, 15.3; 32 (41e6) 20.9, 17.7; 4 behind 2048 (34e6) 20.0, 19.1; 8 (68e6) 30.6, 27.0; 16 behind 1024
// (68e6) 26.4, 27.8; prompts of 200 tokens, two (20e6) 11.5, 12.8; four (41e6) 19.1, 13.5; of 500, one (64e6) 18.9,
// 20.2; two 33.1, 21.2.  Heads of 64: 16 tokens, 32 behind 1024 (68e6) 25.0, 31.0; four prompts of 500 31.3, 22.7.
static bool tiled(const PagedAttnArgs& a, bool shared, long first, int elem_bytes) {
  const PagedRows& r = a.r;
  if (elem_bytes != 2 || rows_of(a, shared) <= 16) return false;
  return shared || (double)row_blocks(a, false, 16) * r.n_kv_heads * r.head_dim * keys_of(a, first, 16) > 40e6;
}
static int block_size(const PagedAttnArgs& a, bool shared, long first, int elem_bytes) {
  return tiled(a, shared, first, elem_bytes) ? kTileRows : 16 * rows_nt(a, elem_bytes);
}
// Whether the rows kernel's pages come by non-temporal loads: where each is read by one workgroup
// and all of them may be more than twice the 256 MB memory-side cache (64 steps over 4100 keys, 1.08
// GB: 165 us against 185; 64 steps over up to 1024 keys of their own beside a prefix, at most 268
// MB: 58.2 us against 54.4 with plain loads).
static bool streamed(const PagedAttnArgs& a, long first, int elem_bytes) {
  const PagedRows& r = a.r;
  return a.prefix <= first && (long)a.max_rows * (r.n_q_heads / r.n_kv_heads) <= 16 &&
         2.0 * r.n_seqs * keys_of(a, first, a.max_rows) * r.n_kv_heads * r.head_dim * elem_bytes > 512e6;
}

PagedPlan paged_plan(const PagedAttnArgs& a, int elem_bytes) {
  const PagedRows& r = a.r;
  PagedPlan p{1, 0};
  // A pass over the shared prefix of its own pays where the sequences' rows do not, on the average, fill tiles by
  // themselves and reading the prefix once for each would move over 60 MB more than reading it once, and 56 bytes
  // more for every element of the rows' outputs: two parts of 4 bytes are written and read, and count
  // 3.5 times, since what is read again mostly lies in caches.  In one pass against two, us, 8 KV heads of 128: single
  // tokens, four query heads each, 8 sequences behind 2048 keys (59 MB) 13.1, 13.7; 8 behind 4096 17.8, 14.5; 16 behind
  // 4096 28.1, 15.5; 64 behind 1024 27.6, 18.2.  Blocks of 16 tokens: 4 behind 4096 (50 MB) 24.0, 22.6; 16 behind 1024
  // (63) 25.4, 24.6; 32 behind 1024 (130) 38.0, 38.4; 64 behind 1024 (264) 50.3, 62.3; 16 behind 2048 34.2, 30.1; 32
  // behind 2048 55.9, 52.0; 16 behind 4096 52.5, 47.4.  Heads of 64: 64 behind 1024 (132) 38.2, 50.6; 16 behind 4096
  // 40.2, 32.7; 8 heads over 4, 64 behind 1024 (66) 14.7, 20.7; 64 behind 4096 50.6, 35.4.
  // A prompt of 96 rows among 63 tokens, all behind 8192: 394, 58; of 200 among 15 behind 4096 93, 48.  In fp32 the pass
  // goes in blocks of 16, which 16 pairs fill: 8 KV heads of 64 with four query heads each, 64 behind 1024, one token
  // 34.0, 21.6, 16 tokens 93, 117; 32 behind 2048, four tokens 35.2, 34.9; 4 KV heads with two, four tokens 22.3, 17.5.
  const double pre = 2.0 * a.prefix * r.n_kv_heads * r.head_dim * elem_bytes;
  const bool apart = a.prefix > 0 && rows_of(a, false) < (elem_bytes == 2 ? kTileRows : 16) &&
                     (r.n_seqs - 1) * pre > 60e6 + 56.0 * r.n_rows * r.n_q_heads * r.head_dim;
  const long first = apart ? a.prefix : 0;
  auto pick = [&](bool shared, long keys) {
    const bool tile = tiled(a, shared, first, elem_bytes);
    const long units = row_blocks(a, shared, block_size(a, shared, first, elem_bytes)) * r.n_kv_heads;
    // two workgroups for each of the 256 compute units; more than 32 parts, which a merge then reads,
    // only as far as the chip is half filled by them (one step over 131072 keys of two KV heads: 56.8 us with
    // 32, 40.4 with 64; of eight 87.1 and 89.5)
    long s = 512 / units;
    if (s > kMaxParts) s = apart || 128 / units < kMaxParts ? kMaxParts : 128 / units;
    long most = keys / (tile ? 4 * kChunkT : 8 * kStep);
    if (shared && tile) {
      // Over the prefix a part is written and read for every row of the batch, 0.3 us per 2^17 elements,
      // while a split takes 1.3 us a chunk (64 tokens of 32 heads behind 8192 keys: 38.5 us; reckoned with 1.0 39.7,
      // with 1.7 42.7): the sum of both is least at the root below; up to the time that
      // the sequences' own keys take beside it a split costs nothing.
      const double part = 0.3 / (1 << 17) * r.n_rows * r.n_q_heads * r.head_dim;
      const double own = 1e-6 / 5 * r.n_seqs * keys_of(a, first, a.max_rows) * r.n_kv_heads * r.head_dim * elem_bytes;
      const double chunks = fmin(16, fmax(4, fmax(sqrt(keys / (double)kChunkT * part / 1.3), own / 1.3)));
      most = (long)(keys / (kChunkT * chunks) + 0.5);
    }
    // Parts need a merge of some 3 us, as much as a few steps of a wave: fewer steps are one part.  In fp32 at
    // head_dim 128 a step is 4096 cycles of matrix instructions, and two parts pay at once.  Four tokens
    // and 8 KV heads, in parts and as one, us: bf16 of 128, 577 keys 9.9 10.1, 640 9.8 9.9, 768 9.1 11.1, 1028 9.7
    // 14.4; bf16 of 64, 577 8.8 7.0, 768 8.1 7.4, 900 8.7 8.6, 1028 8.6 9.1; fp32 of 64, 577 12.0 12.2, 640 11.6
    // 11.8, 768 10.5 13.2; fp32 of 128, 577 18.3 24.1, 768 15.0 28.1.
    const int few = elem_bytes == 2 ? (r.head_dim == 64 ? 7 : 5) : r.head_dim == 64 ? 5 : 0;
    if (!shared && !tile && keys <= few * 4 * kStep) most = 1;
    if (s > most) s = most;
    return (int)(s < 1 ? 1 : s > kMaxMerge ? kMaxMerge : s);
  };
  p.splits = pick(false, keys_of(a, first, block_size(a, false, first, elem_bytes) * r.n_kv_heads / r.n_q_heads + 1));
  if (apart) p.shared = pick(true, a.prefix);
  return p;
}

size_t paged_part_floats(const PagedAttnArgs& a, const PagedPlan& p, size_t* ml) {
  const size_t rows = (size_t)p.parts() * a.r.n_rows * a.r.n_q_heads;
  *ml = rows * 2;
  return rows * a.r.head_dim;
}

PagedChoice paged_choice(const PagedAttnArgs& a, const PagedPlan& p, int elem_bytes) {
  const long first = p.shared ? a.prefix : 0;
  PagedChoice c{};
  c.g0 = p.shared ? row_blocks(a, true, block_size(a, true, first, elem_bytes)) * p.shared * a.r.n_kv_heads : 0;
  c.g1 = row_blocks(a, false, block_size(a, false, first, elem_bytes)) * p.splits * a.r.n_kv_heads;
  // (own rows in tiles: more than 16 rows of a sequence, the prefix is in tiles too)
  c.kernel = tiled(a, false, first, elem_bytes)              ? RT_A_TILES
             : p.shared && tiled(a, true, first, elem_bytes) ? RT_A_PREFIX_TILES
             : rows_nt(a, elem_bytes) == 2                   ? RT_A_ROWS_PAIRS
                                                             : RT_A_ROWS;
  c.streamed = (c.kernel == RT_A_ROWS || c.kernel == RT_A_PREFIX_TILES) && streamed(a, first, elem_bytes);
  return c;
}

template <typename T, int HD>
static hipError_t launch_hd(const PagedAttnArgs& a, const PagedPlan& p, int i, hipStream_t s) {
  const PagedRows& r = a.r;
  if (i > 0) {
    const long rows = (long)r.n_rows * r.n_q_heads;
    RT_LAUNCH((paged_merge_kernel<T, HD>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a, p.parts());
    return hipGetLastError();
  }
  const PagedChoice c = paged_choice(a, p, sizeof(T));
  if (c.g0 + c.g1 <= 0) return hipSuccess;
  if (c.g0 + c.g1 > kMaxGrid || (p.parts() && ((long)r.n_rows * r.n_q_heads + 3) / 4 > kMaxGrid)) return hipErrorInvalidValue;
  const PagedPass p0{1, 0, p.shared, 0, (int)c.g0};
  const PagedPass p1{0, p.shared ? a.prefix : 0, p.splits, p.parts() ? p.shared : -1, (int)c.g1};
  const dim3 gd((unsigned)(c.g0 + c.g1));
  if constexpr (sizeof(T) == 2) {
    if (c.kernel == RT_A_TILES) RT_LAUNCH((paged_tile_kernel<HD>), gd, dim3(256), 0, s, a, p0, p1);
    else if (c.kernel == RT_A_PREFIX_TILES && c.streamed) RT_LAUNCH((paged_both_kernel<HD, true>), gd, dim3(256), 0, s, a, p0, p1);
    else if (c.kernel == RT_A_PREFIX_TILES) RT_LAUNCH((paged_both_kernel<HD, false>), gd, dim3(256), 0, s, a, p0, p1);
    if (c.kernel != RT_A_ROWS) return hipGetLastError();
  } else if constexpr (HD == 64) {
    if (c.kernel == RT_A_ROWS_PAIRS) {
      RT_LAUNCH((paged_rows_kernel<T, HD, 2, 4, false>), gd, dim3(256), 0, s, a, p0, p1);
      return hipGetLastError();
    }
  }
  if (c.streamed) RT_LAUNCH((paged_rows_kernel<T, HD, 1, 4, true>), gd, dim3(256), 0, s, a, p0, p1);
  else RT_LAUNCH((paged_rows_kernel<T, HD, 1, 4, false>), gd, dim3(256), 0, s, a, p0, p1);
  return hipGetLastError();
}
template <typename T>
hipError_t paged_launch(const PagedAttnArgs& a, const PagedPlan& p, int i, hipStream_t s) {
  if (a.r.n_rows <= 0 || a.r.n_seqs <= 0) return hipSuccess;
  return a.r.head_dim == 128 ? launch_hd<T, 128>(a, p, i, s) : launch_hd<T, 64>(a, p, i, s);
}
template hipError_t paged_launch<bf16_t>(const PagedAttnArgs&, const PagedPlan&, int, hipStream_t);
template hipError_t paged_launch<float>(const PagedAttnArgs&, const PagedPlan&, int, hipStream_t);

}  // namespace rt
