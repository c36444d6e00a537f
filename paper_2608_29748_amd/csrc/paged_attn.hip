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
//   prefix      keys [0, prefix) in one pass over the rows of all sequences, whose tiles so
//               fill with rows that read the same pages; [prefix, p] sequence by sequence.
#include "paged.h"

namespace rt {

typedef __attribute__((address_space(4))) const int32_t const_i32_t;

constexpr int kStep = 32;                  // keys per step of a wave: two pages
constexpr float kMrefInit = -1.0e30f;      // running maximum before any visible key (log2 units)

struct RowRange { int lo, hi, snk; };
__device__ __forceinline__ RowRange row_range(const PagedAttnArgs& a, bool shared, long pos, int keys) {
  const long cap = (long)a.r.max_pages * kPage;
  long hi = a.causal ? pos + 1 : (long)keys;
  hi = max(0l, min(hi, shared ? min(cap, (long)a.prefix) : cap));
  long lo = shared ? 0 : (long)a.prefix;
  if (a.window > 0) lo = max(lo, pos - a.window + 1);
  lo = min(max(lo, 0l), hi);
  return RowRange{(int)lo, (int)hi, (int)min((long)a.sinks, lo)};
}

// Steps of the keys [0, snk) and [lo, hi), those of the sinks first.
struct Steps {
  int n_snk, first, n;
  __device__ __forceinline__ int key(int i) const { return (i < n_snk ? i : first + (i - n_snk)) * kStep; }
};
__device__ __forceinline__ Steps steps_of(int snk, int lo, int hi) {
  Steps t;
  t.first = lo / kStep;
  const int last = (hi + kStep - 1) / kStep;
  t.n_snk = min((snk + kStep - 1) / kStep, t.first);
  if (last <= t.first) t.first = last;
  t.n = t.n_snk + last - t.first;
  return t;
}

__device__ __forceinline__ int rows16_min(int v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = min(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ int rows16_max(int v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = max(v, __shfl_xor(v, o, 64));
  return v;
}

// Rows kernel: one workgroup of NW waves per block of 16 NT (token, head) rows, KV head and key
// split.  Every wave takes every NW-th step of 32 keys of the split straight from memory into
// registers in MFMA operand order (S^T = K Q^T, O^T = V^T P^T; the K rows of a 16-row tile are
// the keys 8(r/4) + 4 tile + r%4, so that a lane ends up with eight consecutive keys of its
// query, whose V^T fragment is one contiguous read); the waves' results meet in LDS.
template <typename T, int HD, int NT, int NW>
__global__ __launch_bounds__(64 * NW) void paged_rows_kernel(PagedAttnArgs a, int shared, int splits, int z0, int zs) {
  constexpr int NHT = HD / 16, NKS = HD / 32;
  constexpr int RB = 16 * NT;
  constexpr int OP = HD + 4;                               // fp32 pitch of a merged row
  __shared__ __attribute__((aligned(16))) float sO[NW][RB][OP];
  __shared__ float sML[NW][RB][2];
  __shared__ float sP[NW][kStep][16];                      // one tile's weights (non-finite V only)
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 63, g4 = lane >> 4, c16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % r.n_kv_heads, split = blockIdx.x / r.n_kv_heads % splits;
  const int blk = blockIdx.x / (r.n_kv_heads * splits);
  const int G = r.n_q_heads / r.n_kv_heads;
  int s = 0, rb = blk;
  SeqRows sr{0, r.n_rows, 0};
  if (!shared) {
    if (r.row_start) {
      if (!find_block(r.n_seqs, blk, [&](int i) { return (seq_rows(r, i).n * G + RB - 1) / RB; }, s, rb)) return;
    } else {
      const int per = (r.rows_each * G + RB - 1) / RB;
      s = blk / per;
      rb = blk % per;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    rb = __builtin_amdgcn_readfirstlane(rb);
    sr = seq_rows(r, s);
  }
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
    SeqRows q = sr;
    if (shared) {
      int sq;
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
      if (tok < q.a || tok >= q.a + q.n) q.keys = q.n = 0;     // a row of no sequence
    }
    const long pos = (long)q.keys - q.n + (tok - q.a);
    rg[t] = row_range(a, shared, pos, q.keys);
    if (shared && q.n == 0) rg[t] = RowRange{0, 0, 0};
    const T* qp = (const T*)a.q + (size_t)tok * a.ldq + (size_t)(kvh * G + rr % G) * HD;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[t][ks].load(qp + ks * 32 + g4 * 8);
    all_lo = min(all_lo, rows16_min(rg[t].lo));
    max_lo = max(max_lo, rows16_max(rg[t].lo));
    all_hi = max(all_hi, rows16_max(rg[t].hi));
    min_hi = min(min_hi, rows16_min(rg[t].hi));
    all_snk = max(all_snk, rows16_max(rg[t].snk));
    min_snk = min(min_snk, rows16_min(rg[t].snk));
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  max_lo = __builtin_amdgcn_readfirstlane(max_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  min_hi = __builtin_amdgcn_readfirstlane(min_hi);
  all_snk = __builtin_amdgcn_readfirstlane(all_snk);
  min_snk = __builtin_amdgcn_readfirstlane(min_snk);
  const Steps st = steps_of(all_snk, all_lo, all_hi);
  const int per = (st.n + splits - 1) / splits;
  const int i_end = min(st.n, (split + 1) * per);

  const_i32_t* pt = (const_i32_t*)(r.page_table + (size_t)s * r.max_pages);
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

  for (int i = split * per + w; i < i_end; i += NW) {
    const int k0 = st.key(i);
    const int p0 = pt[min(k0 / kPage, last_page)], p1 = pt[min(k0 / kPage + 1, last_page)];
    const bool ok0 = p0 >= 0 && p0 < r.n_pages, ok1 = p1 >= 0 && p1 < r.n_pages;
    const size_t PE = (size_t)kPage * HD;
    const size_t b0 = ((size_t)(ok0 ? p0 : 0) * r.n_kv_heads + kvh) * PE;
    const size_t b1 = ((size_t)(ok1 ? p1 : 0) * r.n_kv_heads + kvh) * PE;
    const T* kp = (const T*)r.k + ((c16 >> 3) ? b1 : b0) + (size_t)(8 * ((c16 >> 2) & 1) + (c16 & 3)) * HD + g4 * 8;
    const T* vp = (const T*)r.v + ((g4 >> 1) ? b1 : b0) + (size_t)c16 * kPage + (g4 & 1) * 8;
    Frag<T> kf[2][NKS], vf[NHT];
#pragma unroll
    for (int ta = 0; ta < 2; ++ta)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) kf[ta][ks].load(kp + ta * 4 * HD + ks * 32);
#pragma unroll
    for (int h = 0; h < NHT; ++h) vf[h].load(vp + h * 16 * kPage);
    const bool whole = ok0 && ok1 && k0 + kStep <= min_hi && (k0 >= max_lo || k0 + kStep <= min_snk);
    // keys (of the 32) with a non-finite V element somewhere: a weight of zero must not meet
    // them in a product, so where rows differ in what they see they are added one by one
    uint32_t bad = 0;
    if (!whole) {
      uint32_t mine = 0;
#pragma unroll
      for (int h = 0; h < NHT; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) mine |= (__builtin_isfinite(vf[h].get(e)) ? 0u : 1u) << e;
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) mine |= __shfl_xor((int)mine, x, 64);
      if (__ballot(mine != 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (mine >> e & 1)
#pragma unroll
            for (int h = 0; h < NHT; ++h) vf[h].set(e, 0.f);
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
        mma(sc[0], kf[0][ks], qf[t][ks]);
        mma(sc[1], kf[1][ks], qf[t][ks]);
      }
      if (!whole) {
        const bool ok = g4 < 2 ? ok0 : ok1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = k0 + 8 * g4 + e;
          const bool vis = ok && j < rg[t].hi && (j >= rg[t].lo || j < rg[t].snk);
          sc[e >> 2][e & 3] = vis ? sc[e >> 2][e & 3] : -INFINITY;
        }
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
      // products (the matrix units have nothing else to do while the keys come in)
      Frag<T> ph, pl;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ph.set(e, p[e]);
        if constexpr (sizeof(T) == 2) pl.set(e, p[e] - ph.get(e));
      }
#pragma unroll
      for (int h = 0; h < NHT; ++h) {
        mma(o[t][h], vf[h], ph);
        if constexpr (sizeof(T) == 2) mma(o[t][h], vf[h], pl);
      }
      if (bad) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sP[w][8 * g4 + e][c16] = p[e];
        wait_lds();
        for (uint32_t m = bad; m; m &= m - 1) {
          const int j = __builtin_ctz(m);
          const float pj = *(volatile float*)&sP[w][j][c16];
          const T* vj = (const T*)r.v + (j < 16 ? b0 : b1) + (j & 15) + (size_t)(4 * g4) * kPage;
#pragma unroll
          for (int h = 0; h < NHT; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[t][h][e] += pj != 0.f ? pj * Elem<T>::to_f32(vj[(h * 16 + e) * kPage]) : 0.f;
        }
      }
    }
  }
  // join the waves
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
  for (int i = threadIdx.x; i < RB * (HD / 8); i += 64 * NW) {
    const int rl = i / (HD / 8), d = i % (HD / 8) * 8, rr = row0 + rl;
    if (rr >= nrows) continue;
    const int tok = sr.a + rr / G, h = kvh * G + rr % G;
    float M = sML[0][rl][0];
#pragma unroll
    for (int u = 1; u < NW; ++u) M = fmaxf(M, sML[u][rl][0]);
    float L = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NW; ++u) {
      const float f = __builtin_amdgcn_exp2f(sML[u][rl][0] - M);
      L += f * sML[u][rl][1];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += f * sO[u][rl][d + e];
    }
    if (zs > 1) {
      const size_t row = ((size_t)(z0 + split) * r.n_rows + tok) * r.n_q_heads + h;
      float* op = a.part_o + row * HD + d;
      *reinterpret_cast<float4*>(op) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(op + 4) = make_float4(v[4], v[5], v[6], v[7]);
      if (d == 0) {
        a.part_ml[row * 2] = M;
        a.part_ml[row * 2 + 1] = L;
      }
    } else {
      const float inv = L == 0.f ? 0.f : 1.f / L;       // (NaN stays NaN)
      Frag<T> f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f.set(e, L == 0.f ? 0.f : v[e] * inv);
      const size_t at = a.packed ? pa_index(tok, h * HD + d, (size_t)a.ldo) : (size_t)tok * a.ldo + (size_t)h * HD + d;
      f.store((T*)a.out + at);
    }
  }
}

// Joins the z partial results of every (row, head): one wave each, HD / 64 elements a lane.
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a, int zs) {
  constexpr int E = HD / 64;
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 63;
  const long rh = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (rh >= (long)r.n_rows * r.n_q_heads) return;
  const int tok = (int)(rh / r.n_q_heads), h = (int)(rh % r.n_q_heads);
  const int s = row_seq(r, tok);
  if (s >= r.n_seqs) return;               // a row behind the last sequence: left as it was
  const SeqRows sr = seq_rows(r, s);
  if (tok < sr.a || tok >= sr.a + sr.n) return;
  const size_t zst = (size_t)r.n_rows * r.n_q_heads;
  float m = kMrefInit, l = 0.f;
  if (lane < zs) {
    m = a.part_ml[(lane * zst + rh) * 2];
    l = a.part_ml[(lane * zst + rh) * 2 + 1];
  }
  const float M = warp_max(m);
  const float f = lane < zs ? __builtin_amdgcn_exp2f(m - M) : 0.f;
  const float L = warp_sum(f * l);
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0.f;
  for (int z = 0; z < zs; ++z) {
    const float fz = __shfl(f, z, 64);
    const float* op = a.part_o + (z * zst + rh) * HD + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += fz * op[e];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int col = h * HD + lane * E + e;
    const size_t at = a.packed ? pa_index(tok, col, (size_t)a.ldo) : (size_t)tok * a.ldo + col;
    ((T*)a.out)[at] = Elem<T>::from_f32(L == 0.f ? 0.f : v[e] * inv);
  }
}

// ------------------------------------------------------------------ host
constexpr int kRowsNT = 1;
constexpr int kRowsNW = 4;

static long rows_blocks(const PagedAttnArgs& a, bool shared, int rb) {
  const PagedRows& r = a.r;
  const int G = r.n_q_heads / r.n_kv_heads;
  if (shared) return ((long)r.n_rows * G + rb - 1) / rb;
  if (r.row_start) return (long)r.n_rows * G / rb + r.n_seqs;
  return (long)r.n_seqs * (((long)r.rows_each * G + rb - 1) / rb);
}

PagedPlan paged_plan(const PagedAttnArgs& a, int elem_bytes) {
  (void)elem_bytes;
  const PagedRows& r = a.r;
  PagedPlan p{1, 0};
  auto pick = [&](long units, long keys) {
    long s = (512 + units - 1) / units;
    const long most = keys / (2 * kStep * kRowsNW);
    if (s > most) s = most;
    return (int)(s < 1 ? 1 : s > 32 ? 32 : s);
  };
  long keys = a.max_kv - a.prefix;
  if (a.window > 0 && keys > (long)a.window + a.sinks + a.max_rows) keys = (long)a.window + a.sinks + a.max_rows;
  p.splits = pick(rows_blocks(a, false, 16 * kRowsNT) * r.n_kv_heads, keys);
  if (a.prefix > 0) p.shared = pick(rows_blocks(a, true, 16 * kRowsNT) * r.n_kv_heads, a.prefix);
  return p;
}

size_t paged_part_floats(const PagedAttnArgs& a, const PagedPlan& p, size_t* ml) {
  const size_t rows = p.z() > 1 ? (size_t)p.z() * a.r.n_rows * a.r.n_q_heads : 0;
  *ml = rows * 2;
  return rows * a.r.head_dim;
}

template <typename T, int HD>
static hipError_t attention_hd(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  const PagedRows& r = a.r;
  auto launch = [&](bool shared, int splits, int z0) {
    const long grid = rows_blocks(a, shared, 16 * kRowsNT) * splits * r.n_kv_heads;
    if (grid <= 0) return hipSuccess;
    if (grid > 0x7fffffffl) return hipErrorInvalidValue;
    RT_LAUNCH((paged_rows_kernel<T, HD, kRowsNT, kRowsNW>), dim3((unsigned)grid), dim3(64 * kRowsNW), 0, s, a,
              shared ? 1 : 0, splits, z0, p.z());
    return hipGetLastError();
  };
  hipError_t e = p.shared ? launch(true, p.shared, p.splits) : hipSuccess;
  if (e == hipSuccess) e = launch(false, p.splits, 0);
  if (e != hipSuccess || p.z() == 1) return e;
  const long rows = (long)r.n_rows * r.n_q_heads;
  RT_LAUNCH((paged_merge_kernel<T, HD>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a, p.z());
  return hipGetLastError();
}
template <typename T>
hipError_t paged_attention(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (a.r.n_rows <= 0 || a.r.n_seqs <= 0) return hipSuccess;
  return a.r.head_dim == 128 ? attention_hd<T, 128>(a, p, s) : attention_hd<T, 64>(a, p, s);
}
template hipError_t paged_attention<bf16_t>(const PagedAttnArgs&, const PagedPlan&, hipStream_t);
template hipError_t paged_attention<float>(const PagedAttnArgs&, const PagedPlan&, hipStream_t);

}  // namespace rt
