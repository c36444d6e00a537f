// Appending rows to the paged KV cache, with the per-head RMSNorm and the position rotation
// applied on the way, and the same for the rows' queries.
//
//   y = x / sqrt(mean(x^2) + eps) * w                        (with norm weights w)
//   z_j = y_j cos(p, j) - y_{j + r/2} sin(p, j),  z_{j + r/2} = y_{j + r/2} cos(p, j) + y_j sin(p, j)
//
// for j < r / 2, r = rot_dim, p the row's position; elements r and up stay.  All in fp32,
// rounded once to the storage type.  Bound by memory: every row is read and written once.
#include "paged.h"

namespace rt {

// Eight consecutive elements as floats.
template <typename S>
__device__ __forceinline__ void load8(const S* p, float (&v)[8]) {
  Frag<S> f;
  f.load(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = f.get(e);
}

// One head's vector over LPV = hd / 16 lanes: lane c holds the runs of eight elements at o0 and
// o1, which rotate with each other where 8c < rot / 2 (partners rot / 2 apart) and lie behind
// the rotated part otherwise.
struct Runs { int o0, o1; bool rot; };
__device__ __forceinline__ Runs runs_of(int c, int rot) {
  const int nr = rot >> 4;
  if (c < nr) return Runs{8 * c, (rot >> 1) + 8 * c, true};
  return Runs{16 * c, 16 * c + 8, false};
}
template <int LPV>
__device__ __forceinline__ void norm_rotate(float (&x0)[8], float (&x1)[8], bool norm, const float (&w0)[8],
                                            const float (&w1)[8], float eps, bool rot, const float (&cs)[8],
                                            const float (&sn)[8]) {
  if (norm) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x0[e] * x0[e] + x1[e] * x1[e];
#pragma unroll
    for (int o = LPV / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
    const float inv = 1.0f / sqrtf(ss / (float)(16 * LPV) + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x0[e] *= inv * w0[e];
      x1[e] *= inv * w1[e];
    }
  }
  if (rot) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x0[e], b = x1[e];
      x0[e] = a * cs[e] - b * sn[e];
      x1[e] = b * cs[e] + a * sn[e];
    }
  }
}

// Workgroups 0 .. n_kv-1: one page item (the rows of one sequence that fall into one page) and
// one KV head each, so that a page's V is turned in registers and leaves as whole lines; the rest: queries, one
// wave per row and group of 64 / LPV heads, whose loads go out before the row's position is known (two
// prompts of 8192..16384 rows, 32 heads over 8 of 128, 554 MB: 117 -> 112 us, 4.93 TB/s; with four groups of
// heads a wave 120).
template <typename T, typename S, int HD>
__global__ __launch_bounds__(2 * HD) void append_kernel(AppendArgs a, int n_kv) {
  constexpr int LPV = HD / 16;              // lanes per head vector
  constexpr int VPW = 64 / LPV;             // head vectors per wave
  constexpr int NT = 2 * HD;                // threads: 16 rows x LPV lanes for K, as many for V
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 63;
  const int c = threadIdx.x % LPV;
  const Runs u = runs_of(c, a.cos ? a.rot_dim : 0);
  const long cap = (long)r.max_pages * kPage;
  auto store8 = [&](T* p, const float (&v)[8]) {
    Frag<T> f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.set(e, v[e]);
    f.store(p);
  };
  // a head's vector x, with norm weights w (or null) and at position pos, to dst where live
  auto turn = [&](const Frag<S> (&x)[2], long pos, const void* w, bool live, T* dst) {
    const bool rot = a.cos && u.rot;
    float w0[8], w1[8], fc[8], fs[8];
    if (w) {
      load8((const T*)w + u.o0, w0);
      load8((const T*)w + u.o1, w1);
    }
    if (rot) {
      load8(a.cos + (size_t)pos * (a.rot_dim / 2) + 8 * c, fc);
      load8(a.sin + (size_t)pos * (a.rot_dim / 2) + 8 * c, fs);
    }
    float x0[8], x1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x0[e] = x[0].get(e);
      x1[e] = x[1].get(e);
    }
    norm_rotate<LPV>(x0, x1, w != nullptr, w0, w1, a.eps, rot, fc, fs);
    if (!live) return;
    store8(dst + u.o0, x0);
    store8(dst + u.o1, x1);
  };
  if ((int)blockIdx.x >= n_kv) {                                  // queries
    const int groups = (r.n_q_heads + VPW - 1) / VPW;
    const int unit = ((int)blockIdx.x - n_kv) * (NT / 64) + (int)(threadIdx.x >> 6);
    const int row = unit / groups, h = unit % groups * VPW + lane / LPV;
    if (row >= r.n_rows) return;
    const bool live = h < r.n_q_heads;
    const int hh = live ? h : 0;
    const S* src = (const S*)a.q + (size_t)row * a.ldq + (size_t)hh * HD;
    Frag<S> x[2];                         // (under way while the row's position is found)
    x[0].load(src + u.o0);
    x[1].load(src + u.o1);
    const int s = row_seq(r, row);
    if (s >= r.n_seqs) return;
    const SeqRows sr = seq_rows(r, s);
    const long pos = (long)sr.keys - sr.n + (row - sr.a);
    if (row < sr.a || row >= sr.a + sr.n || pos < 0 || pos >= cap) return;
    turn(x, pos, a.q_norm, live, (T*)a.q_out + (size_t)row * a.ldqo + (size_t)hh * HD);
    return;
  }
  const int kvh = (int)blockIdx.x % r.n_kv_heads, item = (int)blockIdx.x / r.n_kv_heads;
  // pages that the rows of sequence s meet
  auto pages_of = [&](int s) {
    const SeqRows q = seq_rows(r, s);
    const long p0 = max((long)q.keys - q.n, 0l), p1 = min((long)q.keys, cap);
    return p1 > p0 ? (int)((p1 - 1) / kPage - p0 / kPage) + 1 : 0;
  };
  int s, in;
  if (!find_block(r.n_seqs, item, pages_of, s, in)) return;
  const SeqRows sr = seq_rows(r, s);
  const long p0 = max((long)sr.keys - sr.n, 0l), p1 = min((long)sr.keys, cap);
  const long pg = p0 / kPage + in;
  const int lo = (int)(max(p0, pg * kPage) - pg * kPage), hi = (int)(min(p1, (pg + 1) * kPage) - pg * kPage);
  const int page = r.page_table[(size_t)s * r.max_pages + pg];
  if (page < 0 || page >= r.n_pages) return;
  const int row0 = sr.a + (int)(pg * kPage - ((long)sr.keys - sr.n));   // row of the page's slot 0
  const size_t base = ((size_t)page * r.n_kv_heads + kvh) * (size_t)(kPage * HD);
  if (threadIdx.x < NT / 2) {                                     // K: slot t, LPV lanes
    const int t = threadIdx.x / LPV;
    if (t < lo || t >= hi) return;        // (whole LPV groups leave together)
    const S* src = (const S*)a.ks + (size_t)(row0 + t) * a.ldk + (size_t)kvh * HD;
    Frag<S> x[2];
    x[0].load(src + u.o0);
    x[1].load(src + u.o1);
    turn(x, pg * kPage + t, a.k_norm, true, (T*)r.k + base + (size_t)t * HD);
  } else {                                                        // V: element d of every slot
    const int d = threadIdx.x - NT / 2;
    T* dst = (T*)r.v + base + (size_t)d * kPage;
    const S* src = (const S*)a.vs + (long)row0 * a.ldv + (long)kvh * HD + d;   // (slots below lo: not read)
    if (hi - lo == 1) {
      dst[lo] = Elem<T>::from_f32(Elem<S>::to_f32(src[(long)lo * a.ldv]));
      return;
    }
    // all rows' elements are under way before the first is stored (8 sequences of 16 rows that end
    // inside pages: 4.7 us, 5.7 with a loop of loads and stores)
    float v[2][8];
#pragma unroll
    for (int t = 0; t < kPage; ++t) v[t >> 3][t & 7] = Elem<S>::to_f32(src[(long)min(max(t, lo), hi - 1) * a.ldv]);
    if (hi - lo == kPage) {
      store8(dst, v[0]);
      store8(dst + 8, v[1]);
    } else {
#pragma unroll
      for (int t = 0; t < kPage; ++t)
        if (t >= lo && t < hi) dst[t] = Elem<T>::from_f32(v[t >> 3][t & 7]);
    }
  }
}

template <typename T, typename S>
hipError_t paged_append(const AppendArgs& a, hipStream_t s) {
  const PagedRows& r = a.r;
  if (r.n_rows <= 0 || r.n_seqs <= 0) return hipSuccess;
  // page items: a sequence of n rows meets at most (n + 14) / 16 + 1 pages
  const long items = r.row_start ? (long)r.n_rows / kPage + 2l * r.n_seqs
                                 : (long)r.n_seqs * ((r.rows_each + 14) / kPage + 1);
  const long n_kv = items * r.n_kv_heads;
  const int vpw = 1024 / r.head_dim, wpg = r.head_dim / 32;
  const long units = a.q ? (long)r.n_rows * ((r.n_q_heads + vpw - 1) / vpw) : 0;
  const long grid = n_kv + (units + wpg - 1) / wpg;
  if (grid > kMaxGrid) return hipErrorInvalidValue;
  if (r.head_dim == 128) RT_LAUNCH((append_kernel<T, S, 128>), dim3((unsigned)grid), dim3(256), 0, s, a, (int)n_kv);
  else RT_LAUNCH((append_kernel<T, S, 64>), dim3((unsigned)grid), dim3(128), 0, s, a, (int)n_kv);
  return hipGetLastError();
}
template hipError_t paged_append<bf16_t, bf16_t>(const AppendArgs&, hipStream_t);
template hipError_t paged_append<bf16_t, float>(const AppendArgs&, hipStream_t);
template hipError_t paged_append<float, float>(const AppendArgs&, hipStream_t);

}  // namespace rt
