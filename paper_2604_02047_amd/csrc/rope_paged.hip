// q | k | v of the new rows on their way into a paged cache, one launch for all requests: the split-K slices of the projection are
// summed, every head of q and k is normalised over its d columns where the model does that (x * rsqrt(mean(x^2) + eps) * g), the pairs
// (a, b) = (x_j, x_{j + d/2}) become (a cos - b sin, b cos + a sin) with the angle pos * base^(-2j/d), queries go out as rows, k and v
// into slots len + i of the sequence's pages.
//
// It reads ks * rows * (n_heads + 2 n_kv) * d floats once and writes half a slice's bytes: nothing is reused, so memory bounds it
// when there are many rows, and one trip to memory (plus the table's: length -> entry -> count) when there are few.  Two kinds of
// workgroups: 16 query heads of one row; and one KV head of eight slots that begin at a multiple of eight, because in the
// operand order eight consecutive slots of a value column are 16 contiguous bytes and the key chunks of four are 64.
// Measured (kernel trace): 16 requests x 32, 32 + 2 x 8 heads of 128, 4 slices: 11.3 us (57 MB: 5.0 TB/s); one row: 4.4 us (latency);
// 5 ragged requests of 7B heads, 2 slices: 6.5 us (4.5 at a large copy's rate; the K and V rows are asked for behind length, entry and count).
#include "mma16.h"
#include "paged.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int Q_HEADS = 16;  // query heads a workgroup takes of one row: D / 8 threads each

struct RopePagedArgs {
  const float* part;
  size_t split_stride, ld;
  const double* inv_freq;
  const void* gq;
  const void* gk;
  void* q;
  size_t ldq;
  void* kpool;  // of the layer
  void* vpool;
  const int32_t* table;
  const int32_t* len;
  const int32_t* refs;
  int32_t* flags;
  int32_t ks, n_heads, n_kv, table_ld, n_pages, q_parts, q_groups;
  float eps;
};

// (cos, sin) of pos * freq: reduced in double, evaluated in float (|error| ~ 1e-7 rad at any position)
__device__ inline float2 angle(int pos, double freq) {
  double ang = (double)pos * freq;
  const double two_pi = 6.283185307179586476925286766559;
  ang -= two_pi * rint(ang / two_pi);
  float sn, c;
  sincosf((float)ang, &sn, &c);
  return make_float2(c, sn);
}

// Sum of the slices at p, in their order; four of both halves in flight together.
__device__ inline void sum_slices(const float* p, size_t stride, int ks, int half, f32x4& lo, f32x4& hi) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  lo = zero;
  hi = zero;
  for (int s = 0; s < ks; s += 4) {
    f32x4 a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float* at = p + (size_t)(s + k < ks ? s + k : s) * stride;
      a[k] = *reinterpret_cast<const f32x4*>(at);
      b[k] = *reinterpret_cast<const f32x4*>(at + half);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (s + k < ks) { lo += a[k]; hi += b[k]; }
  }
}

template <int D, bool F16, bool NORM>
__global__ __launch_bounds__(2 * D) void k_rope_paged(const RopePagedArgs a, const PagedReqs rq, int q_terms) {
  typedef typename Mma16<F16>::T T;
  typedef typename Mma16<F16>::v4 op4;
  typedef typename Mma16<F16>::v8 op8;
  constexpr int HALF = D / 2, TPH = D / 8;  // threads per head: four columns and their partners each
  __shared__ float2 cs[8][HALF];
  const int tid = threadIdx.x;
  const int lane_h = tid % TPH, j0 = lane_h * 4;
  auto norm_rotate = [&](f32x4& lo, f32x4& hi, const void* gain, const float2* c) {
    if (NORM) {
      const T* g = static_cast<const T*>(gain);
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) ss += lo[e] * lo[e] + hi[e] * hi[e];
#pragma unroll
      for (int off = 1; off < TPH; off <<= 1) ss += __shfl_xor(ss, off, 64);  // the head's threads are neighbours
      const float rstd = 1.0f / sqrtf(ss / (float)D + a.eps);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] *= rstd * (float)g[j0 + e];
        hi[e] *= rstd * (float)g[j0 + HALF + e];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 w = c[j0 + e];
      const float x = lo[e], y = hi[e];
      lo[e] = x * w.x - y * w.y;
      hi[e] = y * w.x + x * w.y;
    }
  };

  if ((int)blockIdx.x < a.q_groups) {
    // ---- Q_HEADS query heads of one row
    const int row_c = (int)blockIdx.x / a.q_parts, part = (int)blockIdx.x - row_c * a.q_parts;
    int r = 0;
    while (r + 1 < rq.n && row_c >= rq.r[r + 1].c0) ++r;
    const int node = row_c - rq.r[r].c0;
    const size_t row = (size_t)rq.r[r].row0 + node;
    const int h = part * Q_HEADS + tid / TPH;
    f32x4 lo, hi;
    const int hc = h < a.n_heads ? h : a.n_heads - 1;  // (threads behind the last head: loads stay inside, nothing is stored)
    const int32_t* const at = static_cast<const int32_t*>(rq.r[r].p);
    const int pos = at ? at[node] : a.len[rq.r[r].seq] + node;
    sum_slices(a.part + row * a.ld + hc * D + j0, a.split_stride, a.ks, HALF, lo, hi);
    if (tid < HALF) cs[0][tid] = angle(pos, a.inv_freq[tid]);
    __syncthreads();
    norm_rotate(lo, hi, a.gq, cs[0]);
    if (h >= a.n_heads) return;
    op4 l, u;
#pragma unroll
    for (int e = 0; e < 4; ++e) { l[e] = (T)lo[e]; u[e] = (T)hi[e]; }
    T* out = static_cast<T*>(a.q) + row * a.ldq;
    const size_t pl = term_pos(q_terms, h * D + j0), pu = term_pos(q_terms, h * D + HALF + j0);
    *reinterpret_cast<op4*>(out + pl) = l;
    *reinterpret_cast<op4*>(out + pu) = u;
    if (q_terms == 2) {
      // a query's rounding error is shared by all scores of its row and does not average out over the keys: under
      // bf16 the second term takes it from 2^-9 to 2^-17
#pragma unroll
      for (int e = 0; e < 4; ++e) { l[e] = (T)(lo[e] - (float)l[e]); u[e] = (T)(hi[e] - (float)u[e]); }
      *reinterpret_cast<op4*>(out + pl + 8) = l;
      *reinterpret_cast<op4*>(out + pu + 8) = u;
    }
    return;
  }

  // ---- one KV head of the slots 8 G .. 8 G + 7 that belong to the tree
  int x = (int)blockIdx.x - a.q_groups;
  const int kvh = x % a.n_kv;
  x /= a.n_kv;
  int r = 0;
  for (;; ++r) {  // a request has (B + 14) / 8 groups at most
    const int g = (rq.r[r].B + 14) / 8;
    if (x < g) break;
    x -= g;
  }
  const PagedReq& q = rq.r[r];
  const int32_t* pos = static_cast<const int32_t*>(q.p);
  int P = a.len[q.seq];
  if (P < 0 || P > q.P_max) {  // (P_max + B fits the table: checked on the host)
    if (tid == 0) atomicOr(a.flags, GOOSE_FLAG_CAPACITY);
    return;
  }
  const int G = (P >> 3) + x, s0 = G << 3;  // first slot of the group, and its tree node (negative: slots in front of the tree)
  const int i0 = s0 - P;
  if (i0 >= q.B) return;
  const int page = a.table[(size_t)q.seq * a.table_ld + (s0 >> 6)];
  if ((unsigned)page >= (unsigned)a.n_pages || a.refs[page] != 1) {
    if (tid == 0) atomicOr(a.flags, GOOSE_FLAG_PAGES);
    return;
  }
  for (int t = tid; t < 8 * HALF; t += 2 * D) {
    const int i = i0 + t / HALF;
    if (i >= 0 && i < q.B) cs[t / HALF][t % HALF] = angle(pos ? pos[i] : P + i, a.inv_freq[t % HALF]);
  }
  const size_t head = page_head<D>(page, a.n_kv, kvh);
  const int kcol = (a.n_heads + kvh) * D, vcol = kcol + a.n_kv * D;
  const int slot = s0 & 63;  // of the page
  if (tid < D) {
    // keys: thread = (slot, four columns and their partners)
    const int u = tid / TPH, i = i0 + u;
    const bool on = i >= 0 && i < q.B;
    const int ic = i < 0 ? 0 : (i < q.B ? i : q.B - 1);
    f32x4 lo, hi;
    sum_slices(a.part + (size_t)(q.row0 + ic) * a.ld + kcol + j0, a.split_stride, a.ks, HALF, lo, hi);
    __syncthreads();
    norm_rotate(lo, hi, a.gk, cs[u]);
    if (!on) return;
    op4 l, h;
#pragma unroll
    for (int e = 0; e < 4; ++e) { l[e] = (T)lo[e]; h[e] = (T)hi[e]; }
    T* kp = static_cast<T*>(a.kpool) + head;
    *reinterpret_cast<op4*>(kp + page_k_chunk<D>(slot + u, j0 >> 3) + (j0 & 7)) = l;
    *reinterpret_cast<op4*>(kp + page_k_chunk<D>(slot + u, (j0 + HALF) >> 3) + (j0 & 7)) = h;
  } else {
    // values: thread = column, eight slots; the slices in their order
    const int c = tid - D;
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = 0.f;
    const float* p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = i0 + u;
      p[u] = a.part + (size_t)(q.row0 + (i < 0 ? 0 : (i < q.B ? i : q.B - 1))) * a.ld + vcol + c;
    }
    for (int s = 0; s < a.ks; ++s) {
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] += p[u][(size_t)s * a.split_stride];
    }
    __syncthreads();
    T* dst = static_cast<T*>(a.vpool) + head + page_v_elem<D>(slot, c);
    op8 w;
#pragma unroll
    for (int u = 0; u < 8; ++u) w[u] = (T)v[u];
    if (i0 >= 0 && i0 + 8 <= q.B) {
      *reinterpret_cast<op8*>(dst) = w;
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u >= 0 && i0 + u < q.B) dst[u] = w[u];
    }
  }
}

template <int D, bool F16>
int launch_d(dim3 grid, bool norm, const RopePagedArgs& a, const PagedReqs& rq, int q_terms, hipStream_t st) {
  if (norm) hipLaunchKernelGGL((k_rope_paged<D, F16, true>), grid, dim3(2 * D), 0, st, a, rq, q_terms);
  else hipLaunchKernelGGL((k_rope_paged<D, F16, false>), grid, dim3(2 * D), 0, st, a, rq, q_terms);
  return goose_launch_status();
}

}  // namespace

int launch_rope_paged(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const double* inv_freq, float eps,
                      const float* part, int ks, size_t split_stride, size_t ld, const void* gq, const void* gk, const PagedReqs& rq,
                      void* q, size_t ldq, int q_terms, int32_t* flags, hipStream_t st) {
  const size_t layer0 = (size_t)layer * page_layer_elems(pg, n_kv, head_dim) * 2;  // bytes
  RopePagedArgs a;
  a.part = part;
  a.split_stride = split_stride;
  a.ld = ld;
  a.inv_freq = inv_freq;
  a.gq = gq;
  a.gk = gk;
  a.q = q;
  a.ldq = ldq;
  a.kpool = static_cast<char*>(pg.d_kpool) + layer0;
  a.vpool = static_cast<char*>(pg.d_vpool) + layer0;
  a.table = pg.d_table;
  a.len = pg.d_len;
  a.refs = pg.d_refs;
  a.flags = flags;
  a.ks = ks;
  a.n_heads = n_heads;
  a.n_kv = n_kv;
  a.table_ld = pg.table_ld;
  a.n_pages = pg.n_pages;
  a.q_parts = (n_heads + Q_HEADS - 1) / Q_HEADS;
  a.q_groups = rq.rows * a.q_parts;
  a.eps = eps;
  int kv_groups = 0;
  for (int r = 0; r < rq.n; ++r) kv_groups += (rq.r[r].B + 14) / 8;
  const dim3 grid(a.q_groups + kv_groups * n_kv);
  const bool f16 = dtype == GOOSE_DTYPE_F16, norm = gq != nullptr;
  if (head_dim == 128)
    return f16 ? launch_d<128, true>(grid, norm, a, rq, q_terms, st) : launch_d<128, false>(grid, norm, a, rq, q_terms, st);
  if (head_dim == 64)
    return f16 ? launch_d<64, true>(grid, norm, a, rq, q_terms, st) : launch_d<64, false>(grid, norm, a, rq, q_terms, st);
  return GOOSE_ERR_SHAPE;
}
