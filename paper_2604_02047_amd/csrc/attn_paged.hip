// Tree attention of up to 16 requests over a paged cache; the pages that all of them share are read once for the rows of all.
//
//   o[row, h] = sum_k softmax_k(q[row, h] . K[k] / sqrt(d)) V[k],   k over the slots that the row sees.
//
// Softmax is associative over sets of keys: with (m, l, O) = (max, sum of 2^(s - m), sum of 2^(s - m) V) of a set, two sets join as
// m = max(m1, m2), l = 2^(m1 - m) l1 + 2^(m2 - m) l2, O likewise.  So the shared keys and a request's own ones are
// separate work items, and either kind is split along the keys as far as it takes to fill the card; k_paged_merge joins what
// the items of a row left, in a fixed order.
//
// The rows of one KV head -- (node, query head of the group), for the shared keys of all requests one behind the other -- are the columns of
// 32-wide matrix-instruction tiles: a single token of a grouped-query model fills 4 of 32 columns with its four heads,
// and sixteen of them share two tiles over the common prefix.  Per 32 keys and 32 rows, as in the contiguous attention:
// S^T = K Q^T, online softmax with two lanes a row, O^T += V^T P^T, operands straight from the pages' operand order.
#include "mma16.h"
#include "paged.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));

__device__ inline unsigned short out_bits16(float f, bool f16) {
  return f16 ? __builtin_bit_cast(unsigned short, (_Float16)f) : __builtin_bit_cast(unsigned short, (__bf16)f);
}
__device__ inline float out_back16(unsigned short b, bool f16) {
  return f16 ? (float)__builtin_bit_cast(_Float16, b) : (float)__builtin_bit_cast(__bf16, b);
}

struct AttnReq {
  int32_t seq, B, P_max, row0, c0;
  int32_t tiles, splits;  // work items over its own keys: tiles x splits, for every KV head
  const uint64_t* mask;
};
struct PagedAttnArgs {
  const void* kpool;  // of the layer
  const void* vpool;
  const int32_t* table;
  const int32_t* len;
  const void* q;
  float* ws_o;    // [split][head][row][d]; splits of the shared keys first
  float* ws_ml;   // [split][head][row][2]
  unsigned short* o;
  int32_t* flags;
  size_t ldq, ldo;
  int32_t table_ld, n_pages, n_heads, n_kv, group, rows, n_req;
  int32_t sh_blocks, sh_tiles, sh_splits;  // shared keys: 32-slot blocks, row tiles, splits
  int32_t direct;                          // every row has one item: it writes o itself
  int32_t o_terms, o_f16;
  AttnReq r[GOOSE_MAX_REQUESTS];
};

// Four neighbouring columns (inside one group of eight) of an output row.
__device__ inline void store_out(const PagedAttnArgs& a, size_t row, int col, const f32x4& x) {
  u16x4 v, v2;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = out_bits16(x[e], a.o_f16);
    v2[e] = out_bits16(x[e] - out_back16(v[e], a.o_f16), a.o_f16);
  }
  unsigned short* dst = a.o + row * a.ldo + term_pos(a.o_terms, col);
  *reinterpret_cast<u16x4*>(dst) = v;
  if (a.o_terms == 2) *reinterpret_cast<u16x4*>(dst + 8) = v2;
}

// The maximum as the exponent's reference: a row that has seen nothing (or only scores of -infinity) takes 0, so that 2^(-inf - 0) = 0.
__device__ inline float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

// Which keys of the 16 from tree node j0 on (negative: committed slots, visible) a mask row shows.
__device__ inline unsigned window16(uint64_t w0, uint64_t w1, int j0) {
  if (j0 <= -16) return 0xFFFFu;
  if (j0 < 0) return (unsigned)(((1u << -j0) - 1u) | (unsigned)(w0 << -j0)) & 0xFFFFu;
  if (j0 >= 128) return 0;
  uint64_t x = j0 < 64 ? w0 >> j0 : w1 >> (j0 - 64);
  if (j0 > 48 && j0 < 64) x |= w1 << (64 - j0);
  return (unsigned)x & 0xFFFFu;
}

// One workgroup = a tile of 32 rows x a range of 32-slot blocks, dealt to four wavefronts in contiguous quarters; every wavefront streams
// its blocks global -> registers -> matrix cores (no barrier in the loop), the next block's keys and values requested as
// soon as the current ones have been used.
template <int D, int TERMS, bool F16>
__global__ __launch_bounds__(256, 2) void k_attn_paged(const PagedAttnArgs a) {
  typedef typename Mma16<F16>::T T;
  typedef typename Mma16<F16>::v8 op8;
  constexpr int NG = 4, NS = D / 16, QUADS = D / 8, QPW = QUADS / NG;
  constexpr int WFLOATS = (QUADS + 1) * 256;  // a wavefront's state at the merge
  constexpr int QL_BYTES = TERMS == 2 ? NS * 1024 : 0;
  __shared__ __attribute__((aligned(16))) unsigned char lds[NG * WFLOATS * 4 + QL_BYTES];
  unsigned char* const ql_lds = lds + NG * WFLOATS * 4;
  const int tid = threadIdx.x, lane = tid & 63, g = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x;  // the fast index: where 8 divides the KV heads, all items of a head run on one XCD and find each other's blocks in its L2
  // ---- the item
  int y = blockIdx.y, tile, split, nsplit, rec_split, ri = 0, b_first, n_blocks, P = 0, B = 0;
  const bool shared = y < a.sh_tiles * a.sh_splits;
  if (shared) {
    split = (int)((unsigned)y / (unsigned)a.sh_tiles);
    tile = y - split * a.sh_tiles;
    nsplit = a.sh_splits;
    rec_split = split;
    b_first = 0;
    n_blocks = a.sh_blocks;
  } else {
    y -= a.sh_tiles * a.sh_splits;
    while (y >= a.r[ri].tiles * a.r[ri].splits) { y -= a.r[ri].tiles * a.r[ri].splits; ++ri; }
    split = (int)((unsigned)y / (unsigned)a.r[ri].tiles);
    tile = y - split * a.r[ri].tiles;
    nsplit = a.r[ri].splits;
    rec_split = a.sh_splits + split;
    b_first = a.sh_blocks;
    B = a.r[ri].B;
    P = a.len[a.r[ri].seq];
    const int S = a.sh_blocks * 32;
    if ((P < S || P > a.r[ri].P_max) && tid == 0 && kvh == 0 && y == 0) atomicOr(a.flags, GOOSE_FLAG_CAPACITY);
    P = min(max(P, S), a.r[ri].P_max);  // (P_max + B <= 64 table_ld, S <= P_max: checked on the host)
    n_blocks = ((P + B + 31) >> 5) - b_first;
  }
  // ---- this lane's row
  const int rho = tile * 32 + l31;
  const int node = (int)((unsigned)rho / (unsigned)a.group), hg = rho - node * a.group;
  int crow, row;
  bool live;
  if (shared) {
    live = node < a.rows;
    crow = live ? node : 0;
    int r = 0;
    while (r + 1 < a.n_req && crow >= a.r[r + 1].c0) ++r;
    row = a.r[r].row0 + crow - a.r[r].c0;
  } else {
    live = node < B;
    crow = a.r[ri].c0 + (live ? node : 0);
    row = a.r[ri].row0 + (live ? node : 0);
  }
  const int h = kvh * a.group + hg;
  // ---- the queries
  op8 qf[NS];
  {
    const T* qp = static_cast<const T*>(a.q) + (size_t)row * a.ldq + (size_t)h * D * TERMS + hh * 8 * TERMS;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const op8*>(qp + s * 16 * TERMS);
    if (TERMS == 2) {
      // the second term in LDS, one copy for the four wavefronts (each brings a quarter)
#pragma unroll
      for (int s = 0; s < NS / NG; ++s)
        *reinterpret_cast<op8*>(ql_lds + ((g * (NS / NG) + s) * 64 + lane) * 16) =
            *reinterpret_cast<const op8*>(qp + (g * (NS / NG) + s) * 32 + 8);
      __syncthreads();
    }
  }
  uint64_t mw0 = 0, mw1 = 0;
  if (!shared && live) {
    const int W = (B + 63) >> 6;
    mw0 = a.r[ri].mask[(size_t)node * W];
    if (W > 1) mw1 = a.r[ri].mask[(size_t)node * W + 1];
    if (B < 64) mw0 &= (1ull << B) - 1;  // bits at or beyond B count as clear
    if (B < 128) mw1 &= B > 64 ? (1ull << (B - 64)) - 1 : 0;
  }
  // ---- this wavefront's blocks
  const int i_lo = (int)((long long)n_blocks * split / nsplit), i_hi = (int)((long long)n_blocks * (split + 1) / nsplit);
  const int n_wg = i_hi - i_lo;
  const int b0 = b_first + i_lo + n_wg * g / NG, total = b_first + i_lo + n_wg * (g + 1) / NG - b0;
  const int32_t* trow = a.table + (size_t)a.r[ri].seq * a.table_ld;  // (shared: any request's table will do)
  // Page ids, 64 of them a register (one a lane); an entry out of range reads page 0
  int pg_base = b0 >> 1, pg_ids = 0;
  const int pg_last = (b0 + total - 1) >> 1;
  auto load_ids = [&]() {
    const int e = pg_base + lane;
    pg_ids = e <= pg_last ? trow[e] : 0;
    if ((unsigned)pg_ids >= (unsigned)a.n_pages) { atomicOr(a.flags, GOOSE_FLAG_PAGES); pg_ids = 0; }
  };
  if (total > 0) load_ids();
  const size_t head_elems = (size_t)GOOSE_PAGE * D;
  auto block_at = [&](int idx) -> size_t {  // element offset of block idx in a layer's pool
    const int b = b0 + idx;
    if ((b >> 1) - pg_base >= 64) { pg_base = b >> 1; load_ids(); }
    const int page = __builtin_amdgcn_readlane(pg_ids, (b >> 1) - pg_base);
    return ((size_t)page * a.n_kv + kvh) * head_elems + (size_t)(b & 1) * 32 * D;
  };
  const T* const kp = static_cast<const T*>(a.kpool);
  const T* const vp = static_cast<const T*>(a.vpool);
  u32x4 kreg[NS], vreg[NS];
  auto fetch = [&](const T* pool, size_t at, u32x4 (&dst)[NS]) {
    const u32x4* p = reinterpret_cast<const u32x4*>(pool + at) + lane;
#pragma unroll
    for (int s = 0; s < NS; ++s) dst[s] = p[s * 64];
  };
  size_t at = 0;
  if (total > 0) {
    at = block_at(0);
    fetch(kp, at, kreg);
    fetch(vp, at, vreg);
  }
  f32x16 oacc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float scale = 1.4426950408889634f / sqrtf((float)D);  // log2(e) / sqrt(d): softmax in base 2

  for (int idx = 0; idx < total; ++idx) {
    const size_t here = at;
    const int slot0 = (b0 + idx) * 32;
    const bool tree = !shared && slot0 + 32 > P;  // wavefront-uniform
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) s = Mma16<F16>::mfma(__builtin_bit_cast(op8, kreg[k]), qf[k], s);
    if (TERMS == 2) {
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const op8 ql = *reinterpret_cast<const op8*>(ql_lds + (k * 64 + lane) * 16);
        s = Mma16<F16>::mfma(__builtin_bit_cast(op8, kreg[k]), ql, s);
      }
    }
    if (idx + 1 < total) { at = block_at(idx + 1); fetch(kp, at, kreg); }
    unsigned vis = 0xFFFFu;
    if (tree) {
      vis = window16(mw0, mw1, slot0 + hh * 16 - P);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = ((vis >> r) & 1u) ? s[r] : -INFINITY;
    }
    float tmax = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] *= scale;
      tmax = fmaxf(tmax, s[r]);
    }
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
    const bool grew = tmax > m_run;
    const float m_new = fmaxf(m_run, tmax), ref = finite_ref(m_new);
    const float alpha = __builtin_amdgcn_exp2f(m_run - ref);
    m_run = m_new;
    float psum = 0.f;
    op8 pf[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = __builtin_amdgcn_exp2f(s[r] - ref);
      s[r] = p;
      psum += p;
      pf[r >> 3][r & 7] = (T)p;
    }
    // the running maximum settles after a few blocks: skip the rescale when no lane's maximum grew
    if (__builtin_amdgcn_ballot_w64(grew) != 0) {
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
    }
    l_run += psum;
    bool odd = false;
    if (tree) {
      // slots behind the tree may hold anything: their values become zero.  A NaN or an infinity in the value of a node that
      // some rows do not see would reach them as 0 * NaN through the matrix instruction.
      const int mine = P + B - slot0 - hh * 16;  // of this lane's 16 keys, the first `mine` exist
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        u16x8 e = __builtin_bit_cast(u16x8, vreg[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if ((k & 1) * 8 + i >= mine) e[i] = 0;
          constexpr unsigned short EXP = F16 ? 0x7C00 : 0x7F80;
          odd = odd || (e[i] & EXP) == EXP;
        }
        vreg[k] = __builtin_bit_cast(u32x4, e);
      }
    }
    if (tree && __builtin_amdgcn_ballot_w64(odd) != 0) {
      // rare: key by key, skipping the pairs that are masked.  The probabilities go through this wavefront's part of the merge buffer.
      float* const pl = reinterpret_cast<float*>(lds) + (size_t)g * WFLOATS;
#pragma unroll
      for (int r = 0; r < 16; ++r) pl[(hh * 16 + r) * 33 + l31] = ((vis >> r) & 1u) ? (float)(T)s[r] : -1.f;
      const int n_keys = min(32, P + B - slot0);
      for (int kk = 0; kk < n_keys; ++kk) {
        const float p = pl[kk * 33 + l31];
        const T* col = vp + here + (((kk >> 3) & 1) * 64 + 32 * (kk >> 4)) * 8 + (kk & 7);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float v = (float)col[(dt * 128 + 8 * (r >> 2) + 4 * hh + (r & 3)) * 8];
            oacc[dt][r] = p >= 0.f || p != p ? fmaf(p, v, oacc[dt][r]) : oacc[dt][r];
          }
      }
    } else {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          oacc[dt] = Mma16<F16>::mfma(__builtin_bit_cast(op8, vreg[dt * 2 + j]), pf[j], oacc[dt]);
    }
    if (idx + 1 < total) fetch(vp, at, vreg);
  }

  // ---- the four wavefronts' states join in one round through LDS: each leaves its own, then owns a quarter of the columns
  f32x4 res[QPW];
  float l_sum = 0.f;
  {
    float* dst = reinterpret_cast<float*>(lds) + (size_t)g * WFLOATS + lane * 4;
    *reinterpret_cast<f32x4*>(dst) = f32x4{m_run, l_run, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(dst + 256 * (1 + dt * 4 + q)) =
            f32x4{oacc[dt][q * 4], oacc[dt][q * 4 + 1], oacc[dt][q * 4 + 2], oacc[dt][q * 4 + 3]};
    __syncthreads();
    const float* src = reinterpret_cast<const float*>(lds) + lane * 4;
    float mj[NG], lj[NG];
    m_run = -INFINITY;
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const f32x4 ml = *reinterpret_cast<const f32x4*>(src + (size_t)j * WFLOATS);
      mj[j] = ml[0];
      lj[j] = ml[1];
      m_run = fmaxf(m_run, mj[j]);
    }
    const float ref = finite_ref(m_run);
#pragma unroll
    for (int q = 0; q < QPW; ++q) res[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const float w = __builtin_amdgcn_exp2f(mj[j] - ref);
      l_sum += w * lj[j];
#pragma unroll
      for (int q = 0; q < QPW; ++q)
        res[q] += w * *reinterpret_cast<const f32x4*>(src + (size_t)j * WFLOATS + 256 * (1 + g * QPW + q));
    }
  }
  const float l_tot = l_sum + __shfl_xor(l_sum, 32, 64);
  if (!shared && y == 0 && kvh == 0 && g == 0 && ri > 0) {
    // the shared pages must be the same in all tables: one wavefront a request compares them with the first request's
    const int32_t* t0 = a.table + (size_t)a.r[0].seq * a.table_ld;
    bool differs = false;
    for (int i = lane; i < a.sh_blocks / 2; i += 64) differs = differs || trow[i] != t0[i];
    if (differs) atomicOr(a.flags, GOOSE_FLAG_PAGES);
  }
  if (!live) return;
  // quad n of the accumulator = columns 8 n + 4 hh .. + 3
  if (a.direct) {
    const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
#pragma unroll
    for (int q = 0; q < QPW; ++q) store_out(a, row, h * D + (g * QPW + q) * 8 + hh * 4, res[q] * inv);
  } else {
    const size_t rec = ((size_t)rec_split * a.n_heads + h) * a.rows + crow;
    if (hh == 0 && g == 0) *reinterpret_cast<float2*>(a.ws_ml + rec * 2) = make_float2(m_run, l_tot);
    float* dst = a.ws_o + rec * D;
#pragma unroll
    for (int q = 0; q < QPW; ++q) *reinterpret_cast<f32x4*>(dst + (g * QPW + q) * 8 + hh * 4) = res[q];
  }
}

// Joins the items of a row: D / 4 threads a (row, head), four columns each, records in a fixed order, the loads of eight in flight together.
template <int D>
__global__ __launch_bounds__(256) void k_paged_merge(const PagedAttnArgs a) {
  constexpr int TPR = D / 4, CH = 8;
  const int it = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, c = (threadIdx.x % TPR) * 4;
  if (it >= a.rows * a.n_heads) return;
  const int h = (int)((unsigned)it / (unsigned)a.rows), crow = it - h * a.rows;
  int r = 0;
  while (r + 1 < a.n_req && crow >= a.r[r + 1].c0) ++r;
  const int n = a.sh_splits + a.r[r].splits;
  const size_t base = (size_t)h * a.rows + crow, step = (size_t)a.n_heads * a.rows;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f, m = -INFINITY;
  for (int s0 = 0; s0 < n; s0 += CH) {
    float2 ml[CH];
    f32x4 ov[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const size_t rec = base + (size_t)min(s0 + k, n - 1) * step;
      ml[k] = *reinterpret_cast<const float2*>(a.ws_ml + rec * 2);
      ov[k] = *reinterpret_cast<const f32x4*>(a.ws_o + rec * D + c);
    }
    float m_new = m;
#pragma unroll
    for (int k = 0; k < CH; ++k) m_new = fmaxf(m_new, ml[k].x);
    const float ref = finite_ref(m_new), w0 = __builtin_amdgcn_exp2f(m - ref);
    den *= w0;
    num *= w0;
    m = m_new;
#pragma unroll
    for (int k = 0; k < CH; ++k)
      if (s0 + k < n) {
        const float w = __builtin_amdgcn_exp2f(ml[k].x - ref);
        den = fmaf(w, ml[k].y, den);
        num += w * ov[k];
      }
  }
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  store_out(a, (size_t)a.r[r].row0 + crow - a.r[r].c0, h * D + c, num * inv);
}

template <int D, int TERMS>
void launch_t(bool f16, dim3 grid, const PagedAttnArgs& a, hipStream_t st) {
  if (f16) hipLaunchKernelGGL((k_attn_paged<D, TERMS, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_attn_paged<D, TERMS, false>), grid, dim3(256), 0, st, a);
}

}  // namespace

int launch_attn_paged(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const void* q, size_t ldq, int q_terms,
                      const PagedReqs& rq, int shared_pages, float* ws_o, float* ws_ml, size_t max_records, void* o, size_t ldo,
                      int o_dtype, int o_terms, int32_t* flags, hipStream_t st) {
  if (head_dim != 64 && head_dim != 128) return GOOSE_ERR_SHAPE;
  const size_t layer0 = (size_t)layer * page_layer_elems(pg, n_kv, head_dim) * 2;  // bytes
  PagedAttnArgs a{};
  a.kpool = static_cast<const char*>(pg.d_kpool) + layer0;
  a.vpool = static_cast<const char*>(pg.d_vpool) + layer0;
  a.table = pg.d_table;
  a.len = pg.d_len;
  a.q = q;
  a.ws_o = ws_o;
  a.ws_ml = ws_ml;
  a.o = (unsigned short*)o;
  a.flags = flags;
  a.ldq = ldq;
  a.ldo = ldo;
  a.table_ld = pg.table_ld;
  a.n_pages = pg.n_pages;
  a.n_heads = n_heads;
  a.n_kv = n_kv;
  a.group = n_heads / n_kv;
  a.rows = rq.rows;
  a.n_req = rq.n;
  a.o_terms = o_terms;
  a.o_f16 = o_dtype == GOOSE_DTYPE_F16;
  a.sh_blocks = shared_pages * 2;
  a.sh_tiles = shared_pages > 0 ? (rq.rows * a.group + 31) / 32 : 0;
  // Blocks per item: enough items for two workgroups a compute unit, but at least eight blocks each (two a wavefront).
  long long work = (long long)a.sh_tiles * a.sh_blocks;
  int own_max = 0;
  for (int r = 0; r < rq.n; ++r) {
    const PagedReq& s = rq.r[r];
    a.r[r] = AttnReq{s.seq, s.B, s.P_max, s.row0, s.c0, (s.B * a.group + 31) / 32, 0, (const uint64_t*)s.p};
    const int nb = (s.P_max + s.B + 31) / 32 - a.sh_blocks;
    own_max = nb > own_max ? nb : own_max;
    work += (long long)a.r[r].tiles * nb;
  }
  long long per = (work * n_kv + 511) / 512;
  if (per < 8) per = 8;
  const size_t step = (size_t)n_heads * rq.rows;  // records of one split
  int own_splits;
  for (;; per *= 2) {
    a.sh_splits = (int)((a.sh_blocks + per - 1) / per);
    own_splits = (int)((own_max + per - 1) / per);
    if (a.sh_splits + own_splits <= 1 || (size_t)(a.sh_splits + own_splits) * step <= max_records) break;
    if (per > a.sh_blocks + own_max) return GOOSE_ERR_CAPACITY;
  }
  unsigned items = (unsigned)(a.sh_tiles * a.sh_splits);
  for (int r = 0; r < rq.n; ++r) {
    const int nb = (rq.r[r].P_max + rq.r[r].B + 31) / 32 - a.sh_blocks;
    a.r[r].splits = (int)((nb + per - 1) / per);
    items += (unsigned)(a.r[r].tiles * a.r[r].splits);
  }
  a.direct = a.sh_splits + own_splits == 1;
  const dim3 grid(n_kv, items);
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  if (head_dim == 128) {
    if (q_terms == 2) launch_t<128, 2>(f16, grid, a, st);
    else launch_t<128, 1>(f16, grid, a, st);
  } else {
    if (q_terms == 2) launch_t<64, 2>(f16, grid, a, st);
    else launch_t<64, 1>(f16, grid, a, st);
  }
  int rc = goose_launch_status();
  if (rc != GOOSE_OK || a.direct) return rc;
  const int per_wg = 1024 / head_dim;
  const dim3 mgrid((unsigned)((rq.rows * n_heads + per_wg - 1) / per_wg));
  if (head_dim == 128) hipLaunchKernelGGL(k_paged_merge<128>, mgrid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_paged_merge<64>, mgrid, dim3(256), 0, st, a);
  return goose_launch_status();
}
