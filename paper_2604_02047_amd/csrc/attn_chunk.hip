// Causal attention of chunks of new tokens over a paged cache.
//
//   o[i, h] = sum_s softmax_s(q[i, h] . K[s] / sqrt(d)) V[s],  s <= P + i;   lse[h, i] = log sum_s exp(q[i, h] . K[s] / sqrt(d))
//
// The rows of one KV head are (token, query head of the group), the heads fastest, so that a group's heads share what is read of the
// pages.  Per 32 keys and 32 rows: S^T = K Q^T, online softmax with two lanes a row, O^T += V^T P^T, operands straight from the pages'
// operand order.  A workgroup takes 128 rows, a wavefront 32 of them, and streams the blocks that its tokens see.
#include "chunk.h"

namespace {

struct ChunkArgs {
  const void* kpool;  // of the layer
  const void* vpool;
  const int32_t* table;
  const int32_t* len;
  const void* q;
  unsigned short* o;
  float* lse;
  int32_t* flags;
  size_t ldq, ldo, ld_lse;
  int32_t table_ld, n_pages, n_kv, group, n;
  int32_t o_terms, o_f16;
  int32_t tiles[GOOSE_MAX_REQUESTS];
  ChunkReq r[GOOSE_MAX_REQUESTS];
};

template <int D, int QT, bool F16>
__global__ __launch_bounds__(256, 2) void k_chunk_stream(const ChunkArgs a) {
  typedef RowTile<D, QT, F16> Tile;
  typedef typename Tile::T T;
  constexpr int NS = D / 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, hh = lane >> 5;
  int y = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (unsigned)a.n_kv));
  const int kvh = (int)blockIdx.x - y * a.n_kv;
  int ri = 0;
  while (y >= a.tiles[ri]) y -= a.tiles[ri++];
  const ChunkReq& rq = a.r[ri];
  const int P = chunk_length(a.len, rq, a.flags, tid == 0 && y == 0 && kvh == 0);
  const int rows = rq.C * a.group, row_first = y * 128 + wave * 32;
  if (row_first >= rows) return;
  const int rho = min(row_first + l31, rows - 1);
  const int tok = (int)((unsigned)rho / (unsigned)a.group), h = kvh * a.group + rho - tok * a.group;
  const int tok_lo = __builtin_amdgcn_readfirstlane((int)((unsigned)row_first / (unsigned)a.group));
  const int tok_hi = __builtin_amdgcn_readfirstlane((int)((unsigned)min(row_first + 31, rows - 1) / (unsigned)a.group));
  const int total = (P + tok_hi) / 32 + 1, full = (P + tok_lo + 1) / 32;  // blocks that a row sees, that all rows see whole
  PageIds pg{a.table + (size_t)rq.seq * a.table_ld, a.flags, 0, (total - 1) >> 1, a.n_pages, 0};
  pg.load(lane);
  const T* const kp = static_cast<const T*>(a.kpool);
  const T* const vp = static_cast<const T*>(a.vpool);
  auto block_at = [&](int b) -> size_t {
    return ((size_t)pg.of(b, lane) * a.n_kv + kvh) * (GOOSE_PAGE * D) + (size_t)(b & 1) * 32 * D;
  };
  u32x4 kreg[NS], vreg[NS];
  size_t at = block_at(0);
  fetch(kp + at, lane, kreg);
  fetch(vp + at, lane, vreg);
  Tile t;
  const size_t row = (size_t)rq.row0 + tok;
  t.init(static_cast<const T*>(a.q) + row * a.ldq + ((size_t)h * D + hh * 8) * QT);
  const float scale = softmax_scale(D);
  auto block = [&](int b, auto edge) {
    constexpr bool EDGE = decltype(edge)::value;
    t.scores(kreg);
    if (b + 1 < total) { at = block_at(b + 1); fetch(kp + at, lane, kreg); }
    unsigned vis = 0xFFFFu;
    bool odd = false;
    if (EDGE) {
      vis = seen16(P + tok - b * 32 - hh * 16);
      t.mask(vis);
      odd = clean_values<F16>(vreg, P + rq.C - b * 32 - hh * 16);
    }
    t.maximum();
    t.rescale(scale);
    t.weights();
    if (EDGE && odd) t.values_odd(vreg, vis);
    else t.values(vreg);
    if (b + 1 < total) fetch(vp + at, lane, vreg);
  };
  for (int b = 0; b < full; ++b) block(b, std::false_type());
  for (int b = full; b < total; ++b) block(b, std::true_type());

  const float l = t.l + __shfl_xor(t.l, 32, 64);
  if (row_first + l31 >= rows) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      store_columns(a.o + row * a.ldo, a.o_terms, a.o_f16, h * D + (dt * 4 + q) * 8 + hh * 4,
                    f32x4{t.o[dt][q * 4], t.o[dt][q * 4 + 1], t.o[dt][q * 4 + 2], t.o[dt][q * 4 + 3]} * inv);
  if (a.lse && hh == 0) a.lse[(size_t)h * a.ld_lse + row] = log_of_sum(t.m, l, scale);
}

template <int D>
void launch_d(bool f16, int q_terms, dim3 grid, const ChunkArgs& a, hipStream_t st) {
  if (q_terms == 2) {
    if (f16) hipLaunchKernelGGL((k_chunk_stream<D, 2, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_chunk_stream<D, 2, false>), grid, dim3(256), 0, st, a);
  } else {
    if (f16) hipLaunchKernelGGL((k_chunk_stream<D, 1, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_chunk_stream<D, 1, false>), grid, dim3(256), 0, st, a);
  }
}

}  // namespace

int launch_attn_chunk(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const void* q, size_t ldq, int q_terms,
                      const ChunkReqs& ck, void* o, size_t ldo, int o_dtype, int o_terms, float* lse, size_t ld_lse, int32_t* flags,
                      hipStream_t st) {
  const size_t layer0 = (size_t)layer * page_layer_elems(pg, n_kv, head_dim) * 2;  // bytes
  ChunkArgs a{};
  a.kpool = static_cast<const char*>(pg.d_kpool) + layer0;
  a.vpool = static_cast<const char*>(pg.d_vpool) + layer0;
  a.table = pg.d_table;
  a.len = pg.d_len;
  a.q = q;
  a.o = (unsigned short*)o;
  a.lse = lse;
  a.flags = flags;
  a.ldq = ldq;
  a.ldo = ldo;
  a.ld_lse = ld_lse;
  a.table_ld = pg.table_ld;
  a.n_pages = pg.n_pages;
  a.n_kv = n_kv;
  a.group = n_heads / n_kv;
  a.n = ck.n;
  a.o_terms = o_terms;
  a.o_f16 = o_dtype == GOOSE_DTYPE_F16;
  unsigned items = 0;
  for (int i = 0; i < ck.n; ++i) {
    a.r[i] = ck.r[i];
    a.tiles[i] = (ck.r[i].C * a.group + 127) / 128;
    items += (unsigned)a.tiles[i];
  }
  if ((unsigned long long)items * n_kv > INT32_MAX) return GOOSE_ERR_CAPACITY;
  const dim3 grid(items * (unsigned)n_kv);
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  if (head_dim == 128) launch_d<128>(f16, q_terms, grid, a, st);
  else if (head_dim == 64) launch_d<64>(f16, q_terms, grid, a, st);
  else return GOOSE_ERR_SHAPE;
  return goose_launch_status();
}
