// The attention weight that the slots of a paged cache receive from chunks of tokens.
//
//   w[s] = decay w[s] + sum over tokens i >= first with s <= P + i, and over the query heads of the KV head, of
//          2^(q . K[s] c - lse log2(e)),   c = log2(e) / sqrt(d)
//
// A workgroup owns the 64 slots of a page under one KV head: their keys stay in registers, the rows (token, query head of the group)
// stream by, 32 of them a tile, dealt out to four wavefronts.  S^T = K Q^T leaves 16 keys of one row in a lane, so a slot's sum
// grows in one register and is joined over lanes and wavefronts at the end, in a fixed order.
#include "chunk.h"

namespace {

struct WeightArgs {
  const void* kpool;  // of the layer
  const int32_t* table;
  const int32_t* len;
  const void* q;
  const float* lse;
  float* weight;  // of the layer
  int32_t* flags;
  size_t ldq, ld_lse;
  int32_t table_ld, n_pages, n_kv, group, n;
  float decay;
  ChunkReq r[GOOSE_MAX_REQUESTS];
};

template <int D, int QT, bool F16>
__global__ __launch_bounds__(256, 2) void k_slot_weights(const WeightArgs a) {
  typedef typename Mma16<F16>::T T;
  typedef typename Mma16<F16>::v8 op8;
  constexpr int NS = D / 16;
  __shared__ float part[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, hh = lane >> 5;
  int page_i = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (unsigned)a.n_kv));
  const int kvh = (int)blockIdx.x - page_i * a.n_kv;
  const ChunkReq& rq = a.r[blockIdx.y];
  const int P = __builtin_amdgcn_readfirstlane(a.len[rq.seq]);
  if (P < 0 || P > rq.P_max) {
    if (tid == 0 && blockIdx.x == 0) atomicOr(a.flags, GOOSE_FLAG_CAPACITY);
    return;
  }
  const int slot0 = page_i * GOOSE_PAGE, end = P + rq.C;
  if (slot0 >= end) return;
  const int page = a.table[(size_t)rq.seq * a.table_ld + page_i];
  if ((unsigned)page >= (unsigned)a.n_pages) {
    if (tid == 0) atomicOr(a.flags, GOOSE_FLAG_PAGES);
    return;
  }
  u32x4 k[2][NS];
  const T* const kp = static_cast<const T*>(a.kpool) + page_head<D>(page, a.n_kv, kvh);
  fetch(kp, lane, k[0]);
  fetch(kp + 32 * D, lane, k[1]);
  const int first = max(rq.first, slot0 - P);  // the first token that sees one of them
  const int rows = rq.C * a.group;
  const float scale = softmax_scale(D);
  f32x16 sum[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[b][r] = 0.f;
  for (int row0 = first * a.group + wave * 32; row0 < rows; row0 += 128) {
    const bool live = row0 + l31 < rows;
    const int rho = live ? row0 + l31 : rows - 1;
    const int tok = (int)((unsigned)rho / (unsigned)a.group), h = kvh * a.group + rho - tok * a.group;
    const size_t row = (size_t)rq.row0 + tok;
    const T* const at = static_cast<const T*>(a.q) + row * a.ldq + ((size_t)h * D + hh * 8) * QT;
    const float lse = a.lse[(size_t)h * a.ld_lse + row];
    op8 q[NS], ql[QT == 2 ? NS : 1];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = *reinterpret_cast<const op8*>(at + s * 16 * QT);
      if (QT == 2) ql[s] = *reinterpret_cast<const op8*>(at + s * 32 + 8);
    }
    // (a row of scores of -infinity only: its logarithm would make them NaN)
    const float l2 = lse * 1.4426950408889634f;
    const int last = live && lse != -INFINITY ? P + tok - slot0 - hh * 16 : -1;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) s = Mma16<F16>::mfma(__builtin_bit_cast(op8, k[b][i]), q[i], s);
      if (QT == 2) {
#pragma unroll
        for (int i = 0; i < NS; ++i) s = Mma16<F16>::mfma(__builtin_bit_cast(op8, k[b][i]), ql[i], s);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -l2));
        sum[b][r] += b * 32 + r <= last ? w : 0.f;
      }
    }
  }
  // over the 32 rows of a tile, then over the wavefronts; register r of half hh is key 16 hh + r
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = sum[b][r];
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) x += __shfl_xor(x, off, 64);
      if (l31 == 0) part[wave][b * 32 + hh * 16 + r] = x;
    }
  __syncthreads();
  const int slot = slot0 + tid;
  if (tid >= GOOSE_PAGE || slot >= end) return;
  float w = (part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]);
  float* const out = a.weight + ((size_t)rq.seq * a.n_kv + kvh) * a.table_ld * GOOSE_PAGE + slot;
  if (slot < P && a.decay != 0.f) w += a.decay * *out;
  *out = w;
}

template <int D>
void launch_d(bool f16, int q_terms, dim3 grid, const WeightArgs& a, hipStream_t st) {
  if (q_terms == 2) {
    if (f16) hipLaunchKernelGGL((k_slot_weights<D, 2, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_slot_weights<D, 2, false>), grid, dim3(256), 0, st, a);
  } else {
    if (f16) hipLaunchKernelGGL((k_slot_weights<D, 1, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_slot_weights<D, 1, false>), grid, dim3(256), 0, st, a);
  }
}

}  // namespace

int launch_attn_weight(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const void* q, size_t ldq, int q_terms,
                       const ChunkReqs& ck, const float* lse, size_t ld_lse, float decay, float* weight, int32_t* flags, hipStream_t st) {
  WeightArgs a{};
  a.kpool = static_cast<const char*>(pg.d_kpool) + (size_t)layer * page_layer_elems(pg, n_kv, head_dim) * 2;
  a.table = pg.d_table;
  a.len = pg.d_len;
  a.q = q;
  a.lse = lse;
  a.weight = weight + (size_t)layer * pg.n_seqs * n_kv * pg.table_ld * GOOSE_PAGE;
  a.flags = flags;
  a.ldq = ldq;
  a.ld_lse = ld_lse;
  a.table_ld = pg.table_ld;
  a.n_pages = pg.n_pages;
  a.n_kv = n_kv;
  a.group = n_heads / n_kv;
  a.n = ck.n;
  a.decay = decay;
  int most = 0;
  for (int i = 0; i < ck.n; ++i) {
    a.r[i] = ck.r[i];
    const int pages = (ck.r[i].P_max + ck.r[i].C + GOOSE_PAGE - 1) / GOOSE_PAGE;
    most = pages > most ? pages : most;
  }
  if ((long long)most * n_kv > INT32_MAX) return GOOSE_ERR_CAPACITY;
  const dim3 grid((unsigned)most * (unsigned)n_kv, (unsigned)ck.n);
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  if (head_dim == 128) launch_d<128>(f16, q_terms, grid, a, st);
  else if (head_dim == 64) launch_d<64>(f16, q_terms, grid, a, st);
  else return GOOSE_ERR_SHAPE;
  return goose_launch_status();
}
