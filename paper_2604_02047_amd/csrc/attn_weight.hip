// The attention weight that the slots of a paged cache receive from chunks of tokens.
//
//   w[s] = decay w[s] + sum over tokens i >= first with s <= P + i, and over the query heads of the KV head, of
//          2^(q . K[s] c - lse log2(e)),   c = log2(e) / sqrt(d)
//
// A wavefront owns the 64 slots of a page under one KV head: their keys stay in registers while the rows (token, query head of the
// group) stream by, 32 of them a tile.  S^T = K Q^T leaves 16 keys of one row in a lane, so a slot's sum grows in one register and is
// joined over lanes and wavefronts at the end, in a fixed order.
// What bounds it: many rows, the vector ALU and the matrix pipe (a fused multiply-add, an exponential and an addition a score take as long as its products): 2048 tokens
// of 32 / 8 heads behind 6144 slots, fp16, 142 to 160 us, 120 GFLOP at 750 to 850 TFLOP/s, and 117 with products and LDS reads alone.  Few rows, the keys' bytes:
// 16 tokens over 4000 slots each, 107 MB in 26 us (4.1 TB/s); the last 32 tokens of 300 of a 32-head model over 7000, 61 MB in 15 us.
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
  uint32_t group_inv;  // ceil(2^32 / group), 0 for groups of one: mulhi(row, group_inv) is row / group, or one more
  int32_t sg, rg;  // a workgroup's wavefronts: sg pages x rg of the tiles in turn
  int32_t splits;  // of the rows
  float* part;     // splits > 1: [split][chunk][KV head][part_ld]
  size_t part_ld;
  float decay;
  ChunkReq r[GOOSE_MAX_REQUESTS];
};

__device__ __forceinline__ void store_weight(const WeightArgs& a, const ChunkReq& rq, int kvh, int slot, int P, float w) {
  float* const out = a.weight + ((size_t)rq.seq * a.n_kv + kvh) * a.table_ld * GOOSE_PAGE + slot;
  if (slot < P && a.decay != 0.f) w += a.decay * *out;
  *out = w;
}

// Scores of a tile and 64 keys (to s), and beside the matrix instructions the weights of the tile before (scores z, its rows' logarithms l2), which
// need nothing of this one: a workgroup's wavefronts meet at every tile, so that without it they would all be at the matrix instructions
// together and at the exponentials together.
// (The kernel has one LDS array, and it is read here through a pointer of its own: else each read waits for the copies into other parts of it.)
template <int D, int QT, bool F16>
__device__ __forceinline__ void tile_step(const u32x4* __restrict__ tile, const u32x4 (&k)[2][D / 16], f32x16 (&s)[2], const f32x16 (&z)[2], float l2,
                                          float scale, f32x16 (&sum)[2]) {
  typedef typename Mma16<F16>::v8 op8;
  constexpr int PIECES = D / 16 * QT, AHEAD = 2;
  u32x4 piece[PIECES];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) piece[i] = tile[i * 64];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[b][r] = 0.f;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    if (i + AHEAD < PIECES) piece[i + AHEAD] = tile[(i + AHEAD) * 64];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = Mma16<F16>::mfma(__builtin_bit_cast(op8, k[b][i % (D / 16)]), __builtin_bit_cast(op8, piece[i]), s[b]);
#pragma unroll
      for (int e = (2 * i + b) * 16 / PIECES; e < (2 * i + b + 1) * 16 / PIECES; ++e) {
        float x = sum[e >> 4][e & 15] + __builtin_amdgcn_exp2f(fmaf(z[e >> 4][e & 15], scale, -l2));
        GOOSE_HERE(x);  // (the compiler would move it behind the matrix instructions)
        sum[e >> 4][e & 15] = x;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// The tiles come into LDS in operand order, two sets of U rg tiles: while one is worked on the other one arrives, the wavefronts of a tile
// copying their share of it (a lane fetches the 16 bytes that belong at its place).
template <int D, int QT, bool F16>
__global__ __launch_bounds__(512, 2) void k_slot_weights(const WeightArgs a) {
  typedef typename Mma16<F16>::T T;
  constexpr int NS = D / 16, PIECES = NS * QT, U = 2;  // 1 KiB pieces of a tile: the high terms' first
  constexpr int TILE = PIECES * 1024;
  extern __shared__ __attribute__((aligned(1024))) unsigned char tiles[];  // [step % 2][U rg][TILE]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, hh = lane >> 5;
  const int SG = a.sg, RG = a.rg, rg = __builtin_amdgcn_readfirstlane((int)((unsigned)wave / (unsigned)SG)), sg = wave - rg * SG;
  const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x / (unsigned)a.n_kv), kvh = blockIdx.x - item * a.n_kv;
  const unsigned page_group = __builtin_amdgcn_readfirstlane(item / (unsigned)a.splits), split = item - page_group * a.splits;
  const int first_page = (int)page_group * SG;
  const ChunkReq& rq = a.r[blockIdx.y];
  const int P = __builtin_amdgcn_readfirstlane(a.len[rq.seq]);
  if (P < 0 || P > rq.P_max) {
    if (tid == 0 && blockIdx.x == 0) atomicOr(a.flags, GOOSE_FLAG_CAPACITY);
    return;
  }
  const int end = P + rq.C, pages = (end + GOOSE_PAGE - 1) / GOOSE_PAGE;
  if (first_page >= pages) return;
  bool live = first_page + sg < pages;
  const int slot0 = live ? (first_page + sg) * GOOSE_PAGE : 0;
  const int page = __builtin_amdgcn_readfirstlane(live ? a.table[(size_t)rq.seq * a.table_ld + first_page + sg] : 0);
  if ((unsigned)page >= (unsigned)a.n_pages) {
    if (lane == 0) atomicOr(a.flags, GOOSE_FLAG_PAGES);
    live = false;
  }
  u32x4 k[2][NS];
  const T* const kp = static_cast<const T*>(a.kpool) + page_head<D>(live ? page : 0, a.n_kv, (int)kvh);
  fetch(kp, lane, k[0]);
  fetch(kp + 32 * D, lane, k[1]);
  // rows: from the first token that sees a slot of the workgroup
  const int group = a.group, rows = rq.C * group, row0 = max(rq.first, first_page * GOOSE_PAGE - P) * group;
  const unsigned all = (unsigned)(rows - row0 + 32 * U * RG - 1) / (unsigned)(32 * U * RG);
  int step = (int)(all * split / (unsigned)a.splits);
  const int steps = (int)(all * (split + 1) / (unsigned)a.splits);  // from `step`: this split's
  auto tile_of = [&](int step, int u) { return tiles + ((step & 1) * (U * RG) + u * RG + rg) * TILE; };
  const float scale = softmax_scale(D);
  const T* const q0 = static_cast<const T*>(a.q) + (size_t)rq.row0 * a.ldq + (size_t)kvh * group * D * QT;
  const float* const lse0 = a.lse + (size_t)kvh * group * a.ld_lse + rq.row0;
  const unsigned ldq = (unsigned)a.ldq, ld_lse = (unsigned)a.ld_lse, inv = a.group_inv;
  // of the next step's tiles: this lane's rows' tokens (-1: none) and logarithms
  int tok_next[U];
  float lse_next[U];
  auto copy = [&](int step) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int rho = row0 + ((step * U + u) * RG + rg) * 32 + l31, at = min(rho, rows - 1);
      // (behind the last row: that one)
      int tok = inv == 0 ? at : (int)__umulhi((unsigned)at, inv), h = at - tok * group;
      if (h < 0) { --tok; h += group; }
      lse_next[u] = lse0[(size_t)(unsigned)h * ld_lse + (unsigned)tok];
      tok_next[u] = rho < rows ? tok : -1;
#if defined(__HIP_DEVICE_COMPILE__)
      const int tok0 = __builtin_amdgcn_readfirstlane(tok);  // (the tile's first token: 32 rows reach less than 2^32 bytes from there)
      const __amdgpu_buffer_rsrc_t rsrc =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(q0 + (size_t)(unsigned)tok0 * ldq), 0, 0xFFFFFFFFu, GOOSE_BUFFER_WORD3);
      const unsigned offset = (((unsigned)(tok - tok0) * ldq) + (unsigned)(h * D + hh * 8) * QT) * 2;
      for (int p = sg; p < PIECES; p += SG)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, GOOSE_LDS_PTR(tile_of(step, u) + p * 1024), 16, offset, (p % NS * 16 * QT + p / NS * 8) * 2, 0, 0);
#endif
    }
  };
  f32x16 sum[2], s0[2], s1[2];  // scores of the tile before; -infinity: no weight
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sum[b][r] = 0.f;
      s1[b][r] = -INFINITY;
    }
  float l2 = 0.f;
  auto one = [&](const unsigned char* tile, int tok, float lse, f32x16 (&s)[2], const f32x16 (&z)[2]) {
    tile_step<D, QT, F16>(reinterpret_cast<const u32x4*>(tile) + lane, k, s, z, l2, scale, sum);
    // (a row of scores of -infinity only has that as its logarithm, too, and weighs nothing; a NaN concerns the keys that the row sees: it goes into their scores)
    const bool none = lse == -INFINITY, nan = lse != lse;
    l2 = none || nan ? 0.f : lse * 1.4426950408889634f;
    const int last = tok >= 0 && !none ? P + tok - slot0 - hh * 16 : -1;
    if (__builtin_amdgcn_ballot_w64(last < 47 || nan) != 0) {  // some row does not see all of the lane's keys
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] = b * 32 + r <= last ? (nan ? lse : s[b][r]) : -INFINITY;
    }
  };
  auto arrive = [&]() {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto rest = [&](const f32x16 (&z)[2]) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[b][r] += __builtin_amdgcn_exp2f(fmaf(z[b][r], scale, -l2));
  };
  if (step < steps) copy(step);
  for (; step + 1 < steps; ++step) {
    arrive();
    const int t0 = tok_next[0], t1 = tok_next[1];
    const float e0 = lse_next[0], e1 = lse_next[1];
    copy(step + 1);
    one(tile_of(step, 0), t0, e0, s0, s1);
    one(tile_of(step, 1), t1, e1, s1, s0);
  }
  arrive();  // the last step, in which tiles may have no rows
  if (step >= steps) {
  } else if (__builtin_amdgcn_ballot_w64(tok_next[0] >= 0) == 0) {
    rest(s1);
  } else {
    one(tile_of(step, 0), tok_next[0], lse_next[0], s0, s1);
    if (__builtin_amdgcn_ballot_w64(tok_next[1] >= 0) == 0) {
      rest(s0);
    } else {
      one(tile_of(step, 1), tok_next[1], lse_next[1], s1, s0);
      rest(s1);
    }
  }
  // over the 32 rows of a tile: lane l31 is left with value l31 = 16 b + r of its half, slot 32 b + 16 hh + r
  float v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = sum[i >> 4][i & 15];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const bool upper = (l31 & off) != 0;
#pragma unroll
    for (int i = 0; i < off; ++i) {
      const float keep = upper ? v[i + off] : v[i], send = upper ? v[i] : v[i + off];
      v[i] = keep + __shfl_xor(send, off, 64);
    }
  }
  const int mine = (l31 >> 4) * 32 + hh * 16 + (l31 & 15);
  float* const part = reinterpret_cast<float*>(tiles);  // [wavefront][slot]
  __syncthreads();
  part[wave * 64 + mine] = v[0];
  __syncthreads();
  if (rg != 0 || !live) return;
  float w = part[wave * 64 + lane];
  for (int i = 1; i < RG; ++i) w += part[(i * SG + sg) * 64 + lane];
  const int slot = slot0 + lane;
  if (slot >= end) return;
  if (a.splits > 1) {
    a.part[((size_t)(split * a.n + blockIdx.y) * a.n_kv + kvh) * a.part_ld + slot] = w;
    return;
  }
  store_weight(a, rq, (int)kvh, slot, P, w);
}

// Joins the splits, a thread a slot and a workgroup four pages, in their order.
__global__ __launch_bounds__(256) void k_weight_merge(const WeightArgs a) {
  const unsigned block = blockIdx.x / (unsigned)a.n_kv, kvh = blockIdx.x - block * a.n_kv;
  const ChunkReq& rq = a.r[blockIdx.y];
  const int P = a.len[rq.seq], slot = (int)(block * 256 + threadIdx.x);
  if (P < 0 || P > rq.P_max || slot >= P + rq.C) return;
  if ((unsigned)a.table[(size_t)rq.seq * a.table_ld + slot / GOOSE_PAGE] >= (unsigned)a.n_pages) return;
  const size_t step = (size_t)a.n * a.n_kv * a.part_ld;
  const float* const from = a.part + ((size_t)blockIdx.y * a.n_kv + kvh) * a.part_ld + slot;
  float w = 0.f;
  for (int s0 = 0; s0 < a.splits; s0 += 4) {
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = from[min(s0 + k, a.splits - 1) * step];
#pragma unroll
    for (int k = 0; k < 4; ++k) w += s0 + k < a.splits ? v[k] : 0.f;
  }
  store_weight(a, rq, (int)kvh, slot, P, w);
}

template <int D>
void launch_d(bool f16, int q_terms, dim3 grid, size_t lds, const WeightArgs& a, hipStream_t st) {
  const dim3 threads(64 * a.sg * a.rg);
  if (q_terms == 2) {
    if (f16) hipLaunchKernelGGL((k_slot_weights<D, 2, true>), grid, threads, lds, st, a);
    else hipLaunchKernelGGL((k_slot_weights<D, 2, false>), grid, threads, lds, st, a);
  } else {
    if (f16) hipLaunchKernelGGL((k_slot_weights<D, 1, true>), grid, threads, lds, st, a);
    else hipLaunchKernelGGL((k_slot_weights<D, 1, false>), grid, threads, lds, st, a);
  }
}

}  // namespace

int launch_attn_weight(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const void* q, size_t ldq, int q_terms,
                       const ChunkReqs& ck, const float* lse, size_t ld_lse, float decay, float* weight, float* ws, size_t ws_floats, int32_t* flags, hipStream_t st) {
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
  a.group_inv = a.group == 1 ? 0 : UINT32_MAX / (uint32_t)a.group + 1;
  a.n = ck.n;
  a.decay = decay;
  int most = 0, tiles = 0;
  long long waves = 0;  // pages x KV heads
  for (int i = 0; i < ck.n; ++i) {
    a.r[i] = ck.r[i];
    const int pages = (ck.r[i].P_max + ck.r[i].C + GOOSE_PAGE - 1) / GOOSE_PAGE, t = ((ck.r[i].C - ck.r[i].first) * a.group + 31) / 32;
    most = pages > most ? pages : most;
    tiles = t > tiles ? t : tiles;
    waves += (long long)pages * n_kv;
  }
  a.rg = a.sg = a.splits = 1;
  a.part = ws;
  a.part_ld = (size_t)most * GOOSE_PAGE;
  if (tiles >= 16) {
    // Two tiles in turn, so that LDS holds two steps' rows of any type; four pages, so that a workgroup's eight wavefronts fill a CU and a row is copied once for 256 keys.
    a.rg = 2;
    while (a.sg < 4 && a.sg < most) a.sg *= 2;
    // A CU holds one such workgroup.  Those of committed pages go through all rows, those of the chunk's own about half; the rows are split so that the last round of 256
    // is not left half empty, and chunks with few pages fill the CUs.  In units of 10 ns: a workgroup's beginning and end 500, a tile of a wavefront, the merge 500.
    // (2048 tokens of 32 / 8 heads from the start 46 us in four parts, 38 in eight, 71 in one; 512 behind 4000 slots with two-term queries 64 in two, 52 in three, 83 in one.)
    long long full = 0, own = 0, best = INT64_MAX;
    for (int i = 0; i < ck.n; ++i) {
      const int before = ck.r[i].P_max / (GOOSE_PAGE * a.sg), all = (ck.r[i].P_max + ck.r[i].C + GOOSE_PAGE * a.sg - 1) / (GOOSE_PAGE * a.sg);
      full += (long long)before * n_kv;
      own += (long long)(all - before) * n_kv;
    }
    const long long tile = (q_terms == 1 ? 115 : 180) * (head_dim + 32) / 160;
    for (int s = 1; s <= 32 && s * 8 <= tiles && (size_t)s * ck.n * n_kv * a.part_ld <= ws_floats; ++s) {
      const long long one = 500 + (tiles / a.rg + s - 1) / s * tile, half = (500 + one) / 2;
      const long long rounds = (full * s + 255) / 256, left = own * s - 2 * (rounds * 256 - full * s);  // (two of the chunk's own in a place that is left over)
      long long cost = rounds * one + (left > 0 ? (left + 255) / 256 * half : 0);
      cost = (cost > one ? cost : one) + (s > 1 ? 500 : 0);
      if (cost < best) { best = cost; a.splits = s; }
    }
  } else {
    // One wavefront a tile, up to four pages: 16 tokens of 32 / 8 heads over 4000 slots with 1 / 2 / 4 / 8 pages 37 / 26.4 / 25.6 / 32.9 us, one 8 / 9 / 9 / 10.5.
    while (a.sg < 4 && waves >= 512ll * a.sg) a.sg *= 2;
  }
  const int groups = (most + a.sg - 1) / a.sg;
  if ((long long)groups * a.splits * n_kv * (64 * a.sg * a.rg) > UINT32_MAX) return GOOSE_ERR_CAPACITY;  // (threads of a launch)
  const dim3 grid((unsigned)groups * (unsigned)a.splits * (unsigned)n_kv, (unsigned)ck.n);
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  const int sets = tiles > 2 * a.rg ? 2 : 1;  // (one step needs one)
  const size_t lds = (size_t)sets * 2 * a.rg * (head_dim / 16 * q_terms) * 1024;
  if (head_dim == 128) launch_d<128>(f16, q_terms, grid, lds, a, st);
  else if (head_dim == 64) launch_d<64>(f16, q_terms, grid, lds, a, st);
  else return GOOSE_ERR_SHAPE;
  const int rc = goose_launch_status();
  if (rc != GOOSE_OK || a.splits == 1) return rc;
  hipLaunchKernelGGL(k_weight_merge, dim3((unsigned)((most + 3) / 4) * (unsigned)n_kv, (unsigned)ck.n), dim3(256), 0, st, a);
  return goose_launch_status();
}
