// Causal attention of chunks of new tokens over a paged cache.
//
//   o[i, h] = sum_s softmax_s(q[i, h] . K[s] / sqrt(d)) V[s],  s <= P + i;   lse[h, i] = log sum_s exp(q[i, h] . K[s] / sqrt(d))
//
// The rows of one KV head are (token, query head of the group), the heads fastest, so that a group's heads share what is read of the
// pages.  Per 32 keys and 32 rows: S^T = K Q^T, online softmax with two lanes a row, O^T += V^T P^T, operands straight from the pages'
// operand order.
#include "chunk.h"

namespace {

struct ChunkItems {
  int32_t tiles, splits;  // work items: tiles of 32 NW rows x ranges of their blocks, for every KV head
  int32_t waves;          // 32-row tiles of a KV head
  int32_t join0;          // its first 32-row tile in the merge
  uint32_t rec0;          // its first record
};
struct ChunkArgs {
  const void* kpool;  // of the layer
  const void* vpool;
  const int32_t* table;
  const int32_t* len;
  const void* q;
  float* ws_o;    // [record][d / 8][64 lanes][4], a wavefront's accumulators as it holds them; records of a chunk: [split][KV head][32-row tile]
  float* ws_ml;   // [record][32][2]: largest score (unscaled), sum of weights
  unsigned short* o;
  float* lse;
  int32_t* flags;
  size_t ldq, ldo, ld_lse;
  int32_t table_ld, n_pages, n_heads, n_kv, group, n;
  int32_t o_terms, o_f16;
  int32_t groups, turn;  // of items (one for every KV head); from group `turn` on (0: never) the shortest come first
  ChunkItems it[GOOSE_MAX_REQUESTS];
  ChunkReq r[GOOSE_MAX_REQUESTS];
};

__device__ __forceinline__ void finish(const ChunkArgs& a, size_t row, int h, int D, int c, const f32x4& x, float m, float l) {
  store_columns(a.o + row * a.ldo, a.o_terms, a.o_f16, h * D + c, x * (l == 0.f ? 0.f : 1.0f / l));
  if (a.lse != nullptr && c == 0) a.lse[(size_t)h * a.ld_lse + row] = log_of_sum(m, l, softmax_scale(D));
}

// One workgroup = NW wavefronts, two on a SIMD (of one workgroup of eight or two of four), 32 rows each x a range of blocks.  Every block comes into LDS
// once, global -> LDS without registers, into a ring that runs several blocks ahead; a wavefront has three blocks under way at once (ring_step).  Blocks
// that a wavefront's rows do not see whole are masked on the way, and behind the last one that it sees it only goes on copying.
// A weight of zero does not keep a NaN or an infinity of an unseen slot's values out of the matrix instruction: a wavefront that has such a thing in its
// outputs at the end starts again, block by block with values_odd and sums in the ring's order: rows that do not see the thing keep their bits.  The block
// that the chunk ends in, whose other slots may hold anything, follows that way always.
// A weight enters the second product in two 16-bit terms whatever the output keeps: one term would be off by half a step of the type, as much again as the store of a
// one-term output, and by all of that in a row that a single key with a weight other than one dominates (4096 tokens behind 12288 slots 890 us so instead of 1195).
// What bounds it: the matrix and vector pipes together, at the clock that their load leaves.  4096 tokens of 32 / 8 heads behind 12288 slots, fp16, 1195 us: 805
// TFLOP/s, 1210 counting both terms of the weights (a large matrix product alone 1430); matrix pipe busy 66 %, vector ALU 53 %, clock 1.5 GHz (up to 1360 us on
// other cards and under the profiler).  Short ranges: 33B, 2000 tokens, 92 us (575 and 860 TFLOP/s), matrix pipe 39 %, 2.1 GHz.
template <int D, int QT, bool F16, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_chunk_ring(const ChunkArgs a) {
  typedef RowTile<D, QT, F16> Tile;
  typedef typename Tile::T T;
  constexpr int NS = D / 16;
  constexpr int BLOCK = 2 * NS * 1024, BU = BLOCK / 16;  // keys and values of 32 slots: bytes, 16-byte units
  constexpr int RING = NW;                               // blocks
  constexpr int CP = 2 * NS / NW;                        // pieces of 1 KiB that a wavefront copies of a block
  constexpr int ROWS = 32 * NW;
  constexpr int AHEAD = 4;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RING * BLOCK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, hh = lane >> 5;
  int y = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (unsigned)a.n_kv));
  const int kvh = (int)blockIdx.x - y * a.n_kv;  // the fast index: where 8 divides the KV heads, all items of a head run on one XCD
  // (Items run from the longest to the shortest.  Where two fit a CU and all run at once, the second of a CU comes from the other end.)
  if (a.turn > 0 && y >= a.turn) y = a.groups - 1 - (y - a.turn);
  int ri = 0;
  while (y >= a.it[ri].tiles * a.it[ri].splits) { y -= a.it[ri].tiles * a.it[ri].splits; ++ri; }
  ri = __builtin_amdgcn_readfirstlane(ri);
  y = __builtin_amdgcn_readfirstlane(y);
  const ChunkReq& rq = a.r[ri];
  const ChunkItems& ci = a.it[ri];
  const unsigned longest = __builtin_amdgcn_readfirstlane((unsigned)y / (unsigned)ci.splits);
  const int tile = ci.tiles - 1 - (int)longest, split = y - (int)longest * ci.splits;
  const int rows = rq.C * a.group, wg_first = tile * ROWS, row_first = wg_first + wave * 32;
  auto query = [&](int rho) -> const T* {
    const int at = min(rho, rows - 1), tok = (int)((unsigned)at / (unsigned)a.group), h = kvh * a.group + at - tok * a.group;
    return static_cast<const T*>(a.q) + ((size_t)rq.row0 + tok) * a.ldq + ((size_t)h * D + hh * 8) * QT;
  };
  Tile t;
  t.init(query(row_first + l31));  // (asked for in front of the length, which all else waits for)
  const int32_t* const table = a.table + (size_t)rq.seq * a.table_ld;
  auto token_of = [&](int rho) { return __builtin_amdgcn_readfirstlane((int)((unsigned)min(rho, rows - 1) / (unsigned)a.group)); };
  // blocks that the tile's last row sees behind a length, and those before part s of them
  auto total_of = [&](int P) { return (P + token_of(wg_first + ROWS - 1)) / 32 + 1; };
  auto part_of = [&](int total, int s) { return __builtin_amdgcn_readfirstlane((int)((unsigned)total * (unsigned)s / (unsigned)ci.splits)); };
  // (the first page ids, too: where they are if the length is its bound)
  const int likely = part_of(total_of(rq.P_max), split) >> 1, entry = likely + lane < a.table_ld ? table[likely + lane] : 0;
  const int P = chunk_length(a.len, rq, a.flags, tid == 0 && y == 0 && kvh == 0);
  auto clamp = [](int x, int lo, int hi) { return min(max(x, lo), hi); };
  // this item's range of blocks, and those of it in front of the chunk's end
  const int total = total_of(P), b_lo = part_of(total, split), b_hi = part_of(total, split + 1);
  const int units = __builtin_amdgcn_readfirstlane(clamp((P + rq.C) / 32 - b_lo, 0, b_hi - b_lo));
  // of the ring's units: from `whole` on some rows of this wavefront do not see all of it, from `seen` on none sees any
  const int whole = __builtin_amdgcn_readfirstlane((P + token_of(row_first) + 1) / 32 - b_lo);
  const int seen = __builtin_amdgcn_readfirstlane(row_first < rows ? clamp((P + token_of(row_first + 31)) / 32 + 1 - b_lo, 0, units) : -1);
  PageIds pg{table, a.flags, b_lo >> 1, (b_hi - 1) >> 1, a.n_pages, 0};
  if (b_hi > b_lo) {
    if (pg.base == likely) pg.take(lane, entry);
    else pg.load(lane);
  }
  const char* const kp = static_cast<const char*>(a.kpool);
  const char* const vp = static_cast<const char*>(a.vpool);
  auto block_at = [&](int b) -> size_t {  // bytes (pages times KV heads stays below 2^29: checked on the host)
    return (size_t)(unsigned)((pg.of(b, lane) * a.n_kv + kvh) * 2 + (b & 1)) * (32 * D * 2);
  };
  const int last = P + (int)((unsigned)min(row_first + l31, rows - 1) / (unsigned)a.group) - b_lo * 32 - hh * 16;  // the last slot that this lane's row sees
  const float scale = softmax_scale(D);
  const bool keys = wave < NW / 2;     // the first half of the wavefronts copy keys, the others values
  const int share = wave * CP * 1024;  // this wavefront's pieces of a block
  const char* const pool = (keys ? kp : vp) + (wave & (NW / 2 - 1)) * CP * 1024;
  auto barrier = [&]() {  // (raw: __syncthreads would also drain every copy in flight)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  const u32x4* const base = reinterpret_cast<const u32x4*>(ring) + lane;
  auto keys_of = [&](int u) { return base + (u & (RING - 1)) * BU; };
  if (units > 0) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // (all that was loaded so far: the counts below are those of the ring's copies)
    int next = 0;  // the unit copied next
    auto copy = [&]() {  // (behind the range: its last block again, never used)
      copy_pieces<CP>(pool + block_at(min(b_lo + next, b_hi - 1)), lane, ring + (next & (RING - 1)) * BLOCK + share);
      ++next;
    };
    const int first = keys ? RING : RING - (NW == 8 ? 2 : 1);
    while (next < first) copy();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((RING - 3) * CP));  // units 0 to 2 (values: 0, with the short ring 0 and 1)
    barrier();
    u32x4 pc[AHEAD];
    f32x16 z1;
    typename Tile::op8 w1[2], wl1[2];
    if (seen > 0) {
      u32x4 k[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) k[s] = keys_of(0)[s * 64];
      t.template scores<true>(k);
      if (whole <= 0) t.mask(seen16(last));
      t.maximum();
      t.rescale(scale);
      t.weights();
#pragma unroll
      for (int s = 0; s < NS; ++s) k[s] = keys_of(1)[s * 64];
      t.template scores<true>(k);
      if (whole <= 1) t.mask(seen16(last - 32));
      t.maximum();
      t.rescale_later(scale, t.s, units > 1);
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) pc[n] = keys_of(2)[n * 64];
    }
    // With the long ring steps j and j + 1 between two barriers.  Before them the keys of units up to j + 3 and the values of units up to j have landed in every
    // wavefront's share; keys of units up to j and values of units up to j - 2 are no longer read, and make room for those RING units later.
    // With the short one step j: keys up to j + 2 and values up to j - 1 have landed, keys up to j and values up to j - 2 make room.
    auto arrive = [&](int j) {
      if constexpr (NW == 8) __builtin_amdgcn_s_waitcnt(vmcnt_imm(3 * CP));
      else if (j == 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      else __builtin_amdgcn_s_waitcnt(vmcnt_imm(CP));
      barrier();
      __builtin_amdgcn_sched_barrier(0);
      copy();
      if (NW == 8 || (j == 1 && keys)) copy();
    };
    auto step = [&](int j, const f32x16& za, f32x16& zb, const auto& w, const auto& wl, auto& wn, auto& wln) {
      if (j > seen || seen == 0) return;
      ring_step<D, QT, F16, 1, AHEAD>(t, pc, keys_of(j + 1), keys_of(j - 1) + BU / 2, keys_of(j + 2), za, zb, w, wl, wn, wln, j + 1 < units, scale,
                                          [&](f32x16& s) {
                                            if (j + 1 >= whole) {
                                              const unsigned vis = seen16(last - (j + 1) * 32);
#pragma unroll
                                              for (int r = 0; r < 16; ++r) s[r] = ((vis >> r) & 1u) ? s[r] : -INFINITY;
                                            }
                                          });
    };
    int j = 1;
    for (; j + 1 < units; j += 2) {
      arrive(j);
      step(j, t.s, z1, t.p, t.pl, w1, wl1);
      if constexpr (NW == 4) arrive(j + 1);
      step(j + 1, z1, t.s, w1, wl1, t.p, t.pl);
    }
    if (j < units) {
      arrive(j);
      step(j, t.s, z1, t.p, t.pl, w1, wl1);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        t.p[i] = w1[i];
        t.pl[i] = wl1[i];
      }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // (the last values, and copies behind the range)
    barrier();
    if (seen == units) {
      u32x4 v[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) v[s] = keys_of(units - 1)[BU / 2 + s * 64];
      t.template values<true>(v);
    }
  }
  if (row_first >= rows) return;
  // ---- the block that the chunk ends in (in LDS already where the ring ran), or all of them again from memory
  // (the row again: kept over the ring's loop it would take registers that it needs)
  int rho = row_first + l31;
  GOOSE_HERE(rho);
  const int tok = (int)((unsigned)min(rho, rows - 1) / (unsigned)a.group), h = kvh * a.group + rho - tok * a.group;
  const int end = min(b_hi, (P + token_of(row_first + 31)) / 32 + 1);
  float odd_out = 0.f;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd_out = fmaf(t.o[dt][r], 0.f, odd_out);
  const bool again = units > 0 && __builtin_amdgcn_ballot_w64(odd_out != 0.f) != 0;
  if (again || b_lo + units < end) {
    if (again) t.init(query(rho));
    pg.base = (again ? b_lo : b_lo + units) >> 1;  // (the window may have run ahead)
    pg.load(lane);
#pragma unroll 1
    for (int u = again ? 0 : units, b = b_lo + u; b < end; ++u, ++b) {
      u32x4 k[NS], v[NS];
      if (u == units && units > 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          k[s] = keys_of(u)[s * 64];
          v[s] = keys_of(u)[BU / 2 + s * 64];
        }
      } else {
        const size_t at = block_at(b);
        fetch(kp + at, lane, k);
        fetch(vp + at, lane, v);
      }
      const unsigned vis = seen16(P + tok - b * 32 - hh * 16);
      t.template scores<true>(k);
      t.mask(vis);
      const bool odd = clean_values<F16>(v, P + rq.C - b * 32 - hh * 16);
      t.maximum();
      t.rescale(scale);
      t.weights();
      if (odd) t.template values_odd<true>(v, vis);
      else t.template values<true>(v);
    }
  }
  const float l = t.l + __shfl_xor(t.l, 32, 64);
  auto quads = [&](auto each) {  // (accumulators 4 q to 4 q + 3 of column tile dt are columns 32 dt + 8 q + 4 hh .. + 3)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) each(dt * 4 + q, f32x4{t.o[dt][q * 4], t.o[dt][q * 4 + 1], t.o[dt][q * 4 + 2], t.o[dt][q * 4 + 3]});
  };
  if (ci.splits > 1) {
    const size_t rec = ci.rec0 + ((size_t)split * a.n_kv + kvh) * ci.waves + tile * NW + wave;
    if (hh == 0) *reinterpret_cast<float2*>(a.ws_ml + (rec * 32 + l31) * 2) = make_float2(t.m, l);
    quads([&](int i, const f32x4& x) { *reinterpret_cast<f32x4*>(a.ws_o + (rec * (D / 8) + i) * 256 + lane * 4) = x; });
  } else if (rho < rows) {
    quads([&](int i, const f32x4& x) { finish(a, (size_t)rq.row0 + tok, h, D, i * 8 + hh * 4, x, t.m, l); });
  }
}

// Joins the splits of a 32-row tile: a thread the four columns that a lane held, records in their order, four in flight together.  512 tokens of 32 heads in four
// splits: 34 MB of records out of the caches behind the L2s, 8.5 us.
template <int D>
__global__ __launch_bounds__(256) void k_chunk_merge(const ChunkArgs a) {
  constexpr int PER = D / 32;  // workgroups a tile, four quads of columns each
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, hh = lane >> 5;
  const int wg = blockIdx.x / PER, quad = (blockIdx.x - wg * PER) * 4 + (tid >> 6);
  int r = 0;
  while (r + 1 < a.n && wg >= a.it[r + 1].join0) ++r;
  const ChunkItems& ci = a.it[r];
  const int kvh = (wg - ci.join0) / ci.waves, wt = wg - ci.join0 - kvh * ci.waves;
  const int rho = wt * 32 + l31;
  if (rho >= a.r[r].C * a.group) return;
  const size_t rec0 = ci.rec0 + (size_t)kvh * ci.waves + wt, step = (size_t)a.n_kv * ci.waves;
  const int n = ci.splits;
  const float scale = softmax_scale(D);
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f, m = -INFINITY;
  for (int s0 = 0; s0 < n; s0 += 4) {
    float2 ml[4];
    f32x4 ov[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const size_t rec = rec0 + (size_t)min(s0 + k, n - 1) * step;
      ml[k] = *reinterpret_cast<const float2*>(a.ws_ml + (rec * 32 + l31) * 2);
      ov[k] = *reinterpret_cast<const f32x4*>(a.ws_o + (rec * (D / 8) + quad) * 256 + lane * 4);
    }
    float m_new = m;
#pragma unroll
    for (int k = 0; k < 4; ++k) m_new = fmaxf(m_new, ml[k].x);
    const float w0 = join_factor(m, m_new, scale);
    den *= w0;
    num *= w0;
    m = m_new;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (s0 + k < n) {
        const float w = join_factor(ml[k].x, m, scale);
        den = fmaf(w, ml[k].y, den);
        num += w * ov[k];
      }
  }
  const int tok = (int)((unsigned)rho / (unsigned)a.group), h = kvh * a.group + rho - tok * a.group;
  finish(a, (size_t)a.r[r].row0 + tok, h, D, quad * 8 + hh * 4, num, m, den);
}

template <int D, int QT, bool F16, int NW>
void launch_t(unsigned items, const ChunkArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_chunk_ring<D, QT, F16, NW>), dim3(items), dim3(64 * NW), 0, st, a);
}
template <int D, int NW>
void launch_d(bool f16, int q_terms, unsigned items, const ChunkArgs& a, hipStream_t st) {
  if (q_terms == 2) f16 ? launch_t<D, 2, true, NW>(items, a, st) : launch_t<D, 2, false, NW>(items, a, st);
  else f16 ? launch_t<D, 1, true, NW>(items, a, st) : launch_t<D, 1, false, NW>(items, a, st);
}

}  // namespace

int launch_attn_chunk(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const void* q, size_t ldq, int q_terms,
                      const ChunkReqs& ck, float* ws_o, float* ws_ml, size_t max_records, void* o, size_t ldo, int o_dtype, int o_terms, float* lse,
                      size_t ld_lse, int32_t* flags, hipStream_t st) {
  if (head_dim != 64 && head_dim != 128) return GOOSE_ERR_SHAPE;
  const int group = n_heads / n_kv;
  // Chunks of few rows are chains of nodes for the tree kernels, which have shapes for them, unless there are hardly any slots to read or so many rows in all that
  // the ring has enough to do.  us, tree / ring, of 32 / 8 heads: one token behind 2000 slots 12 / 19, 16 requests 32 / 34; 64 tokens behind 600 15 / 17, four requests
  // 17 / 23, 15 50 / 30; 64 tokens behind 8000 32 / 27; 40 heads, 15 requests of one token behind nothing 22 / 16, 200 slots 30 / 28, 600 43 / 48; of 16 tokens 52 / 51.
  // (Of a multi-head model chunks of more than 32 tokens always: 64 behind 8000 53 / 35, though behind 300 13 / 16.)
  auto blocks_of = [](const ChunkReq& c) { return (c.P_max + c.C + 31) / 32; };
  auto small = [&](const ChunkReq& c) { return c.C <= GOOSE_MAX_B && c.C * group <= 256 && (group > 1 || c.C <= 32); };
  long long small_tiles = 0, small_work = 0;  // tiles of 32 rows, times blocks
  for (int i = 0; i < ck.n; ++i)
    if (small(ck.r[i])) {
      const long long t = (long long)n_kv * ((ck.r[i].C * group + 31) / 32);
      small_tiles += t;
      small_work += t * blocks_of(ck.r[i]);
    }
  auto by_tree = [&](const ChunkReq& c) {
    const int rows = c.C * group, blocks = blocks_of(c);
    if (!small(c) || blocks <= 2) return false;
    if (small_tiles >= 400 && (rows >= 16 || blocks <= 8)) return false;
    return small_work < 16000 || rows < 64;
  };
  PagedReqs few{};
  ChunkReqs many{};
  for (int i = 0; i < ck.n; ++i) {
    const ChunkReq& c = ck.r[i];
    if (by_tree(c)) {
      few.r[few.n++] = PagedReq{c.seq, c.C, c.P_max, c.row0, few.rows, nullptr, nullptr};
      few.rows += c.C;
    } else {
      int at = many.n++;
      for (; at > 0 && blocks_of(many.r[at - 1]) < blocks_of(c); --at) many.r[at] = many.r[at - 1];  // the longest first
      many.r[at] = c;
    }
  }
  if (few.n > 0) {
    const int rc = launch_attn_paged(dtype, pg, layer, n_heads, n_kv, head_dim, q, ldq, q_terms, few, 0, ws_o, ws_ml, max_records, o, ldo, o_dtype,
                                     o_terms, flags, st, lse, ld_lse);
    if (rc != GOOSE_OK || many.n == 0) return rc;
  }
  const size_t layer0 = (size_t)layer * page_layer_elems(pg, n_kv, head_dim) * 2;  // bytes
  ChunkArgs a{};
  a.kpool = static_cast<const char*>(pg.d_kpool) + layer0;
  a.vpool = static_cast<const char*>(pg.d_vpool) + layer0;
  a.table = pg.d_table;
  a.len = pg.d_len;
  a.q = q;
  a.ws_o = ws_o;
  a.ws_ml = ws_ml;
  a.o = (unsigned short*)o;
  a.lse = lse;
  a.flags = flags;
  a.ldq = ldq;
  a.ldo = ldo;
  a.ld_lse = ld_lse;
  a.table_ld = pg.table_ld;
  a.n_pages = pg.n_pages;
  a.n_heads = n_heads;
  a.n_kv = n_kv;
  a.group = group;
  a.n = many.n;
  a.o_terms = o_terms;
  a.o_f16 = o_dtype == GOOSE_DTYPE_F16;
  // Work items run in rounds of as many as the CUs hold, the longest first.  In units of 10 ns: an item's fixed part (length, table and first blocks one after the
  // other, the last block, stores), a block of it (measured over the terms), the merge and its records.  (300 or 1000 for the fixed part choose splits
  // that take as long, or up to 16 % longer.)  Alone on its CU a workgroup of four takes two thirds of a block's time, which is what the longest item comes to.
  const long long fixed = 700, step = (30 + 34 * (q_terms + 2)) * (head_dim + 64) / 192;
  long long best = INT64_MAX;
  int best_per = 0;
  int longest = 0;
  for (int i = 0; i < many.n; ++i) {
    const int blocks = blocks_of(many.r[i]);
    longest = blocks > longest ? blocks : longest;
  }
  // Two workgroups of four wavefronts a CU hide each other's beginnings and ends, one of eight copies every block once: us with 4 / 8 at 16 blocks (512 tokens of 32
  // heads) 18 / 25, 63 (2000 tokens of 52 heads) 96 / 96, 126 (512 of 32 / 8 heads behind 3500) 69 / 74, 188 (1024 behind 5000) 141 / 144, 282 (behind 8000) 202 / 201, 512
  // (4096 behind 12288) 1222 / 1192.
  const int nw = longest <= 256 ? 4 : 8, slots = 2048 / nw, tile_rows = 32 * nw;
  auto splits_of = [](int blocks, int per) { return (blocks + per - 1) / per; };
  for (int parts = 1; parts <= 32 && parts <= longest; ++parts) {
    const int per = splits_of(longest, parts);
    long long work = 0, items = 0, most = 0, records = 0;
    for (int i = 0; i < many.n; ++i) {
      const ChunkReq& c = many.r[i];
      const long long tiles = ((long long)c.C * group + tile_rows - 1) / tile_rows;
      const int blocks = blocks_of(c), splits = splits_of(blocks, per);
      const long long sum = tiles * (2ll * c.P_max + c.C) / 64 + 2 * tiles;  // blocks of all tiles
      work += (sum * step + tiles * splits * fixed) * n_kv;
      items += tiles * splits * n_kv;
      const long long len = splits_of(blocks, splits) * (nw == 4 ? step * 13 / 20 : step) + fixed;
      most = len > most ? len : most;
      if (splits > 1) records += (long long)splits * n_kv * ((c.C * group + 31) / 32);
    }
    if (records * 32 > (long long)max_records) continue;
    const long long rounds = (items + slots - 1) / slots, time = items <= 256 ? 0 : rounds * (work / items);
    const long long cost = (time > most ? time : most) + (records > 0 ? 600 + records * 32 * head_dim * 8 / 50000 : 0);
    if (cost < best) { best = cost; best_per = per; }
  }
  if (best_per == 0) best_per = longest;
  uint32_t records = 0;
  int joins = 0;
  long long items = 0;
  for (int i = 0; i < many.n; ++i) {
    const ChunkReq& c = many.r[i];
    const int tiles = (c.C * group + tile_rows - 1) / tile_rows, waves = (c.C * group + 31) / 32, splits = splits_of(blocks_of(c), best_per);
    a.it[i] = ChunkItems{tiles, splits, waves, joins, records};
    if (splits > 1) {
      records += (uint32_t)(splits * n_kv * waves);
      joins += n_kv * waves;
    }
    a.r[i] = c;
    items += (long long)tiles * splits * n_kv;
  }
  if (items * 64 * nw > UINT32_MAX) return GOOSE_ERR_CAPACITY;  // (threads of a launch)
  a.groups = (int)(items / n_kv);
  a.turn = nw == 4 && items > 256 && items <= 512 ? 256 / n_kv : 0;
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  if (head_dim == 128) nw == 4 ? launch_d<128, 4>(f16, q_terms, (unsigned)items, a, st) : launch_d<128, 8>(f16, q_terms, (unsigned)items, a, st);
  else nw == 4 ? launch_d<64, 4>(f16, q_terms, (unsigned)items, a, st) : launch_d<64, 8>(f16, q_terms, (unsigned)items, a, st);
  const int rc = goose_launch_status();
  if (rc != GOOSE_OK || joins == 0) return rc;
  const dim3 grid((unsigned)(joins * (head_dim / 32)));
  if (head_dim == 128) hipLaunchKernelGGL(k_chunk_merge<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_chunk_merge<64>, grid, dim3(256), 0, st, a);
  return goose_launch_status();
}
