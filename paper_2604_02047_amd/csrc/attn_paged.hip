// Tree attention of up to 16 requests over a paged cache; pages that all of them share can be read once for the rows of all.
//
//   o[row, h] = sum_k softmax_k(q[row, h] . K[k] / sqrt(d)) V[k],   k over the slots that the row sees.
//
// Softmax is associative over sets of keys: with (m, l, O) = (max, sum of 2^(s - m), sum of 2^(s - m) V) of a set, two sets join as
// m = max(m1, m2), l = 2^(m1 - m) l1 + 2^(m2 - m) l2, O likewise.  So the shared keys and a request's own ones can be
// separate work items (where that is cheaper: the rule is at launch_attn_paged), and either kind is split along the keys as far as it takes to fill the card; k_paged_merge joins what
// the items of a row left, in a fixed order.
//
// The rows of one KV head -- (node, query head of the group), for the shared keys of all requests one behind the other -- are the columns of
// 32-wide matrix-instruction tiles: a single token of a grouped-query model fills 4 of 32 columns with its four heads,
// and sixteen of them share two tiles over the common prefix.  Per 32 keys and 32 rows, as in the contiguous attention:
// S^T = K Q^T, online softmax with two lanes a row, O^T += V^T P^T, operands straight from the pages' operand order.
// The probabilities keep two terms for the second product (hi + lo: 2^-17 under bf16, 2^-22 under fp16), as the plain form keeps them in
// 32 bits.  The output goes on as fp16 or in two terms: one bf16 term of 8 bits would be its largest error by far (16 requests x 1 over 8192
// slots: 0.00085 of the output's size, with two 0.00021 as the output's own rounding), one fp16 term of 11 bits an error as large as the output's own
// rounding (16 x 32 over 16384: 0.00029, with two 0.00021; more for a row that one key with a weight above one dominates, see raise()).  The second fp16
// term costs half the matrix instructions again: 162 us before, now 207; 7B, 5 ragged requests over 1984 slots 26, now 29.
#include "attn_tile.h"

namespace {

struct AttnReq {
  int32_t seq, B, P_max, row0, c0;
  int32_t tiles, splits;  // work items over its own keys: tiles x splits, for every KV head
  const uint64_t* mask;   // null: a chain, node i sees nodes 0 .. i
};
struct PagedAttnArgs {
  const void* kpool;  // of the layer
  const void* vpool;
  const int32_t* table;
  const int32_t* len;
  const void* q;
  float* ws_o;    // [split][head][row][d]; splits of the shared keys first
  float* ws_ml;   // [split][head][row][2]: largest score (unscaled), sum of weights
  unsigned short* o;
  float* lse;     // [n_heads][ld_lse], or null
  int32_t* flags;
  size_t ldq, ldo, ld_lse;
  int32_t table_ld, n_pages, n_heads, n_kv, group, rows, n_req;
  int32_t same_blocks;                     // 32-slot blocks in front that must be the same in all tables
  int32_t sh_blocks, sh_tiles, sh_splits;  // shared keys with items of their own: blocks (all of those, or none), row tiles, splits
  int32_t sh_kg, own_kg;                   // k_paged_tiles: key groups of either kind of item
  int32_t direct;                          // every row has one item: it writes o itself
  int32_t o_terms, o_f16;
  AttnReq r[GOOSE_MAX_REQUESTS];
};

// Four neighbouring columns (inside one group of eight) of an output row.
__device__ inline void store_out(const PagedAttnArgs& a, size_t row, int col, const f32x4& x) {
  store_columns(a.o + row * a.ldo, a.o_terms, a.o_f16, col, x);
}

// Which keys of the 16 from tree node j0 on (negative: committed slots, visible) a mask row shows.
__device__ inline unsigned window16(uint64_t w0, uint64_t w1, int j0) {
  if (j0 <= -16) return 0xFFFFu;
  if (j0 < 0) return (unsigned)(((1u << -j0) - 1u) | (unsigned)(w0 << -j0)) & 0xFFFFu;
  if (j0 >= 128) return 0;
  uint64_t x = j0 < 64 ? w0 >> j0 : w1 >> (j0 - 64);
  if (j0 > 48 && j0 < 64) x |= w1 << (64 - j0);
  return (unsigned)x & 0xFFFFu;
}

// ---- work items -----------------------------------------------------------------------------------------------------
struct Item {
  int ri;        // its request; -1: the shared keys
  int tile, split, nsplit, rec_split;
  int seq, B, P; // of the request
  int b_lo, b_hi;  // its 32-slot blocks, counted from the sequence's start
  bool first;    // the first item of a request
};
__device__ inline Item item_of(const PagedAttnArgs& a, int y, int kvh) {
  Item it;
  int n_blocks, b_first;
  it.ri = -1;
  it.seq = a.r[0].seq;  // (shared keys: any request's table will do)
  it.B = it.P = 0;
  it.first = false;
  if (y < a.sh_tiles * a.sh_splits) {
    it.split = __builtin_amdgcn_readfirstlane((int)((unsigned)y / (unsigned)a.sh_tiles));
    it.tile = y - it.split * a.sh_tiles;
    it.nsplit = a.sh_splits;
    it.rec_split = it.split;
    b_first = 0;
    n_blocks = a.sh_blocks;
  } else {
    y -= a.sh_tiles * a.sh_splits;
    int r = 0;
    while (y >= a.r[r].tiles * a.r[r].splits) { y -= a.r[r].tiles * a.r[r].splits; ++r; }
    it.ri = r;
    it.first = y == 0 && kvh == 0;
    it.split = __builtin_amdgcn_readfirstlane((int)((unsigned)y / (unsigned)a.r[r].tiles));
    it.tile = y - it.split * a.r[r].tiles;
    it.nsplit = a.r[r].splits;
    it.rec_split = a.sh_splits + it.split;
    it.seq = a.r[r].seq;
    it.B = a.r[r].B;
    it.P = __builtin_amdgcn_readfirstlane(a.len[it.seq]);
    const int S = a.sh_blocks * 32;
    if ((it.P < a.same_blocks * 32 || it.P < 0 || it.P > a.r[r].P_max) && it.first && threadIdx.x == 0) atomicOr(a.flags, GOOSE_FLAG_CAPACITY);
    it.P = min(max(it.P, S), a.r[r].P_max);  // (P_max + B <= 64 table_ld, S <= P_max: checked on the host)
    b_first = a.sh_blocks;
    n_blocks = ((it.P + it.B + 31) >> 5) - b_first;
  }
  // (divisions go through vector registers: back to uniform ones)
  it.b_lo = __builtin_amdgcn_readfirstlane(b_first + (int)((unsigned)(n_blocks * it.split) / (unsigned)it.nsplit));
  it.b_hi = __builtin_amdgcn_readfirstlane(b_first + (int)((unsigned)(n_blocks * (it.split + 1)) / (unsigned)it.nsplit));
  return it;
}
// The shared pages must be the same in all tables: one wavefront a request compares them with the first request's.
__device__ inline void check_shared(const PagedAttnArgs& a, const Item& it, int lane) {
  if (!it.first || it.ri <= 0) return;
  const int32_t* t0 = a.table + (size_t)a.r[0].seq * a.table_ld;
  const int32_t* t = a.table + (size_t)it.seq * a.table_ld;
  bool differs = false;
  for (int i = lane; i < a.same_blocks / 2; i += 64) differs = differs || t[i] != t0[i];
  if (differs) atomicOr(a.flags, GOOSE_FLAG_PAGES);
}
// Row rho of an item: (node, query head of the group), the heads fastest.
struct Row {
  bool live;
  int node, crow, row, h;
};
__device__ inline Row row_of(const PagedAttnArgs& a, const Item& it, int rho, int kvh) {
  Row w;
  w.node = (int)((unsigned)rho / (unsigned)a.group);
  w.h = kvh * a.group + rho - w.node * a.group;
  if (it.ri < 0) {
    w.live = w.node < a.rows;
    w.crow = w.live ? w.node : 0;
    int r = 0;
    while (r + 1 < a.n_req && w.crow >= a.r[r + 1].c0) ++r;
    w.row = a.r[r].row0 + w.crow - a.r[r].c0;
  } else {
    w.live = w.node < it.B;
    const int n = w.live ? w.node : 0;
    w.crow = a.r[it.ri].c0 + n;
    w.row = a.r[it.ri].row0 + n;
  }
  return w;
}
// The half of a row's query that a lane holds.
template <int D, int QT, typename T>
__device__ __forceinline__ const T* query_of(const PagedAttnArgs& a, const Row& w, int hh) {
  return static_cast<const T*>(a.q) + (size_t)w.row * a.ldq + ((size_t)w.h * D + hh * 8) * QT;
}

// Mask row of a node, bits at or beyond B cleared.
struct MaskRow { uint64_t w0, w1; };
__device__ inline MaskRow mask_of(const PagedAttnArgs& a, const Item& it, const Row& w) {
  MaskRow k = {0, 0};
  if (it.ri < 0 || !w.live) return k;
  if (a.r[it.ri].mask == nullptr) {
    k.w0 = w.node >= 63 ? ~0ull : (2ull << w.node) - 1;
    k.w1 = w.node >= 127 ? ~0ull : (w.node >= 64 ? (2ull << (w.node - 64)) - 1 : 0);
    return k;
  }
  const int W = (it.B + 63) >> 6;
  const uint64_t* p = a.r[it.ri].mask + (size_t)w.node * W;
  k.w0 = p[0];
  if (W > 1) k.w1 = p[1];
  if (it.B < 64) k.w0 &= (1ull << it.B) - 1;
  if (it.B < 128) k.w1 &= it.B > 64 ? (1ull << (it.B - 64)) - 1 : 0;
  return k;
}
// What an item leaves of a row: columns c .. c + 3 of its (m, l, O), or the output itself.  x: sums of weights, x / l the mean
__device__ inline void leave(const PagedAttnArgs& a, const Item& it, const Row& w, int D, int c, const f32x4& x, float m, float l) {
  if (a.direct) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    store_out(a, w.row, w.h * D + c, x * inv);
    if (a.lse != nullptr && c == 0) a.lse[(size_t)w.h * a.ld_lse + w.row] = log_of_sum(m, l, softmax_scale(D));
  } else {
    const size_t rec = ((size_t)it.rec_split * a.n_heads + w.h) * a.rows + w.crow;
    if (c == 0) *reinterpret_cast<float2*>(a.ws_ml + rec * 2) = make_float2(m, l);
    *reinterpret_cast<f32x4*>(a.ws_o + rec * D + c) = x;
  }
}

// ---- few rows -----------------------------------------------------------------------------------------------------------
// One workgroup = RT tiles of 32 rows x a range of blocks: eight wavefronts, each with one tile and one of 8 / RT contiguous shares of the
// range.  A wavefront streams its blocks global -> registers -> matrix cores (no barrier in the loop), the next block's keys
// and values requested as soon as the current ones have been used; two tiles' wavefronts find each other's blocks in the cache.
template <int D, int QT, bool F16, int RT>
__global__ __launch_bounds__(512, 2) void k_paged_stream(const PagedAttnArgs a) {
  typedef RowTile<D, QT, F16> Tile;
  typedef typename Tile::T T;
  constexpr int NG = 8 / RT, NS = D / 16, QUADS = D / 8, QPW = QUADS / NG;
  static_assert(QUADS % NG == 0, "register quads must divide over the key groups");
  constexpr int WFLOATS = (QUADS + 1) * 256;  // a wavefront's state at the merge
  __shared__ __attribute__((aligned(16))) float lds[8 * WFLOATS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = wave % NG, rt = wave / NG;
  const int l31 = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x;  // the fast index: where 8 divides the KV heads, all items of a head run on one XCD and find each other's blocks in its L2
  const Item it = item_of(a, blockIdx.y, kvh);
  const int n_wg = it.b_hi - it.b_lo;
  const int b0 = it.b_lo + n_wg * g / NG, total = it.b_lo + n_wg * (g + 1) / NG - b0;
  PageIds pg{a.table + (size_t)it.seq * a.table_ld, a.flags, b0 >> 1, (b0 + total - 1) >> 1, a.n_pages, 0};
  const T* const kp = static_cast<const T*>(a.kpool);
  const T* const vp = static_cast<const T*>(a.vpool);
  auto block_at = [&](int b) -> size_t {
    return ((size_t)pg.of(b, lane) * a.n_kv + kvh) * (GOOSE_PAGE * D) + (size_t)(b & 1) * 32 * D;
  };
  const Row row = row_of(a, it, (it.tile * RT + rt) * 32 + l31, kvh);
  const bool work = RT == 1 || __builtin_amdgcn_ballot_w64(row.live) != 0;  // (the second tile may be empty)
  u32x4 kreg[NS], vreg[NS];
  size_t at = 0;
  if (total > 0 && work) {
    pg.load(lane);
    at = block_at(b0);
    fetch(kp + at, lane, kreg);
    fetch(vp + at, lane, vreg);
  }
  Tile t;
  t.init(query_of<D, QT, T>(a, row, hh));
  const float scale = softmax_scale(D);
  if (work) {
    const MaskRow mk = mask_of(a, it, row);
    auto block = [&](int idx, auto tree) {
      constexpr bool TREE = decltype(tree)::value;
      const int slot0 = (b0 + idx) * 32;
      t.scores(kreg);
      if (idx + 1 < total) { at = block_at(b0 + idx + 1); fetch(kp + at, lane, kreg); }
      unsigned vis = 0xFFFFu;
      bool odd = false;
      if (TREE) {
        vis = window16(mk.w0, mk.w1, slot0 + hh * 16 - it.P);
        t.mask(vis);
        odd = clean_values<F16>(vreg, it.P + it.B - slot0 - hh * 16);
      }
      t.maximum();
      t.rescale(scale);
      t.weights();
      if (TREE && odd) t.values_odd(vreg, vis);
      else t.values(vreg);
      if (idx + 1 < total) fetch(vp + at, lane, vreg);
    };
    // blocks that every row sees whole, then those that the tree reaches into
    const int full = it.ri < 0 ? total : max(0, min(total, (it.P >> 5) - b0));
    for (int idx = 0; idx < full; ++idx) block(idx, std::false_type());
    for (int idx = full; idx < total; ++idx) block(idx, std::true_type());
  }
  if (wave == 0) check_shared(a, it, lane);

  // ---- the key groups' states join in one round through LDS: each wavefront leaves its own, then owns some of its tile's columns
  float* dst = lds + (size_t)wave * WFLOATS + lane * 4;
  *reinterpret_cast<f32x4*>(dst) = f32x4{t.m, t.l, 0.f, 0.f};
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4*>(dst + 256 * (1 + dt * 4 + q)) = f32x4{t.o[dt][q * 4], t.o[dt][q * 4 + 1], t.o[dt][q * 4 + 2], t.o[dt][q * 4 + 3]};
  __syncthreads();
  const float* src = lds + (size_t)rt * NG * WFLOATS + lane * 4;
  float mj[NG], lj[NG], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const f32x4 ml = *reinterpret_cast<const f32x4*>(src + (size_t)j * WFLOATS);
    mj[j] = ml[0];
    lj[j] = ml[1];
    m = fmaxf(m, mj[j]);
  }
  f32x4 res[QPW];
#pragma unroll
  for (int q = 0; q < QPW; ++q) res[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const float w = join_factor(mj[j], m, scale);
    l += w * lj[j];
#pragma unroll
    for (int q = 0; q < QPW; ++q)
      res[q] += w * *reinterpret_cast<const f32x4*>(src + (size_t)j * WFLOATS + 256 * (1 + g * QPW + q));
  }
  l += __shfl_xor(l, 32, 64);
  if (!row.live) return;
  // quad i of the accumulator = columns 8 i + 4 hh .. + 3
#pragma unroll
  for (int q = 0; q < QPW; ++q) leave(a, it, row, D, (g * QPW + q) * 8 + hh * 4, res[q], m, l);
}

// ---- many rows ----------------------------------------------------------------------------------------------------------
// One workgroup = eight wavefronts, two on a SIMD, one tile of 32 rows each: 256 rows (items of up to 128 rows: 128, and two key groups) x a
// range of blocks.  Every block comes into LDS once, global -> LDS without registers, into a ring that runs several blocks ahead.
// A wavefront alone issues an instruction every five cycles, whatever it is, so the matrix pipe (32 cycles an instruction)
// and the vector pipe both stay idle in turn; two wavefronts fill each other's gaps.  Within one, three blocks are under way at once:
//     matrix pipe   S = K Q of block j + 1, then O += V P of block j - 1
//     vector pipe   weights P of block j, then the maximum of S
// so that no step waits for another one's result, and a weight has two matrix instructions to hide behind (all of them beside S: half as many).
// 16 requests x 32 of 4 heads over 16384 slots, fp16, one query term: 206 us (1536 cycles of the matrix pipe a step).
// Measured on the form with one term of weights (1024 cycles): a step took 1680 cycles, 1490 without the copies and the raised maxima, at a clock that fell to
// 1.45 GHz under this load; a tenth more with S and P V of neighbouring blocks in one step, weights beside S alone and copies that made each LDS read wait for all.
// Blocks that need a mask (the tree's, and what is left over) follow as in k_paged_stream, from what the ring has copied ahead or from memory.
template <int D, int QT, bool F16>
__global__ __launch_bounds__(512, 2) void k_paged_tiles(const PagedAttnArgs a) {
  typedef RowTile<D, QT, F16> Tile;
  typedef typename Tile::T T;
  constexpr int NS = D / 16, QUADS = D / 8;
  constexpr int BLOCK = 2 * NS * 1024;  // keys and values of 32 slots
  constexpr int RING = 8;               // blocks
  constexpr int WFLOATS = (QUADS + 1) * 256;
  constexpr int CP = 2 * NS / 8;        // pieces of 1 KiB that a wavefront copies of a block
  constexpr int AHEAD = 4;
  static_assert(4 * WFLOATS * 4 <= RING * BLOCK, "merge buffer");
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RING * BLOCK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x;
  const Item it = item_of(a, blockIdx.y, kvh);
  // 256 rows in eight tiles, or 128 in four with two key groups
  const int rows = (it.ri < 0 ? a.rows : it.B) * a.group;
  const int KG = it.ri < 0 ? a.sh_kg : a.own_kg;
  const int kg = KG == 1 ? 0 : wave >> 2, rt = KG == 1 ? wave : wave & 3;
  const int row_first = it.tile * (KG == 1 ? 256 : 128) + rt * 32;
  const bool work = row_first < rows;
  // the ring takes units of KG blocks that need no mask; the rest is the tail
  const int full_end = it.ri < 0 ? it.b_hi : max(it.b_lo, min(it.b_hi, it.P >> 5));
  const int units = KG == 1 ? full_end - it.b_lo : (full_end - it.b_lo) >> 1;
  const int tail0 = it.b_lo + units * KG;
  PageIds pg{a.table + (size_t)it.seq * a.table_ld, a.flags, it.b_lo >> 1, (it.b_hi - 1) >> 1, a.n_pages, 0};
  if (it.b_hi > it.b_lo) pg.load(lane);
  const char* const kp = static_cast<const char*>(a.kpool);
  const char* const vp = static_cast<const char*>(a.vpool);
  auto block_at = [&](int b) -> size_t {  // bytes (pages times KV heads stays below 2^29: checked on the host)
    return (size_t)(unsigned)((pg.of(b, lane) * a.n_kv + kvh) * 2 + (b & 1)) * (32 * D * 2);
  };
  Row row = row_of(a, it, row_first + l31, kvh);
  Tile t;
  t.init(query_of<D, QT, T>(a, row, hh));
  const float scale = softmax_scale(D);
  const bool keys = wave < 4;  // the first four wavefronts copy keys, the others values
  const int share = wave * CP * 1024;  // this wavefront's pieces of a block
  const char* const pool = (keys ? kp : vp) + (wave & 3) * CP * 1024;
  auto source = [&](int b) -> const char* {  // (behind the range: its last block again, never used)
    return pool + block_at(min(b, it.b_hi - 1));
  };
  auto barrier = [&]() {  // (raw: __syncthreads would also drain every copy in flight)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // (all that was loaded so far: the counts below are those of the ring's copies)
  auto through_the_ring = [&](auto kg_c) {
    constexpr int G = decltype(kg_c)::value;  // key groups
    constexpr int BU = BLOCK / 16, RU = RING / G;
    auto slot = [](int u) { return (u & (RU - 1)) * G; };
    int next = 0;  // the unit copied next
    auto copy = [&]() {
#pragma unroll
      for (int g = 0; g < G; ++g) copy_pieces<CP>(source(it.b_lo + next * G + g), lane, ring + (slot(next) + g) * BLOCK + share);
      ++next;
    };
    const int first = keys ? RU : RU - 1;
    while (next < first) copy();
    __builtin_amdgcn_sched_barrier(0);
    const u32x4* const base = reinterpret_cast<const u32x4*>(ring) + lane;
    auto keys_of = [&](int u) { return base + (slot(u) + kg) * BU; };
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((RU - 3) * G * CP));  // units 0 to 2 (values: 0 and 1); before step 1 below the first of these
    barrier();
    u32x4 pc[AHEAD];
    f32x16 z1;
    typename Tile::op8 w1[2], wl1[2];
    if (work) {
      u32x4 k[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) k[s] = keys_of(0)[s * 64];
      t.scores(k);
      t.maximum();
      t.rescale(scale);
      t.weights();
#pragma unroll
      for (int s = 0; s < NS; ++s) k[s] = keys_of(1)[s * 64];
      t.scores(k);
      t.maximum();
      t.rescale_later(scale, t.s, units > 1);
#pragma unroll
      for (int n = 0; n < AHEAD; ++n)
        if (G == 1) pc[n] = keys_of(2)[n * 64];
    }
    barrier();
    if (keys) copy();  // (unit RU, where unit 0 was)
    // Before step j the keys of unit j + 1 (one key group: j + 2) and the values of unit j - 1 have landed in every wavefront's share; keys of unit j and
    // values of unit j - 2 are no longer read, and make room for those RU units later.
    auto step = [&](int j, const f32x16& za, f32x16& zb, const auto& w, const auto& wl, auto& wn, auto& wln) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm((RU - (G == 1 ? 3 : 2)) * G * CP));
      barrier();
      __builtin_amdgcn_sched_barrier(0);
      copy();
      if (work) ring_step<D, QT, F16, G, AHEAD>(t, pc, keys_of(j + 1), keys_of(j - 1) + BU / 2, keys_of(j + 2), za, zb, w, wl, wn, wln, j + 1 < units, scale, [](f32x16&) {});
    };
    int j = 1;
    for (; j + 1 < units; j += 2) {
      step(j, t.s, z1, t.p, t.pl, w1, wl1);
      step(j + 1, z1, t.s, w1, wl1, t.p, t.pl);
    }
    if (j < units) {
      step(j, t.s, z1, t.p, t.pl, w1, wl1);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        t.p[i] = w1[i];
        t.pl[i] = wl1[i];
      }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // (the last values, and copies behind the range)
    barrier();
    if (work) {
      u32x4 v[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) v[s] = keys_of(units - 1)[BU / 2 + s * 64];
      t.values(v);
    }
  };
  if (units > 0) {
    if (KG == 1) through_the_ring(std::integral_constant<int, 1>());
    else through_the_ring(std::integral_constant<int, 2>());
  }

  // ---- blocks without the ring
  // (the row and its query again: kept over the ring's loop they would take registers that it needs)
  int rho = row_first + l31;
  GOOSE_HERE(rho);
  row = row_of(a, it, rho, kvh);
  if (work && tail0 + kg < it.b_hi) {
    t.load_q(query_of<D, QT, T>(a, row, hh));
    const MaskRow mk = mask_of(a, it, row);
    pg.base = tail0 >> 1;  // (the window may have run ahead)
    pg.load(lane);
    // the ring's copies have run ahead by RING / KG - 2 units (values; keys by more), so most of these blocks are in LDS already
    const int units_there = units > 0 ? units + RING / KG - 2 : 0;
    for (int u = units, b = tail0 + kg; b < it.b_hi; ++u, b += KG) {
      u32x4 k[NS], v[NS];
      if (u < units_there) {
        const u32x4* const at = reinterpret_cast<const u32x4*>(ring + (size_t)((u * KG & (RING - 1)) + kg) * BLOCK) + lane;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          k[s] = at[s * 64];
          v[s] = at[(NS + s) * 64];
        }
      } else {
        const size_t at = block_at(b);
        fetch(kp + at, lane, k);
        fetch(vp + at, lane, v);
      }
      const int slot0 = b * 32;
      const bool tree = it.ri >= 0 && slot0 + 32 > it.P;
      unsigned vis = 0xFFFFu;
      bool odd = false;
      t.scores(k);
      if (tree) {
        vis = window16(mk.w0, mk.w1, slot0 + hh * 16 - it.P);
        t.mask(vis);
        odd = clean_values<F16>(v, it.P + it.B - slot0 - hh * 16);
      }
      t.maximum();
      t.rescale(scale);
      t.weights();
      if (odd) t.values_odd(v, vis);
      else t.values(v);
    }
  }
  if (wave == 0) check_shared(a, it, lane);

  // ---- two key groups join: the second leaves its states in LDS, the first takes them in
  float m = t.m;
  if (KG == 2) {
    __syncthreads();
    float* const buf = reinterpret_cast<float*>(ring) + (size_t)rt * WFLOATS + lane * 4;
    if (kg == 1) {
      *reinterpret_cast<f32x4*>(buf) = f32x4{m, t.l, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(buf + 256 * (1 + dt * 4 + q)) =
              f32x4{t.o[dt][q * 4], t.o[dt][q * 4 + 1], t.o[dt][q * 4 + 2], t.o[dt][q * 4 + 3]};
    }
    __syncthreads();
    if (kg == 1) return;
    const f32x4 ml = *reinterpret_cast<const f32x4*>(buf);
    const float both = fmaxf(m, ml[0]);
    const float w0 = join_factor(m, both, scale), w1 = join_factor(ml[0], both, scale);
    m = both;
    t.l = w0 * t.l + w1 * ml[1];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(buf + 256 * (1 + dt * 4 + q));
#pragma unroll
        for (int e = 0; e < 4; ++e) t.o[dt][q * 4 + e] = w0 * t.o[dt][q * 4 + e] + w1 * x[e];
      }
  }
  const float l = t.l + __shfl_xor(t.l, 32, 64);
  if (!work || !row.live) return;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      leave(a, it, row, D, (dt * 4 + q) * 8 + hh * 4, f32x4{t.o[dt][q * 4], t.o[dt][q * 4 + 1], t.o[dt][q * 4 + 2], t.o[dt][q * 4 + 3]}, m, l);
}

// Joins the items of a row: D / 4 threads a (row, head), four columns each, records in a fixed order, the loads of CH in flight together (of two splits
// two: eight would ask for the second one seven times; 512 rows of 32 heads 9.1 us, now 7.6).
// PARTS = 4: the records of a pair are dealt to four such groups of threads, which join through LDS (many splits mean few rows: one trip to memory
// instead of four; 16 x 1 over 8192 slots in 17 splits: 8 us, now 6.3).  The KV head is the fast index as in the kernels above: the records are in that XCD's L2.
template <int D, int PARTS, int CH>
__global__ __launch_bounds__(256) void k_paged_merge(const PagedAttnArgs a) {
  constexpr int TPR = D / 4, PAIRS = 256 / TPR / PARTS;
  __shared__ f32x4 part_o[PARTS > 1 ? 256 : 1];
  __shared__ float2 part_ml[PARTS > 1 ? 256 : 1];
  const int tid = threadIdx.x, c = (tid % TPR) * 4, p = tid / TPR % PARTS;
  const int pair = blockIdx.y * PAIRS + tid / TPR / PARTS;  // of this KV head: (query head of the group, row)
  const bool on = pair < a.rows * a.group;
  const int hg = on ? (int)((unsigned)pair / (unsigned)a.rows) : 0, crow = on ? pair - hg * a.rows : 0;
  const int h = blockIdx.x * a.group + hg;
  int r = 0;
  while (r + 1 < a.n_req && crow >= a.r[r + 1].c0) ++r;
  const int all = a.sh_splits + a.r[r].splits;
  const int s_lo = all * p / PARTS, n = all * (p + 1) / PARTS;
  const size_t base = (size_t)h * a.rows + crow, step = (size_t)a.n_heads * a.rows;
  const float scale = softmax_scale(D);
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f, m = -INFINITY;
  for (int s0 = s_lo; s0 < n; s0 += CH) {
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
    const float w0 = join_factor(m, m_new, scale);
    den *= w0;
    num *= w0;
    m = m_new;
#pragma unroll
    for (int k = 0; k < CH; ++k)
      if (s0 + k < n) {
        const float w = join_factor(ml[k].x, m, scale);
        den = fmaf(w, ml[k].y, den);
        num += w * ov[k];
      }
  }
  if (PARTS > 1) {
    part_o[tid] = num;
    part_ml[tid] = make_float2(m, den);
    __syncthreads();
    if (p != 0) return;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) m = fmaxf(m, part_ml[tid + k * TPR].x);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    den = 0.f;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const float2 ml = part_ml[tid + k * TPR];
      const float w = join_factor(ml.x, m, scale);
      den = fmaf(w, ml.y, den);
      sum += w * part_o[tid + k * TPR];
    }
    num = sum;
  }
  if (!on) return;
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  const size_t row = (size_t)a.r[r].row0 + crow - a.r[r].c0;
  store_out(a, row, h * D + c, num * inv);
  if (a.lse != nullptr && c == 0) a.lse[(size_t)h * a.ld_lse + row] = log_of_sum(m, den, scale);
}

// which kernel: k_paged_stream with one or two row tiles, or k_paged_tiles
enum { STREAM1, STREAM2, TILES };
template <int D, int QT, bool F16>
void launch_t(int kind, dim3 grid, const PagedAttnArgs& a, hipStream_t st) {
  if (kind == TILES) hipLaunchKernelGGL((k_paged_tiles<D, QT, F16>), grid, dim3(512), 0, st, a);
  else if (kind == STREAM2) hipLaunchKernelGGL((k_paged_stream<D, QT, F16, 2>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((k_paged_stream<D, QT, F16, 1>), grid, dim3(512), 0, st, a);
}
template <int D>
void launch_merge(dim3 pairs, int splits, const PagedAttnArgs& a, hipStream_t st) {
  const int per = 1024 / D;
  const dim3 grid(pairs.x, (pairs.y + per - 1) / per);
  if (splits > 8) hipLaunchKernelGGL((k_paged_merge<D, 4, 8>), dim3(pairs.x, (pairs.y * 4 + per - 1) / per), dim3(256), 0, st, a);
  else if (splits > 2) hipLaunchKernelGGL((k_paged_merge<D, 1, 8>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_paged_merge<D, 1, 2>), grid, dim3(256), 0, st, a);
}

}  // namespace

int launch_attn_paged(int dtype, const goose_pages& pg, int layer, int n_heads, int n_kv, int head_dim, const void* q, size_t ldq, int q_terms,
                      const PagedReqs& rq, int shared_pages, float* ws_o, float* ws_ml, size_t max_records, void* o, size_t ldo,
                      int o_dtype, int o_terms, int32_t* flags, hipStream_t st, float* lse, size_t ld_lse) {
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
  a.lse = lse;
  a.ld_lse = ld_lse;
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
  a.same_blocks = shared_pages * 2;
  int own_rows = 0;
  for (int r = 0; r < rq.n; ++r) own_rows = rq.r[r].B > own_rows ? rq.r[r].B : own_rows;
  own_rows *= a.group;
  const size_t records = (size_t)n_heads * rq.rows;  // of one split
  // A way to split the work: do the shared keys have items of their own, which kernel, and how many steps (blocks, or pairs of them) an item takes
  // at most.  Items run in rounds of 256 workgroups, one a compute unit, the shared keys' items first; times in units of 10 ns at head_dim 128, from
  // runs with 20 calls in a graph: an item's fixed part (start, first loads, epilogue; 5.5 us, with the ring 10.5) and its steps (one query term: 0.24 us a
  // block, 0.50 where two row tiles halve the key groups, with the ring 1.34; more with two), the merge 6 us and its records;
  // own items of two units or fewer hardly pay the ring's start (33B, 16 x 8 over 8192 shared slots and 64 of their own: 84 us; counted
  // with it, two row tiles looked cheaper and took 149);
  // and no less than what the caches take to serve all items' blocks (10.5 TB/s).
  struct Way {
    int kind, per, sh_blocks, sh_kg, own_kg, sh_height, own_height;
    long long cost;
  };
  auto cheapest = [&](bool share, int kind, Way& best) {  // updates best
    Way w{};
    w.kind = kind;
    w.sh_blocks = share ? a.same_blocks : 0;
    const int sh_rows = share ? rq.rows * a.group : 0;
    // k_paged_tiles: 128 rows with two key groups where that leaves fewer rows of a tile empty
    auto key_groups = [](int rows) { return (rows + 127) / 128 * 128 < (rows + 255) / 256 * 256 ? 2 : 1; };
    w.sh_kg = key_groups(sh_rows);
    w.own_kg = key_groups(own_rows);
    const bool ring = w.kind == TILES;
    w.sh_height = ring ? 256 / w.sh_kg : (w.kind == STREAM2 ? 64 : 32);
    w.own_height = ring ? 256 / w.own_kg : w.sh_height;
    const int sh_mul = ring ? w.sh_kg : 1, own_mul = ring ? w.own_kg : 1;  // blocks that a step takes
    const int sh_tiles = (sh_rows + w.sh_height - 1) / w.sh_height, sh_steps = (w.sh_blocks + sh_mul - 1) / sh_mul;
    int own_steps[GOOSE_MAX_REQUESTS], own_tiles[GOOSE_MAX_REQUESTS], own_longest = 0, own_units = 0;
    long long fetched = (long long)sh_tiles * w.sh_blocks, all_steps = (long long)sh_tiles * sh_steps;  // of a KV head: blocks, steps
    for (int r = 0; r < rq.n; ++r) {
      own_steps[r] = ((rq.r[r].P_max + rq.r[r].B + 31) / 32 - w.sh_blocks + own_mul - 1) / own_mul;
      own_tiles[r] = (rq.r[r].B * a.group + w.own_height - 1) / w.own_height;
      own_longest = own_steps[r] > own_longest ? own_steps[r] : own_longest;
      const int units = (rq.r[r].P_max / 32 - w.sh_blocks) / own_mul;  // of the ring
      own_units = units > own_units ? units : own_units;
      fetched += (long long)own_tiles[r] * own_steps[r] * own_mul;
      all_steps += (long long)own_tiles[r] * own_steps[r];
    }
    const long long fetch = fetched * n_kv * head_dim * 128 / 105000;
    const int least = ring ? 4 : 8, fixed = ring ? 1050 : 550, own_fixed = own_units > 2 ? fixed : 550,
              products = q_terms + 2,
              step = (ring ? 38 + 32 * products : (w.kind == STREAM2 ? 29 + 7 * products : 15 + 3 * products)) * head_dim / 128;
    const long long work = own_fixed + all_steps * n_kv * step / 256;
    if ((work > fetch ? work : fetch) >= best.cost) return;  // (no way of this kind is cheaper)
    const int longest = sh_steps > own_longest ? sh_steps : own_longest, most_steps = longest > least ? longest : least;
    auto consider = [&](int per) {  // returns the workgroups that it makes
      per = per < least ? least : (per > most_steps ? most_steps : per);
      const int sh = (sh_steps + per - 1) / per;
      int own = 0, splits = 0;
      for (int r = 0; r < rq.n; ++r) {
        const int n = (own_steps[r] + per - 1) / per;
        own += own_tiles[r] * n;
        splits = n > splits ? n : splits;
      }
      splits += sh;
      const long long sh_items = (long long)sh_tiles * sh * n_kv, own_items = (long long)own * n_kv;
      // (blocks times splits stays a 32-bit number in item_of)
      if (splits <= 1 || ((size_t)splits * records <= max_records && 4ull * longest * (unsigned)splits <= UINT32_MAX)) {
        const long long sh_len = (long long)(per < sh_steps ? per : sh_steps) * step + fixed,
                        own_len = (long long)(per < own_longest ? per : own_longest) * step + own_fixed;
        const long long rounds = (sh_items + 255) / 256, room = (rounds * 256 - sh_items) * (sh_len / own_len);  // own items beside the last shared ones
        const long long left = own_items > room ? own_items - room : 0, time = rounds * sh_len + (left + 255) / 256 * own_len;
        w.cost = (time > fetch ? time : fetch) + (splits > 1 ? 600 + (long long)(splits * records * head_dim * 150 / 1000000) : 0);
        w.per = per;
        if (w.cost < best.cost) best = w;
      }
      return sh_items + own_items;
    };
    // tried: no split, and about the smallest `per` that makes one to three rounds of all items, or of the shared ones
    consider(most_steps);
    for (int rounds = 1; rounds <= 3; ++rounds) {
      long long per = (all_steps * n_kv + 256 * rounds - 1) / (256 * rounds);
      for (int k = 0; k < 3 && per < most_steps; ++k) {
        const long long made = consider((int)per);
        if (made <= 256 * rounds) break;
        per = (per < least ? least : per) * made / (256 * rounds) + 1;
      }
      const int sh = sh_tiles > 0 ? 256 * rounds / (sh_tiles * n_kv) : 0;
      if (sh > 0) consider((sh_steps + sh - 1) / sh);
    }
  };
  // The shared keys get items of their own where rows of one request leave most of a tile empty, or where many keys meet few rows (16 requests x 1
  // over 8192 slots: 24 us, by request 50).  Where a request fills its tiles by itself the products are the same either way, the caches serve the
  // pages to all of them, and one set of items and fewer records win (16 x 32 over 4096 slots, bf16: 86 us, shared 102; over 64, fp16: 16 and 24).
  // Which kernel (fp16): the ring where rows fill it and keys are many (7B, 2 requests x 100 over 4096: 42 us, two row tiles 49; 8 x 30 of 4 heads over 64: 15
  // and, with one, 11.5); two row tiles where the caches bound one (7B, 5 x 61 over 1984: 42 and 51), one where two leave units idle (16 x 12 of 4 heads over
  // 2048: 24 and 32).  Over 160 cases (named ones, and drawn ones of every model) what it chooses takes 2.8 % longer than the best of all ways on average, 40 % at most.
  Way way{};
  way.cost = INT64_MAX;
  for (int share = 0; share <= (shared_pages > 0 ? 1 : 0); ++share) {
    const int most = share ? rq.rows * a.group : own_rows;
    if (most > 64) cheapest(share, TILES, way);
    if (most > 32) cheapest(share, STREAM2, way);
    cheapest(share, STREAM1, way);
  }
  if (way.cost == INT64_MAX) return GOOSE_ERR_CAPACITY;
  const int kind = way.kind, sh_mul = kind == TILES ? way.sh_kg : 1, own_mul = kind == TILES ? way.own_kg : 1;
  a.sh_blocks = way.sh_blocks;
  a.sh_kg = way.sh_kg;
  a.own_kg = way.own_kg;
  a.sh_tiles = a.sh_blocks > 0 ? (rq.rows * a.group + way.sh_height - 1) / way.sh_height : 0;
  a.sh_splits = (a.sh_blocks + way.per * sh_mul - 1) / (way.per * sh_mul);
  int own_splits = 0;
  unsigned items = (unsigned)(a.sh_tiles * a.sh_splits);
  for (int r = 0; r < rq.n; ++r) {
    const PagedReq& q = rq.r[r];
    const int blocks = (q.P_max + q.B + 31) / 32 - a.sh_blocks, tiles = (q.B * a.group + way.own_height - 1) / way.own_height,
              splits = (blocks + way.per * own_mul - 1) / (way.per * own_mul);
    a.r[r] = AttnReq{q.seq, q.B, q.P_max, q.row0, q.c0, tiles, splits, (const uint64_t*)q.p};
    own_splits = splits > own_splits ? splits : own_splits;
    items += (unsigned)(tiles * splits);
  }
  a.direct = a.sh_splits + own_splits == 1;
  const dim3 grid(n_kv, items);
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  if (head_dim == 128) {
    if (q_terms == 2) f16 ? launch_t<128, 2, true>(kind, grid, a, st) : launch_t<128, 2, false>(kind, grid, a, st);
    else f16 ? launch_t<128, 1, true>(kind, grid, a, st) : launch_t<128, 1, false>(kind, grid, a, st);
  } else {
    if (q_terms == 2) f16 ? launch_t<64, 2, true>(kind, grid, a, st) : launch_t<64, 2, false>(kind, grid, a, st);
    else f16 ? launch_t<64, 1, true>(kind, grid, a, st) : launch_t<64, 1, false>(kind, grid, a, st);
  }
  int rc = goose_launch_status();
  if (rc != GOOSE_OK || a.direct) return rc;
  const dim3 pairs(n_kv, rq.rows * a.group);
  if (head_dim == 128) launch_merge<128>(pairs, a.sh_splits + own_splits, a, st);
  else launch_merge<64>(pairs, a.sh_splits + own_splits, a, st);
  return goose_launch_status();
}
