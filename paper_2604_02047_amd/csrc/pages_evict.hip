// Lengths of a paged cache that change by whole chunks: the commit of new tokens, and eviction.
//
// An eviction keeps, per layer and KV head, the first `sink` slots, the last `recent` ones and the heaviest of the others.  Three launches:
//   k_evict_select  a workgroup per (layer, KV head): the m-th largest weight by radix selection over order-preserving bit patterns
//                   (2048 + 2048 + 1024 bins), ties to the lowest slots, the kept slots as bit words, weights to the front
//   k_evict_move    one, four or eight wavefronts per (layer, KV head, K or V, 2 KiB of a 32-slot block): the blocks stream through registers in order,
//                   kept rows are collected in LDS and leave as whole blocks.  In place: a destination block never lies behind the
//                   block that its last row came from, and blocks ahead are only read
//   k_evict_settle  lengths and pages (the last workgroup to move could do it, but thousands that count themselves in one word cost more than the launch:
//                   13B, 8 layers of 4 sequences of 28 slots 139 us against 67)
// What bounds it: memory, where there is much to move (the move of Llama 3 8B heads, 8 layers of 4 sequences from 8192 to 2048 slots that lie anywhere: 1.33 GB in 285 us, 4.7 TB/s;
// 7B, 4 layers of 2 from 3001 to 2500: 0.73 GB in 128 to 147 us), else the launches and the trips to memory that follow from each other.  (Where earlier cuts have left the heavy slots
// side by side there is less to read: the same 8192 to 2048 over and over on one cache, whose old weights stay behind the cut, come down from 320 to 185 us a call.)
// A rotation by the position that a key gives up needs both halves of its pairs, which is why a wavefront of the keys has columns
// 16 u .. 16 u + 15 and those d/2 further.
#include "mma16.h"
#include "paged.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

__device__ inline void release(const goose_pages& pg, size_t at, int32_t* flags) {
  const int e = pg.d_table[at];
  if (e == -1) return;
  pg.d_table[at] = -1;
  if ((unsigned)e >= (unsigned)pg.n_pages) { atomicOr(flags, GOOSE_FLAG_PAGES); return; }
  if (atomicSub(&pg.d_refs[e], 1) < 1) {  // a count that was wrong before: back to free
    atomicAdd(&pg.d_refs[e], 1);
    atomicOr(flags, GOOSE_FLAG_PAGES);
  }
}

// A workgroup a chunk.
__global__ __launch_bounds__(256) void k_pages_append(const goose_pages pg, const ChunkReqs ck, int32_t* __restrict__ flags) {
  const ChunkReq& q = ck.r[blockIdx.x];
  const int tid = threadIdx.x, P = pg.d_len[q.seq];
  const size_t row = (size_t)q.seq * pg.table_ld;
  if (P < 0 || (long long)P + q.C > (long long)pg.table_ld * GOOSE_PAGE) {
    if (tid == 0) atomicOr(flags, GOOSE_FLAG_CAPACITY);
    return;
  }
  const int end = P + q.C, behind = (end + GOOSE_PAGE - 1) / GOOSE_PAGE;
  bool bad = false;
  for (int i = P / GOOSE_PAGE + tid; i < behind; i += 256) {
    const int e = pg.d_table[row + i];
    bad = bad || (unsigned)e >= (unsigned)pg.n_pages || pg.d_refs[e] != 1;
  }
  if (__syncthreads_or(bad)) {  // (and every thread has the old length)
    if (tid == 0) atomicOr(flags, GOOSE_FLAG_PAGES);
    return;
  }
  for (int i = behind + tid; i < pg.table_ld; i += 256) release(pg, row + i, flags);
  if (tid == 0) pg.d_len[q.seq] = end;
}

// Larger weights have larger keys; -0 is 0; a NaN is below every number.
__device__ __forceinline__ unsigned key_of(float w) {
  if (w != w) return 0;
  const unsigned u = __builtin_bit_cast(unsigned, w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which flags a request raises instead of being cut (every workgroup of a launch that changes no table comes to the same verdict).
// mine: entry tid of its table (asked for beside the length).
template <int NT>
__device__ inline int verdict_of(const goose_pages& pg, const goose_eviction& q, int len, int tid, int mine) {
  if (len < 0 || (long long)len > (long long)pg.table_ld * GOOSE_PAGE) return GOOSE_FLAG_CAPACITY;
  const int pages = (len + GOOSE_PAGE - 1) / GOOSE_PAGE;
  // pages that rows move into must be the sequence's own
  const bool moves = q.keep < len && q.sink < q.keep;
  const int own_lo = q.sink / GOOSE_PAGE, own_hi = moves ? (q.keep - 1) / GOOSE_PAGE : -1;
  bool bad = false;
  for (int i = tid; i < pages; i += NT) {
    const int e = i == tid ? mine : pg.d_table[(size_t)q.seq * pg.table_ld + i];
    bad = bad || (unsigned)e >= (unsigned)pg.n_pages || (i >= own_lo && i <= own_hi && pg.d_refs[e] != 1);
  }
  return __syncthreads_or(bad) ? GOOSE_FLAG_PAGES : 0;
}

// What the wavefronts in front of this one have left in ws, and all of them.
template <int W>
__device__ __forceinline__ void sums_of(const int (&ws)[W], int wave, int* before, int* all) {
  int v[W];
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = ws[i];
  *before = *all = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    *before += i < wave ? v[i] : 0;
    *all += v[i];
  }
}

// Sum of x over the lanes in front: within rows of 16 by shifts, then from the last lane of a row to the next row, and of the first half to the second.
__device__ __forceinline__ int lanes_before(int x) {
  int sum = x;
#define GOOSE_ADD(CONTROL, ROWS) sum += __builtin_amdgcn_update_dpp(0, sum, CONTROL, ROWS, 0xF, false)
  GOOSE_ADD(0x111, 0xF);
  GOOSE_ADD(0x112, 0xF);
  GOOSE_ADD(0x114, 0xF);
  GOOSE_ADD(0x118, 0xF);
  GOOSE_ADD(0x142, 0xA);
  GOOSE_ADD(0x143, 0xC);
#undef GOOSE_ADD
  return sum - x;
}

// Latency counts here, not bandwidth.  What does not depend on the length is loaded beside it; the slots that the workgroup takes at a time, WORDS words a
// wavefront, stay in LDS over all passes where they are all there are; and loops stay rolled, since code that runs once is paid for by its bytes
// (10 KB unrolled; 200 slots of 8 heads 8.8 us, 10.1 so; 256 heads of 8192 slots 17 us).
template <int NT>
__global__ __launch_bounds__(NT) void k_evict_select(const goose_pages pg, const Evictions ev, int n_layers, int n_kv, float* __restrict__ weight,
                                                     uint64_t* __restrict__ kept, int32_t* __restrict__ verdict) {
  constexpr int WORDS = 8, SEG = NT * WORDS, W = NT / 64, PER = 2048 / NT;  // PER: bins of a thread
  __shared__ __attribute__((aligned(32))) unsigned hist[2048];
  __shared__ float seg[SEG];
  __shared__ __attribute__((aligned(16))) int ws[W], wt[W];
  __shared__ int found[3];
  const goose_eviction q = ev.r[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int layer = blockIdx.x / n_kv, head = blockIdx.x - layer * n_kv;
  uint64_t* const words = kept + (((size_t)blockIdx.y * n_layers + layer) * n_kv + head) * pg.table_ld;
  float* const w = weight + (((size_t)layer * pg.n_seqs + q.seq) * n_kv + head) * pg.table_ld * GOOSE_PAGE;
  float* const own = seg + wave * WORDS * GOOSE_PAGE + lane;  // of words first_word .. first_word + WORDS - 1
  auto fetch = [&](int first_word, int end) {
    float v[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v[i] = first_word + i < end ? w[(size_t)(first_word + i) * GOOSE_PAGE + lane] : 0.f;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) own[i * GOOSE_PAGE] = v[i];
  };
  const int mine = tid < pg.table_ld ? pg.d_table[(size_t)q.seq * pg.table_ld + tid] : 0;
  const int len = __builtin_amdgcn_readfirstlane(pg.d_len[q.seq]);
  fetch(wave * WORDS, pg.table_ld);
#pragma unroll 1
  for (int j = tid; j < 2048; j += NT) hist[j] = 0;
  const int bad = verdict_of<NT>(pg, q, len, tid, mine);
  const int n_words = bad ? 0 : (len + GOOSE_PAGE - 1) / GOOSE_PAGE;
  auto close = [&]() {  // (behind everything else: a barrier would wait for these stores)
    if (blockIdx.x == 0 && tid == 0) verdict[blockIdx.y] = bad;
    if (!bad)
      for (int i = n_words + tid; i < pg.table_ld; i += NT) words[i] = 0;
  };
  if (bad) return close();
  if (len <= q.keep) {
    for (int i = tid; i < n_words; i += NT) {
      const int m = min(GOOSE_PAGE, len - i * GOOSE_PAGE);
      words[i] = m == 64 ? ~0ull : (1ull << m) - 1;
    }
    return close();
  }
  // ---- the m-th largest weight of slots lo .. hi - 1: its key, and how many slots of just that weight are kept (ties)
  const int lo = q.sink, hi = len - q.recent, m = q.keep - q.sink - q.recent;
  const bool one = len <= SEG;
  unsigned key = 0;
  int ties = 0;
  if (m > 0) {
    ties = m;
    int shift = 21;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int bins = pass < 2 ? 2048 : 1024;
      const unsigned above = pass == 0 ? 0u : key >> (pass == 1 ? 21 : 10);
#pragma unroll 1
      for (unsigned c0 = one ? 0 : (unsigned)lo / SEG * SEG; c0 < (unsigned)hi; c0 += SEG) {
        const int first = (int)(c0 >> 6) + wave * WORDS;
        if (!one) fetch(first, n_words);
        const int some_words = min(WORDS, n_words - first);
#pragma unroll 1
        for (int i = 0; i < some_words; ++i) {
          const int s = (first + i) * GOOSE_PAGE + lane;
          const unsigned x = key_of(own[i * GOOSE_PAGE]);
          if (s >= lo && s < hi && (pass == 0 || x >> (pass == 1 ? 21 : 10) == above)) {
            const unsigned bin = (x >> shift) & (bins - 1), some = __builtin_amdgcn_readfirstlane(bin);
            const uint64_t here = __builtin_amdgcn_ballot_w64(true);
            if (__builtin_amdgcn_ballot_w64(bin == some) == here) {  // (equal weights would come one after the other)
              if ((here & ((1ull << lane) - 1)) == 0) atomicAdd(&hist[some], (unsigned)__popcll(here));
            } else {
              atomicAdd(&hist[bin], 1u);
            }
          }
        }
      }
      __syncthreads();
      // thread t owns PER bins, from the top: how many slots lie above them
      const int top = bins - 1 - PER * tid;
      typedef int Bins __attribute__((ext_vector_type(PER)));
      int c[PER], x = 0;
      Bins some = 0;
      if (top >= 0) {
        Bins* const at = reinterpret_cast<Bins*>(&hist[top + 1 - PER]);
        some = *at;
        *at = 0;  // (for the next pass)
      }
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        c[j] = some[PER - 1 - j];
        x += c[j];
      }
      const int mine_before = lanes_before(x);
      if (lane == 63) ws[wave] = mine_before + x;
      __syncthreads();
      int before, all;
      sums_of(ws, wave, &before, &all);
      before += mine_before;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (before < ties && ties <= before + c[j]) { found[0] = top - j; found[1] = before; found[2] = c[j]; }
        before += c[j];
      }
      __syncthreads();
      key |= (unsigned)found[0] << shift;
      ties -= found[1];
      if (ties == found[2] && key != 0) {  // all of this bin stay: no need to look into it
        --key;
        ties = 0;
        break;
      }
      shift = pass == 0 ? 10 : 0;
    }
  }
  // ---- the words, ties to the lowest slots, and weights to the front: none of them is behind where it goes, and all of a segment are loaded before one
  // is stored.  Lane i has word i of the wavefront.
  int left = ties, base = 0;
#pragma unroll 1
  for (unsigned c0 = 0; c0 < (unsigned)len; c0 += SEG) {
    const int first = (int)(c0 >> 6) + wave * WORDS, some_words = min(WORDS, n_words - first);
    if (!one) fetch(first, n_words);
    uint64_t same = 0, stay = 0;
#pragma unroll 1
    for (int i = 0; i < some_words; ++i) {
      const int s = (first + i) * GOOSE_PAGE + lane;
      const unsigned x = key_of(own[i * GOOSE_PAGE]);
      const bool mid = m > 0 && s >= lo && s < hi;
      const uint64_t equal = __builtin_amdgcn_ballot_w64(mid && x == key);
      const uint64_t more = __builtin_amdgcn_ballot_w64(s < lo || (s >= hi && s < len) || (mid && x > key));
      if (lane == i) { same = equal; stay = more; }
    }
    const int n_same = (int)__popcll(same), same_before = lanes_before(n_same);
    if (lane == 63) wt[wave] = same_before + n_same;
    __syncthreads();
    int before, all;
    sums_of(wt, wave, &before, &all);
    const int take = min(max(left - before - same_before, 0), n_same);  // of its word's ties
    left -= all;
    uint64_t rest = same;
    if (take == n_same) rest = 0;
    else for (int k = 0; k < take; ++k) rest &= rest - 1;
    stay |= same & ~rest;
    const int n_stay = (int)__popcll(stay), stay_before = lanes_before(n_stay);
    if (lane == 63) ws[wave] = stay_before + n_stay;
    __syncthreads();
    sums_of(ws, wave, &before, &all);
    if (lane < some_words) words[first + lane] = stay;
#pragma unroll 1
    for (int i = 0; i < some_words; ++i) {
      const uint64_t word = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(stay >> 32), i) << 32 | (unsigned)__builtin_amdgcn_readlane((int)stay, i);
      const int at = base + before + __builtin_amdgcn_readlane(stay_before, i);
      if ((word >> lane) & 1) w[at + (int)__popcll(word & ((1ull << lane) - 1))] = own[i * GOOSE_PAGE];
    }
    base += all;
    if (!one) __syncthreads();
  }
  close();
}

__device__ __forceinline__ void in_order() {  // LDS of one wavefront: its instructions execute in order, the compiler is to keep them so
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// Sine and cosine of 2 pi t for |t| <= 1/2: power series on an eighth of a turn to both sides (what they leave out is below 2^-25).
__device__ __forceinline__ void turn(float t, float* sine, float* cosine) {
  const float k = rintf(4.f * t), x = fmaf(k, -0.25f, t) * 6.2831853071795865f, z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int q = (int)k;
  const float a = (q & 1) ? c : s, b = (q & 1) ? s : c;
  *sine = (q & 2) ? -a : a;
  *cosine = ((q + 1) & 2) ? -b : b;
}

// A window is NW * AHEAD blocks, AHEAD in a row a wavefront.  Its rows go into LDS, at the places of the destination blocks that they fill, while the next
// window's loads are on their way; then the blocks that are full leave, and the wavefronts take turns at them.
template <int D, bool F16, int NW>
__global__ __launch_bounds__(64 * NW) void k_evict_move(const goose_pages pg, const Evictions ev, int n_layers, int n_kv, const double* __restrict__ inv_freq,
                                                        const uint64_t* __restrict__ kept, bool reposition, const int32_t* __restrict__ verdict) {
  typedef typename Mma16<F16>::T T;
  typedef typename Mma16<F16>::v8 op8;
  constexpr int UNITS = D / 32, AHEAD = NW == 1 ? 6 : 3, WINDOW = NW * AHEAD, STAGES = NW == 8 ? 32 : (NW == 4 ? 16 : 8);
  static_assert(WINDOW + 1 <= STAGES, "a window reaches into WINDOW + 1 destination blocks");
  // Destination blocks that fill up.  Keys: [block % STAGES][piece][...], and the slots that they come from.  Values: [column][slot % (32 STAGES)], a column's slots
  // turned on by eight against those of the one before (else all would be in one bank), and behind them what takes the slots that go.
  constexpr unsigned RING = STAGES * 32;
  __shared__ __attribute__((aligned(16))) unsigned short stage[32 * RING + 64];
  __shared__ int from[STAGES][32];
  const goose_eviction q = ev.r[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l31 = lane & 31, hh = lane >> 5;
  const int len = __builtin_amdgcn_readfirstlane(pg.d_len[q.seq]);
  if (__builtin_amdgcn_readfirstlane(verdict[blockIdx.y]) != 0 || len <= q.keep || q.sink >= q.keep) return;
  auto sync = [&]() {  // LDS only: __syncthreads would wait for every load in flight
    if constexpr (NW == 1) {
      in_order();
    } else {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
  };
  const int lh = blockIdx.x / (2 * UNITS), unit = blockIdx.x - lh * (2 * UNITS);
  const int layer = lh / n_kv, head = lh - layer * n_kv;
  const bool keys = unit < UNITS;
  const int p0 = keys ? unit : 2 * (unit - UNITS), p1 = keys ? unit + UNITS : p0 + 1;  // its two pieces of a block's 1 KiB pieces
  T* const pool = static_cast<T*>(keys ? pg.d_kpool : pg.d_vpool) + (size_t)layer * pg.n_pages * n_kv * (GOOSE_PAGE * D);
  const int32_t* const row = pg.d_table + (size_t)q.seq * pg.table_ld;
  const uint64_t* const words = kept + (((size_t)blockIdx.y * n_layers + layer) * n_kv + head) * pg.table_ld;
  auto block_of = [&](int page, int b) -> T* { return pool + ((size_t)page * n_kv + head) * (GOOSE_PAGE * D) + (size_t)(b & 1) * 32 * D + lane * 8; };
  // a lane of the keys has eight columns of slot kk of a block; one of the values has 16 slots of a column: 16 hh to 16 hh + 15
  const int kk = ((l31 >> 2) & 1) * 16 + (l31 >> 3) * 4 + (l31 & 3);
  double turns[8];  // of a pair from one position to the next
  if (keys && reposition) {
#pragma unroll
    for (int e = 0; e < 8; ++e) turns[e] = inv_freq[unit * 16 + hh * 8 + e] * 0.15915494309189533577;
  }
  u32x4 r0[AHEAD], r1[AHEAD];
  unsigned masks[AHEAD];
  int blocks[AHEAD], places[AHEAD];  // which they are, and where their first kept rows go
  // Only blocks of which something stays are looked at (8192 to 512 slots: level at 186 us where they lie anywhere, 108 -> 73 where earlier cuts left them side by side).  Ids and words of 64 pages at a time, one a lane, with a sum over the lanes
  // of kept rows and of such blocks; ids where rows go (which never steps ahead of that): asked for block by block they would be two trips to memory each.
  const int pages = (len + GOOSE_PAGE - 1) / GOOSE_PAGE;
  int src0 = q.sink / GOOSE_PAGE, dst0 = src0, src_ids, dst_ids, sum;  // sum: blocks << 16 | rows
  int rows_passed = src0 * GOOSE_PAGE, blocks_passed = 0;  // in front of these pages (all slots in front of the first stay)
  uint64_t src_words;
  auto src_window = [&]() {
    const int i = min(src0 + lane, pages - 1);
    src_ids = row[i];
    const uint64_t word = words[i];
    src_words = src0 + lane < pages ? word : 0;
    sum = (int)__popcll(src_words) + (((unsigned)src_words != 0) + ((src_words >> 32) != 0)) * 65536;
    sum += lanes_before(sum);
  };
  // the n-th such block (n never falls): its number or -1, its word, its page, and how many kept rows lie in front of it
  auto find = [&](int n, unsigned* word, int* page, int* before) -> int {
    for (int all; n - blocks_passed >= (all = __builtin_amdgcn_readlane(sum, 63)) >> 16;) {
      if (src0 + 64 >= pages) return -1;
      blocks_passed += all >> 16;
      rows_passed += all & 0xFFFF;
      src0 += 64;
      src_window();
    }
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum >> 16 > n - blocks_passed)), upto = __builtin_amdgcn_readlane(sum, l);
    const unsigned low = (unsigned)__builtin_amdgcn_readlane((int)src_words, l), high = (unsigned)__builtin_amdgcn_readlane((int)(src_words >> 32), l);
    // (the last of its page's if the sum up to there leaves none behind it)
    const bool second = high != 0 && upto >> 16 == n - blocks_passed + 1;
    *word = second ? high : low;
    *page = __builtin_amdgcn_readlane(src_ids, l);
    *before = rows_passed + (upto & 0xFFFF) - __popc(high) - (second ? 0 : __popc(low));
    return 2 * (src0 + l) + (second ? 1 : 0);
  };
  src_window();
  dst_ids = src_ids;
  const T* fetched = block_of(__builtin_amdgcn_readlane(src_ids, 0), 2 * src0);
  // (Always a load, of the last block again behind the end: one that may or may not be in flight would make the others wait for all.)
  auto load = [&](int n, unsigned& mask, int& block, int& place, u32x4& x, u32x4& y) {
    int page;
    block = find(n, &mask, &page, &place);
    if (block >= 0) fetched = block_of(page, block);
    else mask = 0;
    x = *reinterpret_cast<const u32x4*>(fetched + p0 * 512);
    y = *reinterpret_cast<const u32x4*>(fetched + p1 * 512);
  };
  // whole destination block b, or its first n < 32 slots.  Keys are turned here, where every lane has one that is kept
  auto flush = [&](int b, int n) {
    while ((b >> 1) - dst0 >= 64) { dst0 += 64; dst_ids = row[min(dst0 + lane, pages - 1)]; }
    T* const p = block_of(__builtin_amdgcn_readlane(dst_ids, (b >> 1) - dst0), b);
    u32x4 x, y;
    if (keys) {
      x = *reinterpret_cast<const u32x4*>(&stage[(b & (STAGES - 1)) * 1024 + lane * 8]);
      y = *reinterpret_cast<const u32x4*>(&stage[(b & (STAGES - 1)) * 1024 + 512 + lane * 8]);
    } else {
      const unsigned at = (unsigned)(b * 32 + hh * 16 + l31 * 8);
      x = *reinterpret_cast<const u32x4*>(&stage[l31 * RING + (at & (RING - 1))]);
      y = *reinterpret_cast<const u32x4*>(&stage[l31 * RING + ((at + 8) & (RING - 1))]);
    }
    if (keys && reposition) {
      const int delta = b * 32 + kk - from[b & (STAGES - 1)][kk];
      if (delta != 0 && kk < n) {
        op8 lo = __builtin_bit_cast(op8, x), hi = __builtin_bit_cast(op8, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          double t = (double)delta * turns[e];
          t -= rint(t);
          float sn, c;
          turn((float)t, &sn, &c);
          const float u = (float)lo[e], v = (float)hi[e];
          lo[e] = (T)(u * c - v * sn);
          hi[e] = (T)(v * c + u * sn);
        }
        x = __builtin_bit_cast(u32x4, lo);
        y = __builtin_bit_cast(u32x4, hi);
      }
    }
    if (n == 32 || (keys && kk < n)) {
      *reinterpret_cast<u32x4*>(p + p0 * 512) = x;
      *reinterpret_cast<u32x4*>(p + p1 * 512) = y;
    } else if (!keys) {
      const u16x8 a = __builtin_bit_cast(u16x8, x), c = __builtin_bit_cast(u16x8, y);
      unsigned short* const d0 = reinterpret_cast<unsigned short*>(p + p0 * 512);
      unsigned short* const d1 = reinterpret_cast<unsigned short*>(p + p1 * 512);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (hh * 16 + e < n) d0[e] = a[e];
        if (hh * 16 + 8 + e < n) d1[e] = c[e];
      }
    }
  };
  auto place = [&](int b, unsigned mask, int at, const u32x4& x, const u32x4& y) {
    if (mask == 0) return;
    if (keys) {
      const int to = at + __popc(mask & ((1u << kk) - 1)), d = to & 31;
      if ((mask >> kk) & 1) {
        const int l = (((d >> 2) & 3) << 3 | (d >> 4) << 2 | (d & 3)) + 32 * hh;
        *reinterpret_cast<u32x4*>(&stage[((to >> 5) & (STAGES - 1)) * 1024 + l * 8]) = x;
        *reinterpret_cast<u32x4*>(&stage[((to >> 5) & (STAGES - 1)) * 1024 + 512 + l * 8]) = y;
        from[(to >> 5) & (STAGES - 1)][d] = b * 32 + kk;
      }
    } else {
      // (every slot is written, those that go behind the ring: no branches)
      const u16x8 a = __builtin_bit_cast(u16x8, x), c = __builtin_bit_cast(u16x8, y);
      const int mine = (int)(hh ? mask >> 16 : mask & 0xFFFFu);
      unsigned to = (unsigned)(at + (hh ? __popc(mask & 0xFFFFu) : 0) + l31 * 8);
      const unsigned column = l31 * RING, gone = 32 * RING + lane;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const unsigned stays = (unsigned)((mine << (31 - e)) >> 31);  // all ones or none
        const unsigned there = (to & (RING - 1)) | column;
        stage[(there & stays) | (gone & ~stays)] = e < 8 ? a[e & 7] : c[e & 7];
        to -= stays;
      }
    }
  };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) load(wave * AHEAD + k, masks[k], blocks[k], places[k], r0[k], r1[k]);
  // (one copy of flush: its code would not fit the instruction cache several times)
  int done = 2 * dst0;  // destination blocks written
#pragma unroll 1
  for (int n = WINDOW;; n += WINDOW) {
    unsigned word;
    int page, rows;  // that the windows so far hold
    const bool last = find(n, &word, &page, &rows) < 0;
    if (last) rows = q.keep;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      place(blocks[k], masks[k], places[k], r0[k], r1[k]);
      load(n + wave * AHEAD + k, masks[k], blocks[k], places[k], r0[k], r1[k]);
    }
    sync();
    const int full = last ? (rows + 31) >> 5 : rows >> 5;
#pragma unroll 1
    for (int d = done + wave; d < full; d += NW) flush(d, min(32, rows - d * 32));
    done = full;
    if (last) break;
    sync();
  }
}

__global__ __launch_bounds__(256) void k_evict_settle(const goose_pages pg, const Evictions ev, const int32_t* __restrict__ verdict,
                                                      int32_t* __restrict__ flags) {
  const goose_eviction q = ev.r[blockIdx.x];
  const int bad = verdict[blockIdx.x], len = pg.d_len[q.seq];
  __syncthreads();  // every thread has the old length
  if (bad) {
    if (threadIdx.x == 0) atomicOr(flags, bad);
    return;
  }
  if (len <= q.keep) return;
  for (int i = (q.keep + GOOSE_PAGE - 1) / GOOSE_PAGE + threadIdx.x; i < pg.table_ld; i += 256) release(pg, (size_t)q.seq * pg.table_ld + i, flags);
  if (threadIdx.x == 0) pg.d_len[q.seq] = q.keep;
}

}  // namespace

int launch_pages_append(const goose_pages& pg, const ChunkReqs& ck, int32_t* flags, hipStream_t st) {
  hipLaunchKernelGGL(k_pages_append, dim3(ck.n), dim3(256), 0, st, pg, ck, flags);
  return goose_launch_status();
}

int launch_pages_evict(int dtype, const goose_pages& pg, const Evictions& ev, int n_layers, int n_kv, int head_dim, const double* inv_freq,
                       float* weight, uint64_t* kept, bool reposition, PageScratch* scratch, int32_t* flags, hipStream_t st) {
  // Where 256 threads' segment in LDS holds a whole table: workgroups of that size, of which more run side by side (1280 heads of 28 slots 11 us, with 1024 55).
  const dim3 heads(n_layers * n_kv, ev.n);
  if (pg.table_ld * GOOSE_PAGE <= 2048)
    hipLaunchKernelGGL(k_evict_select<256>, heads, dim3(256), 0, st, pg, ev, n_layers, n_kv, weight, kept, scratch->verdict);
  else
    hipLaunchKernelGGL(k_evict_select<1024>, heads, dim3(1024), 0, st, pg, ev, n_layers, n_kv, weight, kept, scratch->verdict);
  int rc = goose_launch_status();
  if (rc != GOOSE_OK) return rc;
  // Wavefronts of a stream of blocks, by the streams and the slots that a sequence may have.  us a call with 1 / 4 / 8, from slots that lie anywhere: 64 streams (Llama 3 8B, one
  // layer of 8192 slots to 2048) 215 / 89 / 63; 512 (8 layers) 250 / 116 / 104; 1024 (two sequences) 282 / 172 / 172; 2048 (four) 352 / 313 / 310; 5120 of 500 slots to 250
  // 100 / 90 / 95; 10240 of 28 slots to 14 41 / 59 / 92, of 100 to 70 70 / 79 / 118.
  const dim3 grid(n_layers * n_kv * (head_dim / 16), ev.n);
  const long long streams = (long long)grid.x * grid.y;
  const bool f16 = dtype == GOOSE_DTYPE_F16;
  const int waves = streams <= 512 ? 8 : (streams > 2048 && pg.table_ld <= 4 ? 1 : 4);
#define GOOSE_MOVE(D, H, NW) hipLaunchKernelGGL((k_evict_move<D, H, NW>), grid, dim3(64 * NW), 0, st, pg, ev, n_layers, n_kv, inv_freq, kept, reposition, scratch->verdict)
#define GOOSE_MOVE_D(D, H) do { if (waves == 8) GOOSE_MOVE(D, H, 8); else if (waves == 4) GOOSE_MOVE(D, H, 4); else GOOSE_MOVE(D, H, 1); } while (0)
  if (head_dim == 128) { if (f16) GOOSE_MOVE_D(128, true); else GOOSE_MOVE_D(128, false); }
  else if (head_dim == 64) { if (f16) GOOSE_MOVE_D(64, true); else GOOSE_MOVE_D(64, false); }
  else return GOOSE_ERR_SHAPE;
#undef GOOSE_MOVE_D
#undef GOOSE_MOVE
  rc = goose_launch_status();
  if (rc != GOOSE_OK) return rc;
  hipLaunchKernelGGL(k_evict_settle, dim3(ev.n), dim3(256), 0, st, pg, ev, scratch->verdict, flags);
  return goose_launch_status();
}
