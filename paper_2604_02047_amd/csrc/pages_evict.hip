// Lengths of a paged cache that change by whole chunks: the commit of new tokens, and eviction.
//
// An eviction keeps, per layer and KV head, the first `sink` slots, the last `recent` ones and the heaviest of the others.  Three launches:
//   k_evict_select  a workgroup per (layer, KV head): the m-th largest weight by radix selection over order-preserving bit patterns
//                   (2048 + 2048 + 1024 bins), ties to the lowest slots, the kept slots as bit words, weights to the front
//   k_evict_move    a wavefront per (layer, KV head, K or V, 2 KiB of a 32-slot block): the blocks stream through registers in order,
//                   kept rows are collected in LDS and leave as whole blocks.  In place: a destination block never lies behind the
//                   block that its last row came from, and blocks ahead are only read.
//   k_evict_settle  lengths and pages
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

constexpr int NT = 1024;

// Larger weights have larger keys; -0 is 0; a NaN is below every number.
__device__ __forceinline__ unsigned key_of(float w) {
  if (w != w) return 0;
  const unsigned u = __builtin_bit_cast(unsigned, w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which flags a request raises instead of being cut (every workgroup of a launch that changes no table comes to the same verdict).
__device__ inline int verdict_of(const goose_pages& pg, const goose_eviction& q, int len, int tid) {
  if (len < 0 || (long long)len > (long long)pg.table_ld * GOOSE_PAGE) return GOOSE_FLAG_CAPACITY;
  const int pages = (len + GOOSE_PAGE - 1) / GOOSE_PAGE;
  // pages that rows move into must be the sequence's own
  const bool moves = q.keep < len && q.sink < q.keep;
  const int own_lo = q.sink / GOOSE_PAGE, own_hi = moves ? (q.keep - 1) / GOOSE_PAGE : -1;
  bool bad = false;
  for (int i = tid; i < pages; i += NT) {
    const int e = pg.d_table[(size_t)q.seq * pg.table_ld + i];
    bad = bad || (unsigned)e >= (unsigned)pg.n_pages || (i >= own_lo && i <= own_hi && pg.d_refs[e] != 1);
  }
  return __syncthreads_or(bad) ? GOOSE_FLAG_PAGES : 0;
}

__global__ __launch_bounds__(NT) void k_evict_select(const goose_pages pg, const Evictions ev, int n_layers, int n_kv, float* __restrict__ weight,
                                                     uint64_t* __restrict__ kept, int32_t* __restrict__ verdict) {
  __shared__ unsigned hist[2048];
  __shared__ int ws[NT / 64], found[2];
  const goose_eviction q = ev.r[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int layer = blockIdx.x / n_kv, head = blockIdx.x - layer * n_kv;
  const int len = __builtin_amdgcn_readfirstlane(pg.d_len[q.seq]);
  const int bad = verdict_of(pg, q, len, tid);
  if (blockIdx.x == 0 && tid == 0) verdict[blockIdx.y] = bad;
  if (bad) return;
  uint64_t* const words = kept + (((size_t)blockIdx.y * n_layers + layer) * n_kv + head) * pg.table_ld;
  float* const w = weight + (((size_t)layer * pg.n_seqs + q.seq) * n_kv + head) * pg.table_ld * GOOSE_PAGE;
  const int n_words = (len + GOOSE_PAGE - 1) / GOOSE_PAGE;
  for (int i = n_words + tid; i < pg.table_ld; i += NT) words[i] = 0;
  if (len <= q.keep) {
    for (int i = tid; i < n_words; i += NT) {
      const int m = min(GOOSE_PAGE, len - i * GOOSE_PAGE);
      words[i] = m == 64 ? ~0ull : (1ull << m) - 1;
    }
    return;
  }
  // ---- the m-th largest weight of slots lo .. hi - 1: its key, and how many slots of just that weight are kept
  const int lo = q.sink, hi = len - q.recent, m = q.keep - q.sink - q.recent;
  unsigned key = 0;
  int ties = 0, equal = 0;
  if (m > 0) {
    ties = m;
    int shift = 21;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int bins = pass < 2 ? 2048 : 1024;
      for (int i = tid; i < bins; i += NT) hist[i] = 0;
      __syncthreads();
      const unsigned above = pass == 0 ? 0u : key >> (pass == 1 ? 21 : 10);
      for (int s = lo + tid; s < hi; s += NT) {
        const unsigned x = key_of(w[s]);
        if (pass == 0 || x >> (pass == 1 ? 21 : 10) == above) atomicAdd(&hist[(x >> shift) & (bins - 1)], 1u);
      }
      __syncthreads();
      // thread t owns the bins 2 t, 2 t + 1 from the top: how many slots lie above them
      const int b0 = bins - 1 - 2 * tid;
      const int c0 = b0 >= 0 ? (int)hist[b0] : 0, c1 = b0 >= 1 ? (int)hist[b0 - 1] : 0;
      int x = c0 + c1;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int up = __shfl_up(x, off, 64);
        if (lane >= off) x += up;
      }
      if (lane == 63) ws[wave] = x;
      __syncthreads();
      int before = x - c0 - c1;
      for (int i = 0; i < wave; ++i) before += ws[i];
      if (before < ties && ties <= before + c0) { found[0] = b0; found[1] = before; }
      else if (before + c0 < ties && ties <= before + c0 + c1) { found[0] = b0 - 1; found[1] = before + c0; }
      __syncthreads();
      key |= (unsigned)found[0] << shift;
      ties -= found[1];
      equal = (int)hist[found[0]];
      shift = pass == 0 ? 10 : 0;
      __syncthreads();
    }
  }
  // ---- the words: a wavefront takes a run of them, one slot a lane.  Ties go to the lowest slots
  const int run = (n_words + NT / 64 - 1) / (NT / 64), w_lo = min(n_words, wave * run), w_hi = min(n_words, w_lo + run);
  int left = ties;
  if (m > 0 && ties < equal) {
    int mine = 0;
    for (int i = w_lo; i < w_hi; ++i) {
      const int s = i * GOOSE_PAGE + lane;
      mine += (int)__popcll(__builtin_amdgcn_ballot_w64(s >= lo && s < hi && key_of(w[s]) == key));
    }
    if (lane == 0) ws[wave] = mine;
    __syncthreads();
    for (int i = 0; i < wave; ++i) left -= ws[i];
  }
  for (int i = w_lo; i < w_hi; ++i) {
    const int s = i * GOOSE_PAGE + lane;
    const bool mid = m > 0 && s >= lo && s < hi;
    const unsigned x = mid ? key_of(w[s]) : 0;
    const uint64_t same = __builtin_amdgcn_ballot_w64(mid && x == key);
    const bool tie = mid && x == key && (int)__popcll(same & ((1ull << lane) - 1)) < left;  // (left may be negative, a count is unsigned)
    const uint64_t word = __builtin_amdgcn_ballot_w64(s < lo || (s >= hi && s < len) || (mid && x > key) || tie);
    left -= (int)__popcll(same);
    if (lane == 0) words[i] = word;
  }
  __syncthreads();
  // ---- weights to the front, 1024 slots at a time: none of them is behind where it goes
  int base = 0;
  for (int c0 = 0; c0 < len; c0 += NT) {
    const int i = (c0 >> 6) + wave, s = c0 + tid;
    const uint64_t word = i < n_words ? words[i] : 0;
    const bool mine = (word >> lane) & 1;
    const float x = mine ? w[s] : 0.f;
    if (lane == 0) ws[wave] = (int)__popcll(word);
    __syncthreads();
    int at = base + (int)__popcll(word & ((1ull << lane) - 1));
    for (int j = 0; j < NT / 64; ++j) {
      if (j < wave) at += ws[j];
      base += ws[j];
    }
    if (mine) w[at] = x;
    __syncthreads();
  }
}

__device__ __forceinline__ void in_order() {  // LDS of one wavefront: its instructions execute in order, the compiler is to keep them so
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

template <int D, bool F16>
__global__ __launch_bounds__(64) void k_evict_move(const goose_pages pg, const Evictions ev, int n_layers, int n_kv, const double* __restrict__ inv_freq,
                                                   const uint64_t* __restrict__ kept, bool reposition, const int32_t* __restrict__ verdict) {
  typedef typename Mma16<F16>::T T;
  typedef typename Mma16<F16>::v8 op8;
  constexpr int UNITS = D / 32, AHEAD = 4;
  __shared__ __attribute__((aligned(16))) unsigned short stage[2][2][64 * 8];  // [destination block % 2][piece][...]
  const goose_eviction q = ev.r[blockIdx.y];
  const int lane = threadIdx.x, l31 = lane & 31, hh = lane >> 5;
  const int len = __builtin_amdgcn_readfirstlane(pg.d_len[q.seq]);
  if (__builtin_amdgcn_readfirstlane(verdict[blockIdx.y]) != 0 || len <= q.keep || q.sink >= q.keep) return;
  const int lh = blockIdx.x / (2 * UNITS), unit = blockIdx.x - lh * (2 * UNITS);
  const int layer = lh / n_kv, head = lh - layer * n_kv;
  const bool keys = unit < UNITS;
  const int p0 = keys ? unit : 2 * (unit - UNITS), p1 = keys ? unit + UNITS : p0 + 1;  // its two pieces of a block's 1 KiB pieces
  T* const pool = static_cast<T*>(keys ? pg.d_kpool : pg.d_vpool) + (size_t)layer * pg.n_pages * n_kv * (GOOSE_PAGE * D);
  const int32_t* const row = pg.d_table + (size_t)q.seq * pg.table_ld;
  const uint64_t* const words = kept + (((size_t)blockIdx.y * n_layers + layer) * n_kv + head) * pg.table_ld;
  auto block_at = [&](int b) -> T* {
    const int page = __builtin_amdgcn_readfirstlane(row[b >> 1]);
    return pool + ((size_t)page * n_kv + head) * (GOOSE_PAGE * D) + (size_t)(b & 1) * 32 * D + lane * 8;
  };
  // a lane of the keys has eight columns of slot kk of a block; one of the values has 16 slots of a column
  const int kk = ((l31 >> 2) & 1) * 16 + (l31 >> 3) * 4 + (l31 & 3);
  double freq[8];
  if (keys && reposition) {
#pragma unroll
    for (int e = 0; e < 8; ++e) freq[e] = inv_freq[unit * 16 + hh * 8 + e];
  }
  const int b0 = q.sink >> 5, b_end = (len + 31) >> 5;
  int at = b0 * 32;  // rows placed so far (all slots in front of b0 stay)
  u32x4 r0[AHEAD], r1[AHEAD];
  auto mask_of = [&](int b) -> unsigned {
    return b < b_end ? (unsigned)__builtin_amdgcn_readfirstlane((int)(words[b >> 1] >> ((b & 1) * 32))) : 0u;
  };
  auto load = [&](int b, u32x4& x, u32x4& y) {
    if (mask_of(b) == 0) return;
    const T* p = block_at(b);
    x = *reinterpret_cast<const u32x4*>(p + p0 * 512);
    y = *reinterpret_cast<const u32x4*>(p + p1 * 512);
  };
  // whole destination block b, or its first n < 32 slots
  auto flush = [&](int b, int n) {
    in_order();
    T* const p = block_at(b);
    const u32x4 x = *reinterpret_cast<const u32x4*>(&stage[b & 1][0][lane * 8]), y = *reinterpret_cast<const u32x4*>(&stage[b & 1][1][lane * 8]);
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
    in_order();
  };
  auto place = [&](int b, u32x4 x, u32x4 y) {
    const unsigned mask = mask_of(b);
    if (mask == 0) return;
    if (keys) {
      const int to = at + __popc(mask & ((1u << kk) - 1)), d = to & 31;
      const int delta = to - (b * 32 + kk);
      if (reposition && delta != 0) {
        op8 lo = __builtin_bit_cast(op8, x), hi = __builtin_bit_cast(op8, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double two_pi = 6.283185307179586476925286766559;
          double ang = (double)delta * freq[e];
          ang -= two_pi * rint(ang / two_pi);
          float sn, c;
          sincosf((float)ang, &sn, &c);
          const float u = (float)lo[e], v = (float)hi[e];
          lo[e] = (T)(u * c - v * sn);
          hi[e] = (T)(v * c + u * sn);
        }
        x = __builtin_bit_cast(u32x4, lo);
        y = __builtin_bit_cast(u32x4, hi);
      }
      if ((mask >> kk) & 1) {
        const int l = (((d >> 2) & 3) << 3 | (d >> 4) << 2 | (d & 3)) + 32 * hh;
        *reinterpret_cast<u32x4*>(&stage[(to >> 5) & 1][0][l * 8]) = x;
        *reinterpret_cast<u32x4*>(&stage[(to >> 5) & 1][1][l * 8]) = y;
      }
    } else {
      const u16x8 a = __builtin_bit_cast(u16x8, x), c = __builtin_bit_cast(u16x8, y);
      int to = at + (hh ? __popc(mask & 0xFFFFu) : 0);
      const unsigned mine = hh ? mask >> 16 : mask & 0xFFFFu;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int d = to & 31;
        if ((mine >> e) & 1) {
          stage[(to >> 5) & 1][(d >> 3) & 1][(l31 + 32 * (d >> 4)) * 8 + (d & 7)] = e < 8 ? a[e & 7] : c[e & 7];
          ++to;
        }
      }
    }
    const int next = at + __popc(mask);
    if ((next >> 5) != (at >> 5)) flush(at >> 5, 32);
    at = next;
  };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) load(b0 + k, r0[k], r1[k]);
  for (int b = b0; b < b_end; b += AHEAD) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      place(b + k, r0[k], r1[k]);
      load(b + k + AHEAD, r0[k], r1[k]);
    }
  }
  if (at & 31) flush(at >> 5, at & 31);
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
  hipLaunchKernelGGL(k_evict_select, dim3(n_layers * n_kv, ev.n), dim3(NT), 0, st, pg, ev, n_layers, n_kv, weight, kept, scratch->verdict);
  int rc = goose_launch_status();
  if (rc != GOOSE_OK) return rc;
  const dim3 grid(n_layers * n_kv * (head_dim / 16), ev.n);
  const bool f16 = dtype == GOOSE_DTYPE_F16;
#define GOOSE_MOVE(D, H) hipLaunchKernelGGL((k_evict_move<D, H>), grid, dim3(64), 0, st, pg, ev, n_layers, n_kv, inv_freq, kept, reposition, scratch->verdict)
  if (head_dim == 128) { if (f16) GOOSE_MOVE(128, true); else GOOSE_MOVE(128, false); }
  else if (head_dim == 64) { if (f16) GOOSE_MOVE(64, true); else GOOSE_MOVE(64, false); }
  else return GOOSE_ERR_SHAPE;
#undef GOOSE_MOVE
  rc = goose_launch_status();
  if (rc != GOOSE_OK) return rc;
  hipLaunchKernelGGL(k_evict_settle, dim3(ev.n), dim3(256), 0, st, pg, ev, scratch->verdict, flags);
  return goose_launch_status();
}
