// What the attention kernels on a paged cache share: softmax bookkeeping, page ids, a tile of 32 rows and its two products.
// Device code only (included by .hip files).
#pragma once
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

// Four neighbouring columns (inside one group of eight) of an output row, in `terms` terms.
__device__ inline void store_columns(unsigned short* row, int terms, bool f16, int col, const f32x4& x) {
  u16x4 v, v2;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = out_bits16(x[e], f16);
    v2[e] = out_bits16(x[e] - out_back16(v[e], f16), f16);
  }
  unsigned short* dst = row + term_pos(terms, col);
  *reinterpret_cast<u16x4*>(dst) = v;
  if (terms == 2) *reinterpret_cast<u16x4*>(dst + 8) = v2;
}

// The maximum as the exponent's reference: a row that has seen nothing (or only scores of -infinity) takes 0, so that 2^(-inf - 0) = 0.
__device__ inline float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }
// Scores are unscaled; c = log2(e) / sqrt(d).  Weights are 2^(s c - ref), ref = m c rounded once.
__device__ __forceinline__ float reference_of(float m, float c) {
#pragma clang fp contract(off)
  return finite_ref(m) * c;
}
// From 2^24 on such products leave no room for the fraction: there (and for infinities) differences of scores are scaled instead.
__device__ __forceinline__ bool far_out(float ref) { return !(fabsf(ref) < 16777216.f); }
// What the sums of a set of keys with the maximum m0 are multiplied by where the maximum becomes m >= m0.
__device__ __forceinline__ float join_factor(float m0, float m, float c) {
#pragma clang fp contract(off)
  const float ref = reference_of(m, c);
  return m0 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(far_out(ref) ? (m0 - finite_ref(m)) * c : m0 * c - ref);
}

// The natural logarithm of a row's sum of exp(score): l = sum of 2^(s c - ref) is relative to the reference that the weights went by.
__device__ inline float log_of_sum(float m, float l, float c) {
  const float ref = reference_of(m, c);
  return l == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}
// Page ids of consecutive blocks, 64 of them a register (one a lane); an entry out of range reads page 0 and is flagged.
struct PageIds {
  const int32_t* row;
  int32_t* flags;
  int base, last, n_pages, ids;
  __device__ __forceinline__ void load(int lane) { take(lane, base + lane <= last ? row[base + lane] : 0); }
  __device__ __forceinline__ void take(int lane, int entry) {
    ids = base + lane <= last ? entry : 0;
    if ((unsigned)ids >= (unsigned)n_pages) { atomicOr(flags, GOOSE_FLAG_PAGES); ids = 0; }
  }
  // the id of block b's page; b never steps below the window, nor beyond page `last`
  __device__ __forceinline__ int of(int b, int lane) {
    if ((b >> 1) - base >= 64) { base = b >> 1; load(lane); }
    return __builtin_amdgcn_readlane(ids, (b >> 1) - base);
  }
};

// An empty statement that takes and gives x: it is computed here, neither earlier nor later.
#if defined(__HIP_DEVICE_COMPILE__)
#define GOOSE_HERE(x) asm volatile("" : "+v"(x))
#else
#define GOOSE_HERE(x) (void)(x)
#endif

// ---- 32 rows of the softmax; weights enter the second product in two terms --------------------------------------------------
template <int D, int QT, bool F16>
struct RowTile {
  static constexpr int NS = D / 16, NDT = D / 32;
  static constexpr float SLACK = 8.f;
  typedef typename Mma16<F16>::T T;
  typedef typename Mma16<F16>::v8 op8;
  op8 q[NS], ql[QT == 2 ? NS : 1];
  f32x16 o[NDT];
  f32x16 s;  // scores of the block at hand
  op8 p[2], pl[2];  // weights of the block at hand: leading and second terms
  float m, l, top;   // largest score so far, sum of weights, this block's largest score of this lane
  float lim, ref, mul;  // see raise()
  float late;           // see rescale_later()
  bool due;
  // query: of this lane's row and half
  __device__ __forceinline__ void init(const T* query) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[j][e] = (T)0.f;
        pl[j][e] = (T)0.f;
      }
    m = lim = -INFINITY;
    l = ref = 0.f;
    mul = late = 1.f;
    due = false;
    load_q(query);
  }
  __device__ __forceinline__ void load_q(const T* at) {
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      q[k] = *reinterpret_cast<const op8*>(at + k * 16 * QT);
      if (QT == 2) ql[k] = *reinterpret_cast<const op8*>(at + k * 32 + 8);
    }
  }
  // PAIRED, here and in values(): the two terms of a piece one after the other, as ring_step adds them up.
  template <bool PAIRED = false>
  __device__ __forceinline__ void scores(const u32x4 (&k)[NS]) {
    f32x16 sum;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[r] = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      sum = Mma16<F16>::mfma(__builtin_bit_cast(op8, k[i]), q[i], sum);
      if (PAIRED && QT == 2) sum = Mma16<F16>::mfma(__builtin_bit_cast(op8, k[i]), ql[i % (QT == 2 ? NS : 1)], sum);
    }
    if (!PAIRED && QT == 2) {
#pragma unroll
      for (int i = 0; i < NS; ++i) sum = Mma16<F16>::mfma(__builtin_bit_cast(op8, k[i]), ql[i], sum);
    }
    s = sum;
  }
  __device__ __forceinline__ void mask(unsigned vis) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = ((vis >> r) & 1u) ? s[r] : -INFINITY;
  }
  // This lane's largest score (unscaled, as m is: the scale is positive), from partial ones: a NaN stays one, and compares as no larger.
  static __device__ __forceinline__ float partial_max(const f32x16& x, int r) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x[r], x[r + 4]), __builtin_elementwise_maximum(x[r + 8], x[r + 12]));
  }
  static __device__ __forceinline__ float join_max(const float (&t)[4]) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(t[0], t[1]), __builtin_elementwise_maximum(t[2], t[3]));
  }
  __device__ __forceinline__ void maximum() {
    const float t[4] = {partial_max(s, 0), partial_max(s, 1), partial_max(s, 2), partial_max(s, 3)};
    top = join_max(t);
  }
  __device__ __forceinline__ bool grown() const { return __builtin_amdgcn_ballot_w64(top > lim) != 0; }
  // m, and with it l and O, follows only where a row's largest score has grown so far that weights would pass 2^SLACK: weights up to there are as
  // good as those up to one in two terms, of which 16 bits hold both with room to spare (a weight other than one is rounded for the second product and not in
  // l: one term would leave a row that a single key dominates off by its whole rounding), and with 32 rows in a tile some row's maximum grows by a
  // little in most blocks (512 rows over 16384 slots: in 3 of 4).
  // A weight is 2^(s c - ref) in one fused multiply-add; the rounding of ref is the same factor in O and l.  Far out
  // the block's scores (x) become differences to m first.
  // Returns the factor that O has to follow by.
  __device__ __forceinline__ float raise(float c, f32x16& x) {
    const float both = fmaxf(top, __shfl_xor(top, 32, 64)), m_new = both > lim ? fmaxf(m, both) : m;
    const float now = finite_ref(m_new), alpha = join_factor(m, m_new, c);
    m = m_new;
    ref = reference_of(m, c);
    const bool far = far_out(ref);
    lim = m + SLACK / c;
    mul = c;
    if (__builtin_amdgcn_ballot_w64(far) != 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = far ? (x[r] - now) * c : fmaf(x[r], c, -ref);
      mul = 1.f;
      ref = 0.f;
      lim = -INFINITY;  // (and so will the next block's)
    }
    l *= alpha;
    return alpha;
  }
  __device__ __forceinline__ void scale_out(float alpha) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
  }
  __device__ __forceinline__ void rescale(float c) {
    if (__builtin_expect(grown(), 0)) scale_out(raise(c, s));
  }
  // The same where O still lacks an earlier block, whose weights go by the reference before: its factor waits until that block is in.
  __device__ __forceinline__ void rescale_later(float c, f32x16& x, bool more) {
    const bool grows = more && grown();
    if (__builtin_expect(grows || due, 0)) {
      if (due) scale_out(late);
      due = grows;
      if (grows) late = raise(c, x);
    }
  }
  // x, y in two 16-bit terms, as weights of keys 2 i, 2 i + 1
  static __device__ __forceinline__ void pair_to(int i, float x, float y, op8 (&w)[2], op8 (&wl)[2]) {
    typedef T T2 __attribute__((ext_vector_type(2)));
    typedef float F2 __attribute__((ext_vector_type(2)));
    unsigned h = __builtin_bit_cast(unsigned, __builtin_convertvector((F2{x, y}), T2));
    GOOSE_HERE(h);  // (the compiler would move it to the next step, which uses it, with no matrix instruction beside it)
    u32x4 v = __builtin_bit_cast(u32x4, w[i >> 2]);
    v[i & 3] = h;
    w[i >> 2] = __builtin_bit_cast(op8, v);
    F2 rest;
    if constexpr (F16) {
      const T2 t = __builtin_bit_cast(T2, h);
      rest = F2{x - (float)t[0], y - (float)t[1]};
    } else {
      rest = F2{x - __builtin_bit_cast(float, h << 16), y - __builtin_bit_cast(float, h & 0xFFFF0000u)};
    }
    v = __builtin_bit_cast(u32x4, wl[i >> 2]);
    unsigned low = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, T2));
    GOOSE_HERE(low);
    v[i & 3] = low;
    wl[i >> 2] = __builtin_bit_cast(op8, v);
  }
  // weights of keys 2 i, 2 i + 1 of the scores in z (a masked score is -infinity: zero)
  __device__ __forceinline__ void weights_of(int i, const f32x16& z, op8 (&w)[2], op8 (&wl)[2]) {
    const float x = __builtin_amdgcn_exp2f(fmaf(z[2 * i], mul, -ref)), y = __builtin_amdgcn_exp2f(fmaf(z[2 * i + 1], mul, -ref));
    l += x;
    l += y;
    pair_to(i, x, y, w, wl);
  }
  __device__ __forceinline__ void weights() {
#pragma unroll
    for (int i = 0; i < 8; ++i) weights_of(i, s, p, pl);
  }
  template <bool PAIRED = false>
  __device__ __forceinline__ void values(const u32x4 (&v)[NS]) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        o[dt] = Mma16<F16>::mfma(__builtin_bit_cast(op8, v[dt * 2 + j]), p[j], o[dt]);
        if constexpr (PAIRED) o[dt] = Mma16<F16>::mfma(__builtin_bit_cast(op8, v[dt * 2 + j]), pl[j], o[dt]);
      }
    if constexpr (PAIRED) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) o[dt] = Mma16<F16>::mfma(__builtin_bit_cast(op8, v[dt * 2 + j]), pl[j], o[dt]);
  }
  // The second product of a block with a NaN or an infinity in a value that some rows do not see (through the matrix instruction it
  // would reach them as 0 * NaN): those elements count as zero there, and a product of indicators (is it +inf, -inf, NaN) x (is it visible) tells
  // which outputs they reach.  Rare.
  template <bool PAIRED = false>
  __device__ __forceinline__ void values_odd(const u32x4 (&v)[NS], unsigned vis) {
    constexpr unsigned short EXP = F16 ? 0x7C00 : 0x7F80;
    const unsigned short ONE = __builtin_bit_cast(unsigned short, (T)1.f);
    u16x8 seen[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) seen[r >> 3][r & 7] = ((vis >> r) & 1u) ? ONE : (unsigned short)0;
#pragma unroll 1
    for (int c = 0; c < 3; ++c) {
      const float special = c == 0 ? INFINITY : (c == 1 ? -INFINITY : __builtin_nanf(""));
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        f32x16 hits;
#pragma unroll
        for (int r = 0; r < 16; ++r) hits[r] = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          u32x4 raw = v[dt * 2 + j];
          asm volatile("" : "+v"(raw));  // (nothing of this may move out of the loop: it would take the registers of the common path)
          u16x8 e = __builtin_bit_cast(u16x8, raw);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int is = (e[i] & EXP) != EXP ? -1 : (e[i] == EXP ? 0 : (e[i] == (EXP | 0x8000) ? 1 : 2));
            e[i] = is == c ? ONE : (unsigned short)0;
          }
          hits = Mma16<F16>::mfma(__builtin_bit_cast(op8, e), __builtin_bit_cast(op8, seen[j]), hits);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = hits[r] > 0.f ? o[dt][r] + special : o[dt][r];
      }
    }
    u32x4 w[NS];
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      u16x8 e = __builtin_bit_cast(u16x8, v[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = (e[i] & EXP) == EXP ? (unsigned short)0 : e[i];
      w[k] = __builtin_bit_cast(u32x4, e);
    }
    values<PAIRED>(w);
  }
};

// Slots behind the tree may hold anything: their values (of this lane's 16 keys those from `mine` on) become zero.  True if a NaN or an
// infinity is left.
template <bool F16, int NS>
__device__ __forceinline__ bool clean_values(u32x4 (&v)[NS], int mine) {
  constexpr unsigned EXP = F16 ? 0x7C00u : 0x7F80u;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // keys 2 i, 2 i + 1: dword i % 4 of the pieces with parity i / 4
    const unsigned keep = 2 * i + 1 < mine ? 0xFFFFFFFFu : (2 * i < mine ? 0xFFFFu : 0u);
#pragma unroll
    for (int k = i >> 2; k < NS; k += 2) {
      const unsigned x = v[k][i & 3] & keep;
      v[k][i & 3] = x;
      odd = odd || (x & EXP) == EXP || (x & (EXP << 16)) == (EXP << 16);
    }
  }
  return __builtin_amdgcn_ballot_w64(odd) != 0;
}
template <int NS>
__device__ __forceinline__ void fetch(const void* at, int lane, u32x4 (&dst)[NS]) {
  const u32x4* p = static_cast<const u32x4*>(at) + lane;
#pragma unroll
  for (int s = 0; s < NS; ++s) dst[s] = p[s * 64];
}
__device__ inline float softmax_scale(int D) { return 1.4426950408889634f / sqrtf((float)D); }  // log2(e) / sqrt(d): softmax in base 2

#define GOOSE_BUFFER_WORD3 0x00020000  // (buffer descriptor: raw 32-bit data)
#define GOOSE_LDS_PTR(p) ((__attribute__((address_space(3))) void*)(p))
constexpr int vmcnt_imm(int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); }  // s_waitcnt vmcnt(n) only

// CP pieces of 1 KiB from src (uniform) to LDS.  Through a buffer descriptor: LDS reads behind a global_load to LDS wait for all reads
// in flight instead of the ones that they need.
template <int CP>
__device__ __forceinline__ void copy_pieces(const char* src, int lane, unsigned char* cp) {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host pass knows no such builtin and would silently drop the kernel's stub)
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(src), 0, CP * 1024, GOOSE_BUFFER_WORD3);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, GOOSE_LDS_PTR(cp), 16, lane * 16, 0, 0, 0);
  if (CP > 1) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, GOOSE_LDS_PTR(cp), 16, lane * 16, 0, 1024, 0);  // (the offset counts on both sides)
  if (CP > 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, GOOSE_LDS_PTR(cp), 16, lane * 16, 0, 2048, 0);
  if (CP > 3) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, GOOSE_LDS_PTR(cp), 16, lane * 16, 0, 3072, 0);
#endif
}
// Step j of a wavefront: scores of block j + 1 (to z1), weights of block j (from z0 to w0), outputs of block j - 1 (its weights in w).  None of the three
// needs another, so the vector work is dealt out evenly beside the matrix instructions, and the last quarter of them hides the maximum of z1.
// The operand pieces come from the ring AHEAD uses before they are needed; with
// one key group pc holds the first ones and is left with those of the next step.  k1, k2: keys of blocks j + 1 and j + 2, v0: values of block j - 1.
// The order is written down: the compiler's own collects the vector work where it waits for the scores.
// edge(s): what becomes of the scores of block j + 1 before their maximum is taken.
template <int D, int QT, bool F16, int G, int AHEAD, typename Edge>
__device__ __forceinline__ void ring_step(RowTile<D, QT, F16>& t, u32x4 (&pc)[AHEAD], const u32x4* __restrict__ k1, const u32x4* __restrict__ v0,
                                          const u32x4* __restrict__ k2, const f32x16& z0, f32x16& z1,
                                          const typename RowTile<D, QT, F16>::op8 (&w)[2], const typename RowTile<D, QT, F16>::op8 (&wl)[2],
                                          typename RowTile<D, QT, F16>::op8 (&w0)[2], typename RowTile<D, QT, F16>::op8 (&wl0)[2],
                                          bool more, float scale, Edge edge) {
  typedef RowTile<D, QT, F16> Tile;
  typedef typename Tile::op8 op8;
  constexpr int NS = Tile::NS, NDT = Tile::NDT, ALL = NS * (QT + 2), SPREAD = ALL * 3 / 4;
  u32x4 piece[2 * NS + AHEAD];
#pragma unroll
  for (int n = 0; n < AHEAD; ++n) piece[n] = G == 1 ? pc[n] : k1[n * 64];
  f32x16 sum;
#pragma unroll
  for (int r = 0; r < 16; ++r) sum[r] = 0.f;
  float part[4];
#pragma unroll
  for (int n = 0; n < 2 * NS; ++n) {
    {
      const int m = n + AHEAD, x = m - NS;
      if (m < NS) piece[m] = k1[m * 64];
      else if (m < 2 * NS) piece[m] = v0[(x % NDT * 2 + x / NDT) * 64];
      else if (G == 1) piece[m] = k2[(m - 2 * NS) * 64];
    }
    const op8 a = __builtin_bit_cast(op8, piece[n]);
    if (n < NS) {
      sum = Mma16<F16>::mfma(a, t.q[n], sum);
      if (QT == 2) sum = Mma16<F16>::mfma(a, t.ql[n % (QT == 2 ? NS : 1)], sum);
      GOOSE_HERE(sum);
    } else {
      const int x = n - NS, j = x / NDT, dt = x % NDT;
      t.o[dt] = Mma16<F16>::mfma(a, w[j], t.o[dt]);
      t.o[dt] = Mma16<F16>::mfma(a, wl[j], t.o[dt]);
      GOOSE_HERE(t.o[dt]);
    }
    const int before = n < NS ? n * QT : NS * QT + (n - NS) * 2, behind = before + (n < NS ? QT : 2);  // matrix instructions so far
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= 8 * before / SPREAD && i < 8 * behind / SPREAD) t.weights_of(i, z0, w0, wl0);
    GOOSE_HERE(t.l);
    if (n == 2 * NS - NS / 2 - 1) edge(sum);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (2 * NS - NS / 2 + r * NS / 8 == n) {
        part[r] = Tile::partial_max(sum, r);
        GOOSE_HERE(part[r]);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
  z1 = sum;
  t.top = Tile::join_max(part);
  t.rescale_later(scale, z1, more);  // (behind the last block the scores are of a block that is not this loop's)
#pragma unroll
  for (int n = 0; n < AHEAD; ++n)
    if (G == 1) pc[n] = piece[2 * NS + n];
}

}  // namespace
