// Book-keeping of a paged KV cache: fork, reserve (with copy on write), commit of an accepted path, free.
//
// State: table[seq][i] names the page of slots 64 i .. 64 i + 63, refs[page] counts the entries that name it, len[seq] the
// committed slots; a page is free when its count is 0, and there is no other list of free pages that could disagree with the
// counts.  Everything is decided on the device from that state, so the calls can be recorded into a graph whose replays allocate
// and release different pages.  The tables are a few KiB: those kernels are chains of dependent loads (length -> entry -> count ->
// stores) in one workgroup, about 1 us a link (fork 3 us, reserve 6, free and settle 2 to 4); only copies and moves touch data, at one workgroup
// per (layer, K or V, head).
#include "goose_internal.h"
#include "paged.h"

namespace {

constexpr int NT = 1024;  // threads of the one-workgroup kernels

__global__ __launch_bounds__(256) void k_pages_clear(const goose_pages pg) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (size_t)pg.n_seqs * pg.table_ld) pg.d_table[i] = -1;
  if (i < (size_t)pg.n_seqs) pg.d_len[i] = 0;
  if (i < (size_t)pg.n_pages) pg.d_refs[i] = 0;
}

__global__ __launch_bounds__(NT) void k_pages_fork(const goose_pages pg, int src, int len, const SeqList dst, int32_t* __restrict__ flags) {
  __shared__ int ok[GOOSE_MAX_REQUESTS];
  const int tid = threadIdx.x;
  const int have = pg.d_len[src];
  const int n = len < 0 ? have : len, np = (n + GOOSE_PAGE - 1) / GOOSE_PAGE;
  if (n > have || n < 0 || np > pg.table_ld) {
    if (tid == 0) atomicOr(flags, GOOSE_FLAG_CAPACITY);
    return;
  }
  if (tid < dst.n) {  // an empty sequence has no first page and no length
    const int q = dst.seq[tid];
    const bool empty = pg.d_len[q] == 0 && pg.d_table[(size_t)q * pg.table_ld] == -1;
    ok[tid] = empty;
    if (!empty) atomicOr(flags, GOOSE_FLAG_PAGES);
  }
  // a hole in the source, or a page of it that counts as free: nothing is shared
  bool hole = false;
  for (int i = tid; i < np; i += NT) {
    const int e = pg.d_table[(size_t)src * pg.table_ld + i];
    hole = hole || (unsigned)e >= (unsigned)pg.n_pages || pg.d_refs[e] < 1;
  }
  if (__syncthreads_or(hole)) {
    if (tid == 0) atomicOr(flags, GOOSE_FLAG_PAGES);
    return;
  }
  int forks = 0;
  for (int r = 0; r < dst.n; ++r) forks += ok[r];
  for (int i = tid; i < np; i += NT) {
    const int e = pg.d_table[(size_t)src * pg.table_ld + i];
    for (int r = 0; r < dst.n; ++r)
      if (ok[r]) pg.d_table[(size_t)dst.seq[r] * pg.table_ld + i] = e;
    atomicAdd(&pg.d_refs[e], forks);  // (integers: the order does not matter)
  }
  if (tid < dst.n && ok[tid]) pg.d_len[dst.seq[tid]] = n;
}

// Exclusive prefix sum of v over the workgroup; *total = sum.  ws: NT / 64 words of LDS.
__device__ inline int block_scan(int v, int* ws, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  __syncthreads();  // (ws may still be read from the call before)
  if (lane == 63) ws[wave] = x;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const int s = ws[w];
    before += w < wave ? s : 0;
    sum += s;
  }
  *total = sum;
  return before + x - v;
}

// Items = (request, page that its new slots touch), requests in order, pages ascending.  An item takes a page where its entry is
// missing, or where it is the first one and shared.  Of several requests of the call that share a page, the last may keep it: the
// i-th of them leaves while refs - i > 1.  The k-th item that takes a page gets the k-th free page.
//
// Of a step (sq.step) the reservation is what decides whether it is done: it also fails where a length is above the request's P_max or below the
// shared pages, where a table names a page out of range in front of its length, or where the shared entries differ.  The kernels behind it would only raise a
// flag for these and leave rows unwritten, or read other keys, and the commit would then keep them.
__global__ __launch_bounds__(NT) void k_pages_reserve(const goose_pages pg, const SeqList sq, int4* __restrict__ copies,
                                                      int32_t* __restrict__ flags) {
  __shared__ int first[GOOSE_MAX_REQUESTS], count[GOOSE_MAX_REQUESTS], entry0[GOOSE_MAX_REQUESTS], leave[GOOSE_MAX_REQUESTS];
  __shared__ int used[GOOSE_MAX_REQUESTS], ws[NT / 64], list[PAGES_PER_CALL], bad;
  const int tid = threadIdx.x;
  int refs0 = 0, f[4];  // counts of this thread's first four pages: asked for beside the lengths
#pragma unroll
  for (int k = 0; k < 4; ++k) f[k] = tid * 4 + k < pg.n_pages ? pg.d_refs[tid * 4 + k] : 1;
  if (tid == 0) bad = 0;
  __syncthreads();
  if (tid < sq.n) {
    const int q = sq.seq[tid], len = pg.d_len[q];
    const int lo = len >> 6;
    const long long end = (long long)len + sq.extra[tid];
    copies[tid] = make_int4(-1, -1, 0, 0);
    int e = -1, cnt = 0;
    if (len < 0 || end > (long long)pg.table_ld * GOOSE_PAGE || (sq.step && (len > sq.most[tid] || len < sq.shared_pages * GOOSE_PAGE))) {
      atomicOr(&bad, GOOSE_FLAG_CAPACITY);
    } else {
      cnt = (int)((end - 1) >> 6) - lo + 1;
      e = pg.d_table[(size_t)q * pg.table_ld + lo];
      if (e < -1 || e >= pg.n_pages) { atomicOr(&bad, GOOSE_FLAG_PAGES); e = -1; }
      else if (e >= 0) refs0 = pg.d_refs[e];
      if (e == -1 && (len & 63) != 0) atomicOr(&bad, GOOSE_FLAG_PAGES);  // committed slots without a page
    }
    first[tid] = cnt > 0 ? lo : 0;
    count[tid] = cnt;
    entry0[tid] = e;
    used[tid] = ((len & 63) + 31) >> 5;  // 32-slot blocks of that page with committed slots
  }
  __syncthreads();
  if (sq.step) {  // a wavefront a request: the entries of its whole committed pages
    static_assert(NT / 64 >= GOOSE_MAX_REQUESTS, "a wavefront for every request");
    const int r = tid >> 6;
    const int32_t* row = pg.d_table + (size_t)sq.seq[r < sq.n ? r : 0] * pg.table_ld;
    const int32_t* row0 = pg.d_table + (size_t)sq.seq[0] * pg.table_ld;
    bool wrong = false;
    const int n = r < sq.n ? first[r] : 0;
    for (int i = tid & 63; i < n; i += 64) {
      const int e = row[i];
      wrong = wrong || (unsigned)e >= (unsigned)pg.n_pages || (i < sq.shared_pages && e != row0[i]);
    }
    if (wrong) atomicOr(&bad, GOOSE_FLAG_PAGES);
  }
  if (tid < sq.n) {
    int before = 0;
    for (int r = 0; r < tid; ++r) before += entry0[r] == entry0[tid];
    leave[tid] = entry0[tid] >= 0 && refs0 - before > 1;
    if (entry0[tid] >= 0 && refs0 < 1) atomicOr(&bad, GOOSE_FLAG_PAGES);
  }
  __syncthreads();
  int items = 0;
  for (int r = 0; r < sq.n; ++r) items += count[r];
  // one item: its request and table entry; does it take a page?
  auto item = [&](int k, int* r_out, size_t* at) {
    int r = 0;
    while (k >= count[r]) k -= count[r++];
    *r_out = r;
    *at = (size_t)sq.seq[r] * pg.table_ld + first[r] + k;
    if (k == 0) return entry0[r] < 0 || leave[r];
    const int e = pg.d_table[*at];
    if (e == -1) return true;
    if ((unsigned)e >= (unsigned)pg.n_pages || pg.d_refs[e] != 1) atomicOr(&bad, GOOSE_FLAG_PAGES);
    return false;
  };
  int need = 0;
  bool mine = false;
  int r0 = 0;
  size_t at0 = 0;
  for (int base = 0; base < items; base += NT) {
    int r, sum;
    size_t at;
    const bool takes = base + tid < items && item(base + tid, &r, &at);
    (void)block_scan(takes, ws, &sum);
    need += sum;
    if (base == 0) { mine = takes; r0 = r; at0 = at; }
  }
  // the lowest `need` free pages, ascending
  int found = 0;
  for (int base = 0; base < pg.n_pages && found < need; base += 4 * NT) {
    const int p0 = base + tid * 4;
    int c = 0, sum;
    if (base > 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = p0 + k < pg.n_pages ? pg.d_refs[p0 + k] : 1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) c += f[k] == 0;
    int at = found + block_scan(c, ws, &sum);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (f[k] == 0) {
        if (at < need && at < PAGES_PER_CALL) list[at] = p0 + k;
        ++at;
      }
    found += sum;
  }
  __syncthreads();
  if (tid == 0 && (found < need || need > PAGES_PER_CALL)) bad |= GOOSE_FLAG_PAGES;
  __syncthreads();
  if (bad) {
    if (tid == 0) {
      atomicOr(flags, bad);
      copies[0].w = 1;  // (the reservation has failed)
    }
    return;
  }
  int done = 0;
  for (int base = 0; base < items; base += NT) {
    int r = r0, sum;
    size_t at = at0;
    const bool takes = base == 0 ? mine : (base + tid < items && item(base + tid, &r, &at));
    const int k = done + block_scan(takes, ws, &sum);
    done += sum;
    if (takes) {
      const int page = list[k];
      pg.d_table[at] = page;
      pg.d_refs[page] = 1;
      const bool is_first = at == (size_t)sq.seq[r] * pg.table_ld + first[r];
      if (is_first && leave[r]) {
        atomicSub(&pg.d_refs[entry0[r]], 1);
        copies[r] = make_int4(entry0[r], page, used[r], 0);
      }
    }
  }
}

// Copies of a reservation: workgroup (2 (layer * n_kv + head) + (K or V), request) moves the 32-slot blocks that hold committed
// slots, contiguous in the operand order: 1 or 2 x 64 d bytes.  Non-temporal stores: pages that stay dirty in the L2s are written back at the
// kernel's end, with nothing beside it (16 requests, 8 layers of 8 heads, 33.5 MB each way: 21 us, now 8.8; loads non-temporal too: 13; half the
// bytes a workgroup: level).
__global__ __launch_bounds__(256) void k_pages_copy(const goose_pages pg, const int4* __restrict__ copies, int n_kv, int D) {
  const int4 c = copies[blockIdx.y];
  if (c.x < 0) return;
  const int lh = blockIdx.x >> 1, layer = lh / n_kv, head = lh - layer * n_kv;
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  u32x4* pool = reinterpret_cast<u32x4*>((blockIdx.x & 1) ? pg.d_vpool : pg.d_kpool);
  const size_t per_head = (size_t)GOOSE_PAGE * D / 8;  // 16-byte units
  const u32x4* src = pool + (((size_t)layer * pg.n_pages + c.x) * n_kv + head) * per_head;
  u32x4* dst = pool + (((size_t)layer * pg.n_pages + c.y) * n_kv + head) * per_head;
  const int units = c.z * 32 * D / 8;
  u32x4 v[4];  // (at most 64 * 128 / 8 = 1024 units: four a thread, all loads in flight together)
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if ((int)threadIdx.x + k * 256 < units) v[k] = src[threadIdx.x + k * 256];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if ((int)threadIdx.x + k * 256 < units) __builtin_nontemporal_store(v[k], dst + threadIdx.x + k * 256);
}

// The accepted path, slot P + path[j] -> P + j for j = 1 .. L, in one (layer, head) of a request.  Thread c owns chunk c of the key rows
// (16 bytes) and column c of the value rows (2 bytes).  MOVES moves at a time, all loads before all stores: path[j] >= j and increasing, so
// no later source lies at or below an earlier destination.  The whole path is fetched at once, an entry a lane, with length, count and page ids
// beside it, and the moves are checked by a lane each: asked for move by move it was a trip to memory each (16 requests, 8 layers of 8
// heads: 24 us), checked one behind the other 11 us; now 9.6 in passes among others (13.8 in a kernel trace), of which the trips (length, entry, loads,
// stores) are the most.
//
// A commit is done as a whole or not at all: L must leave the sequence inside its tree and table, and every page from slot P to the last slot that is read or
// committed must be there and be the sequence's own (one that other tables name too may hold their committed rows in these slots).  Every workgroup
// comes to the same verdict, as this launch changes no table, length or count; k_pages_settle does, and goes by verdict[request] (the flags to raise, 0: done).
// The counts are asked for beside the first round's rows, and nothing is stored before they are there.
constexpr int MOVES = 16;  // (accepted paths are rarely longer)
template <int D>
__global__ __launch_bounds__(D) void k_pages_move(const goose_pages pg, const PagedReqs rq, int n_kv, const int4* __restrict__ reservation,
                                                  int32_t* __restrict__ verdict) {
  typedef unsigned short u16;
  const PagedReq& q = rq.r[blockIdx.y];
  const int layer = blockIdx.x / n_kv, head = blockIdx.x - layer * n_kv, c = threadIdx.x, lane = c & 63;
  const int32_t* path = static_cast<const int32_t*>(q.p);
  const int p_lo = lane < q.B ? path[lane] : -1, p_hi = lane + 64 < q.B ? path[lane + 64] : -1;
  const int P = __builtin_amdgcn_readfirstlane(pg.d_len[q.seq]), L = __builtin_amdgcn_readfirstlane(*q.accept_len);
  if (reservation && reservation->w) return;
  int bad = 0;
  if (P < 0 || L < 0 || L >= q.B || (long long)P + L + 1 > (long long)pg.table_ld * GOOSE_PAGE) bad = GOOSE_FLAG_CAPACITY;
  // lane u: is path[u], path[u + 64] a move (increasing from 0 at the root on, inside the tree)?  The path is followed up to the first that is none.
  const int up_lo = __shfl_up(p_lo, 1, 64), up_hi = __shfl_up(p_hi, 1, 64), end_lo = __shfl(p_lo, 63, 64);
  const bool go_lo = lane == 0 || (lane <= L && p_lo > (lane == 1 ? 0 : up_lo) && p_lo < q.B);
  const bool go_hi = lane + 64 <= L && p_hi > (lane == 0 ? end_lo : up_hi) && p_hi < q.B;
  const uint64_t stop_lo = ~__builtin_amdgcn_ballot_w64(go_lo), stop_hi = ~__builtin_amdgcn_ballot_w64(go_hi);
  const int moves = (stop_lo ? __builtin_ctzll(stop_lo) : 64 + (stop_hi ? __builtin_ctzll(stop_hi) : 64)) - 1;
  const int last = moves < 64 ? __builtin_amdgcn_readlane(p_lo, moves) : __builtin_amdgcn_readlane(p_hi, moves - 64);
  const int reach = moves > 0 ? max(L, last) : L;  // slots P .. P + reach are read or committed: in three pages at most
  const int e0 = P >> 6;
  const bool needed = !bad && lane < 3 && e0 + lane <= (int)((unsigned)(P + reach) >> 6);
  const int id = needed && e0 + lane < pg.table_ld ? pg.d_table[(size_t)q.seq * pg.table_ld + e0 + lane] : -1;
  if (__builtin_amdgcn_ballot_w64(needed && (unsigned)id >= (unsigned)pg.n_pages) != 0) bad = GOOSE_FLAG_PAGES;
  const int count = needed && !bad ? pg.d_refs[id] : 1;
  const size_t layer0 = (size_t)layer * pg.n_pages;
  u16* const kpool = static_cast<u16*>(pg.d_kpool);
  u16* const vpool = static_cast<u16*>(pg.d_vpool);
  const size_t per_page = (size_t)n_kv * (GOOSE_PAGE * D);
  const size_t base = layer0 * per_page + (size_t)head * (GOOSE_PAGE * D);
  for (int j0 = 1; !bad && j0 <= moves; j0 += MOVES) {
    // Lane u: move j0 + u, from slot P + from to slot P + j0 + u, each with its page.
    const int j = j0 + lane, n = min(MOVES, moves - j0 + 1);
    const int lo = __shfl(p_lo, j & 63, 64), hi = __shfl(p_hi, j & 63, 64), from = j < 64 ? lo : hi;
    const int src = P + from, dst = P + j;
    const int ps = __shfl(id, ((src >> 6) - e0) & 63, 64), pd = __shfl(id, ((dst >> 6) - e0) & 63, 64);
    auto part_of = [&](int page, int u) { return base + (size_t)__builtin_amdgcn_readlane(page, u) * per_page; };
    uint4 kr[MOVES];
    u16 vr[MOVES];
#pragma unroll
    for (int u = 0; u < MOVES; ++u)
      if (u < n) {
        const int s = __builtin_amdgcn_readlane(src, u);
        const size_t b = part_of(ps, u);
        if (c < D / 8) kr[u] = *reinterpret_cast<const uint4*>(kpool + b + page_k_chunk<D>(s & 63, c));
        vr[u] = vpool[b + page_v_elem<D>(s & 63, c)];
      }
    if (__builtin_amdgcn_ballot_w64(count != 1) != 0) break;
#pragma unroll
    for (int u = 0; u < MOVES; ++u)
      if (u < n) {
        const int d = P + j0 + u;
        const size_t b = part_of(pd, u);
        if (c < D / 8) *reinterpret_cast<uint4*>(kpool + b + page_k_chunk<D>(d & 63, c)) = kr[u];
        vpool[b + page_v_elem<D>(d & 63, c)] = vr[u];
      }
  }
  if (__builtin_amdgcn_ballot_w64(count != 1) != 0) bad = GOOSE_FLAG_PAGES;
  if (blockIdx.x == 0 && c == 0) verdict[blockIdx.y] = bad;
}

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

// New lengths, and the pages behind them go back; a request whose verdict (k_pages_move) is not 0 stays as it is.
// reservation: where the slots were taken in the same call, and nothing is committed if that failed.
__global__ __launch_bounds__(256) void k_pages_settle(const goose_pages pg, const PagedReqs rq, const int4* __restrict__ reservation,
                                                      const int32_t* __restrict__ verdict, int32_t* __restrict__ flags) {
  if (reservation && reservation->w) return;
  const PagedReq& q = rq.r[blockIdx.x];
  const int bad = verdict[blockIdx.x], len = pg.d_len[q.seq] + *q.accept_len + 1;
  __syncthreads();  // every thread has the old length
  if (bad) {
    if (threadIdx.x == 0) atomicOr(flags, bad);
    return;
  }
  const size_t row = (size_t)q.seq * pg.table_ld;
  for (int i = (len + GOOSE_PAGE - 1) / GOOSE_PAGE + threadIdx.x; i < pg.table_ld; i += 256) release(pg, row + i, flags);
  if (threadIdx.x == 0) pg.d_len[q.seq] = len;
}

__global__ __launch_bounds__(256) void k_pages_free(const goose_pages pg, const SeqList sq, int32_t* __restrict__ flags) {
  const int q = sq.seq[blockIdx.x];
  for (int i = threadIdx.x; i < pg.table_ld; i += 256) release(pg, (size_t)q * pg.table_ld + i, flags);
  if (threadIdx.x == 0) pg.d_len[q] = 0;
}

}  // namespace

int launch_pages_clear(const goose_pages& pg, hipStream_t st) {
  size_t n = (size_t)pg.n_seqs * pg.table_ld;
  if ((size_t)pg.n_pages > n) n = pg.n_pages;
  hipLaunchKernelGGL(k_pages_clear, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, pg);
  return goose_launch_status();
}

int launch_pages_fork(const goose_pages& pg, int src, int len, const SeqList& dst, int32_t* flags, hipStream_t st) {
  hipLaunchKernelGGL(k_pages_fork, dim3(1), dim3(NT), 0, st, pg, src, len, dst, flags);
  return goose_launch_status();
}

int launch_pages_reserve(const goose_pages& pg, const SeqList& seqs, int n_layers, int n_kv, int head_dim, PageScratch* scratch, int32_t* flags,
                         hipStream_t st) {
  hipLaunchKernelGGL(k_pages_reserve, dim3(1), dim3(NT), 0, st, pg, seqs, scratch->copies, flags);
  int rc = goose_launch_status();
  if (rc != GOOSE_OK) return rc;
  hipLaunchKernelGGL(k_pages_copy, dim3(2 * n_layers * n_kv, seqs.n), dim3(256), 0, st, pg, (const int4*)scratch->copies, n_kv, head_dim);
  return goose_launch_status();
}

int launch_pages_commit(const goose_pages& pg, const PagedReqs& rq, int n_layers, int n_kv, int head_dim, PageScratch* scratch, bool reserved,
                        int32_t* flags, hipStream_t st) {
  const int4* res = reserved ? scratch->copies : nullptr;
  const dim3 grid(n_layers * n_kv, rq.n);
  if (head_dim == 128) hipLaunchKernelGGL(k_pages_move<128>, grid, dim3(128), 0, st, pg, rq, n_kv, res, scratch->verdict);
  else if (head_dim == 64) hipLaunchKernelGGL(k_pages_move<64>, grid, dim3(64), 0, st, pg, rq, n_kv, res, scratch->verdict);
  else return GOOSE_ERR_SHAPE;
  int rc = goose_launch_status();
  if (rc != GOOSE_OK) return rc;
  hipLaunchKernelGGL(k_pages_settle, dim3(rq.n), dim3(256), 0, st, pg, rq, res, scratch->verdict, flags);
  return goose_launch_status();
}

int launch_pages_free(const goose_pages& pg, const SeqList& seqs, int32_t* flags, hipStream_t st) {
  hipLaunchKernelGGL(k_pages_free, dim3(seqs.n), dim3(256), 0, st, pg, seqs, flags);
  return goose_launch_status();
}
