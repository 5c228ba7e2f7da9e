// Chunks of new tokens as the kernels see them.  Device code only (included by .hip files).
#pragma once
#include "attn_tile.h"

namespace {

// A chunk's committed slots: its sequence's length, held inside what the host has checked (P_max + C <= 64 table_ld).
__device__ inline int chunk_length(const int32_t* len, const ChunkReq& q, int32_t* flags, bool report) {
  const int P = __builtin_amdgcn_readfirstlane(len[q.seq]);
  const bool bad = P < 0 || P > q.P_max;
  if (bad && report) atomicOr(flags, GOOSE_FLAG_CAPACITY);
  return min(max(P, 0), q.P_max);
}
// Which of a lane's 16 keys a token sees: keys 0 .. last of them (negative: none).
__device__ __forceinline__ unsigned seen16(int last) { return last >= 15 ? 0xFFFFu : (last < 0 ? 0u : (2u << last) - 1u); }

}  // namespace
