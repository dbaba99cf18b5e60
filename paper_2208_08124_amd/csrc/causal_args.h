// What the kernels of the causal attention share: arguments, and the order in which its tiles are taken.
//
// A tile is 128 rows of one sequence: queries in the forward and the dQ pass, keys in the dK/dV pass.  Tile j of a
// sequence with n of them costs j + 1 in the former and, counted from the end, the same in the latter, so both take
// the tiles by falling j and the dK/dV pass reads j as n - 1 - j: the long ones first, the short ones fill the tail.
#pragma once
#include "kernel_args.h"
#include "mfma_tiles.h"

namespace fmha {

constexpr int kCausalSelf = 64;  // sequences up to which a kernel works the order out by itself, one lane each

struct CausalArgs {
  const int32_t* cu;
  int32_t batch, total;
  int32_t heads, kv_heads, group;
  float scale;
  const TileItem* list;  // null: the kernel looks for itself
  const int32_t* count;
  const uint16_t *q, *k, *v, *o_in, *d_o;
  uint16_t *o, *dq, *dk, *dv;
  float* lse;   // [H, T]
  float *dsum, *lse2;  // workspace, [H T + 1] each: -rowsum(dO o O) and lse log2(e)
  int64_t q_stride, k_stride, v_stride, o_stride, do_stride, dq_stride, dk_stride, dv_stride;
};

// Sum over the wavefront, in every lane.
__device__ __forceinline__ int wave_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);  // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);  // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);  // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return __builtin_amdgcn_readlane(x, 63);
}

// Whatever the device array holds, the rows [r0, r0 + len) lie inside the tensors.
__device__ __forceinline__ void causal_sequence(const CausalArgs& a, int i, int& r0, int& len) {
  r0 = min(max(a.cu[i], 0), a.total);
  len = min(max(a.cu[i + 1], r0), a.total) - r0;
}

// The tile of rank `rank` in the order of falling j (len = 0: there is none), for up to 64 sequences.  With
// C(j) = the number of tiles with an index of at least j, its index is the largest j with C(j) > rank, and it is number
// rank - C(j + 1) of the sequences that have such a tile.
__device__ __forceinline__ TileItem causal_find(const CausalArgs& a, int rank) {
  const int lane = threadIdx.x & 63;
  int r0 = 0, len = 0;
  if (lane < a.batch) causal_sequence(a, lane, r0, len);
  const int nt = (len + kTileRows - 1) / kTileRows;
  if (rank >= wave_sum(nt)) return TileItem{0, 0, 0, 0};
  int lo = 0, hi = (a.total + kTileRows - 1) / kTileRows, above = 0;  // C(lo) > rank >= C(hi) = above
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, c = wave_sum(max(nt - mid, 0));
    if (c > rank) {
      lo = mid;
    } else {
      hi = mid;
      above = c;
    }
  }
  uint64_t have = __ballot(nt > lo);
  for (int skip = rank - above; skip > 0; skip--) have &= have - 1;
  const int who = __builtin_ctzll(have);
  return TileItem{__builtin_amdgcn_readlane(r0, who), __builtin_amdgcn_readlane(len, who), 0, lo * kTileRows};
}

__device__ __forceinline__ TileItem causal_tile(const CausalArgs& a, int rank) {
  if (!a.list) return causal_find(a, rank);
  if (rank >= *(ConstInt)(uintptr_t)a.count) return TileItem{0, 0, 0, 0};
  ConstInt p = (ConstInt)(uintptr_t)(a.list + rank);
  return TileItem{p[0], p[1], 0, p[3]};
}

// The same order for more sequences, as a list: count[0] <- tiles, list[0 ..] <- the tiles.  One workgroup.  The
// indexes from 1023 on (sequences of more than 130 944 tokens) are taken together.
constexpr int kCausalListThreads = 1024;
__global__ __launch_bounds__(kCausalListThreads) void causal_list_kernel(const CausalArgs a, int32_t* count, TileItem* list, int cap) {
  __shared__ int have[kCausalListThreads];  // tiles of this index, then places of the index in the list
  __shared__ int part[kCausalListThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int last = kCausalListThreads - 1;
  __shared__ int more;  // tiles beyond the last index
  have[tid] = 0;
  if (tid == 0) more = 0;
  __syncthreads();
  // number of sequences by their number of tiles
  for (int i = tid; i < a.batch; i += kCausalListThreads) {
    int r0, len;
    causal_sequence(a, i, r0, len);
    const int nt = (len + kTileRows - 1) / kTileRows;
    if (nt > 0) atomicAdd(&have[min(nt, last + 1) - 1], 1);
    if (nt > last + 1) atomicAdd(&more, nt - last - 1);
  }
  __syncthreads();
  // tiles of index j = sequences with more than j tiles: sums from the end, so thread t scans in the place of index last - t
  auto scan = [&](int x) {  // inclusive, over the workgroup
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(x, d, 64);
      if (lane >= d) x += up;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; w++) x += part[w];
    __syncthreads();
    return x;
  };
  const int mine = scan(have[last - tid]) + (tid == 0 ? more : 0);  // tiles of index last - tid
  const int upto = scan(mine);
  have[last - tid] = upto - mine;
  if (tid == last) *count = min(upto, cap);
  __syncthreads();
  for (int i = wave; i < a.batch; i += kCausalListThreads / 64) {
    int r0, len;
    causal_sequence(a, i, r0, len);
    for (int j = lane; j * kTileRows < len; j += 64) {
      const int at = atomicAdd(&have[min(j, last)], 1);
      if (at < cap) list[at] = TileItem{r0, len, 0, j * kTileRows};
    }
  }
}

// Workgroup item: tile rank and head.  Consecutive items have different key heads, the eight dies take items
// in turn: with a multiple of eight key heads all that read one key head share a die's L2.
__device__ __forceinline__ int causal_head(int i, int heads, int kv_heads, int group) {
  return (i % kv_heads) * group + i / kv_heads % group;
}

// A block of ROWS rows of D channels in LDS: tiles of 64 channels (mfma_tiles.h), one behind the other.  Requests rows
// [row0, row0 + ROWS) of a tensor (rows behind last_row repeat it); wavefront w of four fills rows 8w .. 8w+7 (and 32 rows on).
template <int D, int ROWS>
__device__ __forceinline__ void dma_block(const uint16_t* base, int64_t stride, int row0, int last_row, int wave, uint32_t addr) {
  const int lane = lane_id();
  const int row = 8 * wave + (lane >> 3), chunk = (lane & 7) ^ swz(row);
  const uint16_t* rows = base + uniform_i64((int64_t)row0 * stride);
  const uint32_t st = (uint32_t)stride;
#pragma unroll
  for (int part = 0; part < ROWS / 32; part++) {
    const uint32_t off = ((uint32_t)min(row + 32 * part, last_row - row0) * st + chunk * 8) * 2u;
#pragma unroll
    for (int h = 0; h < D / 64; h++)
      dma16s(rows + 64 * h, off, __builtin_amdgcn_readfirstlane(addr + (uint32_t)(h * ROWS * 128 + part * 4096 + 1024 * wave)));
  }
}

}  // namespace fmha
