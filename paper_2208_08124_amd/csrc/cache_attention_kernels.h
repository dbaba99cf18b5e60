// Attention of one query token per sequence over a paged cache of keys and values:
//   o = softmax(scale q K^T) V  over the sequence's keys, and the log-sum-exp,
// with the heads of a group (heads / kv_heads query heads that share a key head) taken together, up to sixteen.
//
// Bound by memory: every key and value is read once, 4 head_dim bytes, for 4 head_dim products per query head.  So what
// counts is bytes in flight.  Each wavefront works by itself on blocks of 32 keys, 16 KB at head_dim 128, and requests the
// next block into registers before it works on the present one; nothing in the loop waits for another wavefront.
// The products run on the matrix cores, with the group's heads as the sixteen columns (empty ones cost nothing that
// is short): S^T = K Q^T has a lane hold one head's scores of eight keys, which after the softmax are, in place, the
// operand of O^T += V^T P^T.  K comes straight from memory in the layout of that operand (a lane has a key's
// channels); V passes through LDS, from where it is read transposed.
// A sequence's keys are split over workgroups in chunks, and over a workgroup's four wavefronts in turn; each
// keeps its own running maximum and sum, and what they have is joined in LDS, in a fixed order, and across workgroups
// by cache_join_kernel from normalised partial results and their log-sum-exps.
#pragma once
#include "mfma_tiles.h"

namespace fmha {

constexpr int kCacheThreads = 256;  // of the join
constexpr int kCacheBlock = 32;     // keys a wavefront takes at a time
constexpr int kCacheStep = 8 * kCacheBlock;  // chunks are multiples of it

struct CacheArgs {
  const uint16_t *q, *k, *v;
  uint16_t* o;
  float* lse;
  const int32_t *table, *seqlens;
  int64_t q_stride, o_stride, page_stride;
  int32_t batch, heads, kv_heads, group, tiles;  // tiles of sixteen heads in a group
  int32_t page_shift, num_pages, max_pages;
  int32_t waves;          // of a workgroup
  int32_t chunk, splits;  // keys of a workgroup; the last one takes what is left
  float scale;
  float* part_o;    // [splits][batch][heads][head_dim], where there are several
  float* part_lse;  // [splits][batch][heads], log2 units
};

template <typename T>
struct Mfma16x16;
template <>
struct Mfma16x16<_Float16> {
  static __device__ __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma16x16<__bf16> {
  static __device__ __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// Keys that sequence b has in the cache.
__device__ __forceinline__ int cache_keys(const CacheArgs& a, int b) {
  const int64_t room = (int64_t)a.max_pages << a.page_shift;
  const int n = max(a.seqlens[b], 0);
  return n < room ? n : (int)room;
}

// A block of 32 keys on its way: what the lane holds of K as operand (key 16 t + lane % 16, channels 32 s + 8 (lane / 16) .. +7)
// and of V (row and chunk as below), and which of the keys are attended.
template <int D>
struct CacheBlock {
  u32x4 k[2][D / 32];
  u32x4 v[D / 16];
  uint32_t on;  // bit j: key j of the block
};

// Page of key key0 + lane % 32, or -1.
__device__ __forceinline__ int cache_page(const CacheArgs& a, const int32_t* __restrict__ row, int key0, int end) {
  const int key = key0 + (int)(threadIdx.x & 31);
  return key < end ? row[key >> a.page_shift] : -1;
}

template <int D>
__device__ __forceinline__ void cache_request(CacheBlock<D>& blk, const CacheArgs& a, int page, int key0, int hk) {
  const int lane = threadIdx.x & 63;
  if (page >= a.num_pages) page = -1;
  blk.on = (uint32_t)__ballot(page >= 0);
  const int mask = (1 << a.page_shift) - 1;
  auto at = [&](int pg, int key) {
    return (int64_t)pg * a.page_stride + (((int64_t)hk << a.page_shift) + (key & mask)) * D;
  };
  const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int t = 0; t < 2; t++) {
    const int j = 16 * t + (lane & 15), pg = __shfl(page, j, 64);
    const uint16_t* p = a.k + at(pg, key0 + j) + 8 * (lane >> 4);
#pragma unroll
    for (int s = 0; s < D / 32; s++) blk.k[t][s] = pg >= 0 ? *reinterpret_cast<const u32x4*>(p + 32 * s) : zero;
  }
#pragma unroll
  for (int i = 0; i < D / 16; i++) {
    const int j = i * (512 / D) + lane / (D / 8), pg = __shfl(page, j, 64);
    blk.v[i] = pg >= 0 ? *reinterpret_cast<const u32x4*>(a.v + at(pg, key0 + j) + 8 * (lane % (D / 8))) : zero;
  }
}

// W: wavefronts, four or (for few sequences that are not worth splitting over workgroups) eight.
template <typename T, int D, int W>
__global__ __launch_bounds__(64 * W, D == 64 ? 3 : 2) void cache_attention_kernel(const CacheArgs a) {
  constexpr int kThreads = 64 * W, kStep = W * kCacheBlock;
  constexpr int kOutRow = D + 4;  // floats; (16 lanes write 16 rows at a time)
  __shared__ __align__(16) union {
    uint16_t v[W][D / 64][kCacheBlock * 64];
    float o[W][16][kOutRow];
  } lds;
  __shared__ float stat[2][W][16];  // maximum (log2 units) and sum
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, c = lane >> 4;
  int idx = blockIdx.x;
  const int tile = idx % a.tiles;
  idx /= a.tiles;
  const int hk = idx % a.kv_heads;
  idx /= a.kv_heads;
  const int b = idx % a.batch, split = idx / a.batch;
  const int n = cache_keys(a, b);
  const int begin = split * a.chunk;
  const int end = split == a.splits - 1 ? n : min(n, begin + a.chunk);
  if (begin >= end && split > 0) return;
  const int h0 = hk * a.group + 16 * tile, n_heads = min(16, a.group - 16 * tile);
  const int32_t* row = a.table + (int64_t)b * a.max_pages;

  // Q^T as operand: column = head, the lane's channels as in CacheBlock::k.  Columns without a head repeat the last one.
  u32x4 qb[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; s++)
    qb[s] = *reinterpret_cast<const u32x4*>(a.q + b * a.q_stride + (int64_t)(h0 + min(col, n_heads - 1)) * D + 32 * s + 8 * c);

  f32x4 o[D / 16];  // O^T: column = head, rows = channels 16 dt + 4 c .. +3
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;  // l: of this lane's keys
  const float c2 = a.scale * kLog2e;

  uint16_t* vs = &lds.v[wave][0][0];
  auto work = [&](const CacheBlock<D>& blk) {
#pragma unroll
    for (int i = 0; i < D / 16; i++) {
      const int r = i * (512 / D) + lane / (D / 8), ch = lane % (D / 8);
      *reinterpret_cast<u32x4*>(vs + (ch >> 3) * (kCacheBlock * 64) + tile_off(r, 8 * (ch & 7))) = blk.v[i];
    }
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int i = 0; i < D / 32; i++) s[t] = Mfma16x16<T>::mul(blk.k[t][i], qb[i], s[t]);
    float p[8], top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const bool on = (blk.on >> (16 * t + 4 * c + r)) & 1u;
        p[4 * t + r] = on ? s[t][r] * c2 : -INFINITY;
        top = fmaxf(top, p[4 * t + r]);
      }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new;
    const float keep = fast_exp2(m - base);
    m = m_new;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 8; r++) {
      p[r] = fast_exp2(p[r] - base);
      sum += p[r];
    }
    l = l * keep + sum;
    // (rounded to the operand's type: at most half a step of each probability, which the sum does not share)
    const u32x4 pb = {Op<T>::pack2(p[0], p[1]), Op<T>::pack2(p[2], p[3]), Op<T>::pack2(p[4], p[5]), Op<T>::pack2(p[6], p[7])};
    if (__ballot(keep != 1.f)) {
#pragma unroll
      for (int dt = 0; dt < D / 16; dt++) o[dt] *= keep;
    }
    __builtin_amdgcn_wave_barrier();  // same wavefront: its LDS operations execute in order
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++) {
      const uint16_t* t = vs + (dt >> 2) * (kCacheBlock * 64);
      const int r = 4 * c + (col >> 2), x = 16 * (dt & 3) + 4 * (col & 3);
      const u32x2 lo = lds_read_tr16(t + tile_off(r, x)), hi = lds_read_tr16(t + tile_off(r + 16, x));
      o[dt] = Mfma16x16<T>::mul(u32x4{lo[0], lo[1], hi[0], hi[1]}, pb, o[dt]);
    }
    __builtin_amdgcn_wave_barrier();
  };

  // The pages of a block are looked up ahead of the requests for the block before it, so that the wait for them
  // leaves those requests in flight (loads come back in order).
  int key0 = begin + kCacheBlock * wave;
  if (key0 < end) {
    CacheBlock<D> cur, next;
    const int first = cache_page(a, row, key0, end);
    int page = cache_page(a, row, key0 + kStep, end);
    cache_request(cur, a, first, key0, hk);
    for (; key0 < end; key0 += kStep) {
      const int page2 = cache_page(a, row, key0 + 2 * kStep, end);
      const bool more = key0 + kStep < end;
      if (more) cache_request(next, a, page, key0 + kStep, hk);
      work(cur);
      cur = next;
      page = page2;
    }
  }

  // Join the wavefronts.
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();  // the V blocks are done with
  if (c == 0) {
    stat[0][wave][col] = m;
    stat[1][wave][col] = l;
  }
#pragma unroll
  for (int dt = 0; dt < D / 16; dt++) *reinterpret_cast<f32x4*>(&lds.o[wave][col][16 * dt + 4 * c]) = o[dt];
  __syncthreads();
  for (int i = threadIdx.x; i < n_heads * (D / 4); i += kThreads) {
    const int h = i / (D / 4), x = 4 * (i % (D / 4));
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < W; w++) top = fmaxf(top, stat[0][w][h]);
    const float base = top == -INFINITY ? 0.f : top;
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; w++) {
      const float share = fast_exp2(stat[0][w][h] - base);
      total += share * stat[1][w][h];
      r += share * *reinterpret_cast<const f32x4*>(&lds.o[w][h][x]);
    }
    const float inv = total > 0.f || total != total ? 1.f / total : 0.f;  // (a NaN among the scores stays one)
    r *= inv;
    const float lse2 = top + __log2f(total);  // (no key: -inf, twice)
    if (a.splits == 1) {
      const u32x2 w2 = {Op<T>::pack2(r[0], r[1]), Op<T>::pack2(r[2], r[3])};
      *reinterpret_cast<u32x2*>(a.o + b * a.o_stride + (int64_t)(h0 + h) * D + x) = w2;
      if (x == 0) a.lse[(int64_t)b * a.heads + h0 + h] = lse2 * kLn2;
    } else {
      const int64_t at = ((int64_t)split * a.batch + b) * a.heads + h0 + h;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + x) = r;
      if (x == 0) a.part_lse[at] = lse2;
    }
  }
}

// o and lse of a (sequence, head) from its parts: a workgroup each, whose wavefronts take every fourth part and
// are added up in order.  The weights are formed first, a part to a lane, so that the rows come in without waiting for them.
constexpr int kJoinParts = 256;  // parts whose weights stand in LDS at a time
template <typename T, int D>
__global__ __launch_bounds__(kCacheThreads) void cache_join_kernel(const CacheArgs a) {
  constexpr int W = kCacheThreads / 64;
  __shared__ float share[kJoinParts], tops[W];
  __shared__ __align__(16) float rows[W][D];
  __shared__ float sums[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t at = blockIdx.x, all = (int64_t)a.batch * a.heads;
  const int b = (int)(at / a.heads), h = (int)(at - (int64_t)b * a.heads);
  const int n = cache_keys(a, b);
  const int parts = max(1, min(a.splits, (n + a.chunk - 1) / a.chunk));
  float top = -INFINITY;
  for (int s = tid; s < parts; s += kCacheThreads) top = fmaxf(top, a.part_lse[s * all + at]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; w++) top = fmaxf(top, tops[w]);
  const float base = top == -INFINITY ? 0.f : top;
  float x[D / 64] = {}, total = 0.f;
  for (int s0 = 0; s0 < parts; s0 += kJoinParts) {
    __syncthreads();
    for (int s = tid; s < kJoinParts; s += kCacheThreads)
      share[s] = s0 + s < parts ? fast_exp2(a.part_lse[(s0 + s) * all + at] - base) : 0.f;
    __syncthreads();
    const int upto = min(kJoinParts, parts - s0);
    for (int s = wave; s < upto; s += 16 * W) {
      float y[16][D / 64];
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const float* src = a.part_o + ((s0 + min(s + i * W, upto - 1)) * all + at) * D + lane * (D / 64);
#pragma unroll
        for (int e = 0; e < D / 64; e++) y[i][e] = src[e];
      }
#pragma unroll
      for (int i = 0; i < 16; i++) {
        if (s + i * W >= upto) break;
        const float f = share[s + i * W];
        total += f;
#pragma unroll
        for (int e = 0; e < D / 64; e++) x[e] += f * y[i][e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < D / 64; e++) rows[wave][lane * (D / 64) + e] = x[e];
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  if (tid >= D / 2) return;
  float r0 = 0.f, r1 = 0.f;
  total = 0.f;
#pragma unroll
  for (int w = 0; w < W; w++) {
    total += sums[w];
    r0 += rows[w][2 * tid];
    r1 += rows[w][2 * tid + 1];
  }
  const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
  *reinterpret_cast<uint32_t*>(a.o + b * a.o_stride + (int64_t)h * D + 2 * tid) = Op<T>::pack2(r0 * inv, r1 * inv);
  if (tid == 0) a.lse[at] = (top + __log2f(total)) * kLn2;
}

}  // namespace fmha
