// Norm and rotation of query and key heads, forward and backward, and the same on the way into a
// paged cache.  Per row and head, on the head's channels x:
//   x <- x rstd gamma (rstd = 1 / sqrt(mean x^2 + eps)),  then for the pair (a, b) number i of the rotated part
//   (a, b) <- (a cos - b sin, a sin + b cos) m,  angle = position * inv_freq[i]
// and backward, with g the turned-back gradient and xh = x rstd,
//   dx = rstd (g gamma - xh mean(g gamma xh)),  dgamma = sum g xh.
//
// All of it is bound by memory: two bytes in and two out per channel (backward: four in, two out).  A head is spread over
// head_dim / 16 lanes, each with two pieces of eight channels: in the HALF layout the second piece is the partner
// of the first, so that pairs stay inside a lane and need no exchange; the norm's sum is the only thing that crosses lanes.
// Cosines and sines depend on the position alone: a wavefront forms them once and uses them for all the heads that it takes
// of a row.  The angle is a 64-bit product of position and turns per position whose whole turns are dropped before it
// becomes a float (an fp32 product would be off by 0.06 at position 10^6).
#pragma once
#include "mfma_tiles.h"

namespace fmha {

constexpr int kQkThreads = 256;

struct QkRows {
  int32_t rows, nq, nk, nv;  // nv: heads that are copied (the values, on their way into a cache)
  int32_t dim, lph, lp2;     // channels of a head; lanes of a head (dim / 16), and the power of two they are padded to
  int32_t gs, iters, parts;  // heads of a row that a wavefront takes at a time, how many times, wavefronts per row
  float eps;
  const uint16_t *q, *k, *v;
  uint16_t *qo, *ko;
  int64_t q_stride, k_stride, v_stride, qo_stride, ko_stride;
  const float *gamma_q, *gamma_k;
  const int32_t *positions, *cu, *n_rows;
  int32_t batch;
  int32_t rot;  // rotated channels
  const double* inv_freq;
  float magnitude;
  // the cache
  const int32_t *seqlens, *table;
  uint16_t *kc, *vc;
  int64_t page_stride;
  int32_t page_shift, num_pages, max_pages;
  // backward: q, k are the forward's inputs, dyq, dyk (strides qo, ko) its outputs' gradients
  const uint16_t *dyq, *dyk;
  uint16_t *dq, *dk;
  int64_t dq_stride, dk_stride;
  float* partial;
};

// Rows that are present.
__device__ __forceinline__ int qk_present(const QkRows& a) {
  int n = a.rows;
  if (a.n_rows)
    n = *a.n_rows;
  else if (a.cu)
    n = a.cu[a.batch];
  return min(max(n, 0), a.rows);
}

// The sequence of packed row t (0 <= t < cu[batch]; wave-uniform): the first i with cu[i + 1] > t.  All 64 lanes look at a
// boundary each, so that up to 64 sequences take one memory round trip and 4096 take two.
__device__ __forceinline__ int qk_sequence(const int32_t* __restrict__ cu, int batch, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = batch;
  while (true) {
    const int step = (n + 63) >> 6;
    const int at = min((lane + 1) * step, n);
    const int c = __popcll(__ballot((lane + 1) * step <= n + step - 1 && cu[lo + at] <= t));
    if (step == 1) return min(lo + c, batch - 1);
    lo += min(c * step, n - 1);
    n = min(step, batch - lo);
  }
}

// The pieces (of eight channels) of the lane that is number c of its head, and which of them are rotated.
struct QkPieces {
  int one, two;
  bool turn1, turn2;
  template <bool INTER>
  static __device__ __forceinline__ QkPieces of(int c, int lph, int rot) {
    if (INTER) return QkPieces{c, c + lph, 8 * c < rot, 8 * (c + lph) < rot};
    const int rc = rot >> 4;
    if (c < rc) return QkPieces{c, c + rc, true, true};
    return QkPieces{2 * c, 2 * c + 1, false, false};
  }
};

// Cosines and sines of the lane's eight pairs (HALF: pairs 8 one .. +7; INTER: pairs 4 one .. +3 and 4 two .. +3), times m.
template <bool INTER>
__device__ __forceinline__ void qk_angles(float (&cs)[8], float (&sn)[8], const QkPieces& pc, const double* __restrict__ freq,
                                          int pos, float m) {
#pragma unroll
  for (int j = 0; j < 8; j++) {
    cs[j] = 1.f;
    sn[j] = 0.f;
    const bool on = INTER ? (j < 4 ? pc.turn1 : pc.turn2) : pc.turn1;
    if (!on) continue;
    const int i = INTER ? (j < 4 ? 4 * pc.one + j : 4 * pc.two + j - 4) : 8 * pc.one + j;
    double turns = (double)pos * freq[i] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    sincospif(2.f * (float)turns, &sn[j], &cs[j]);
    cs[j] *= m;
    sn[j] *= m;
  }
}

// Turns the lane's sixteen channels; BACK: by the opposite angle.
template <bool INTER, bool BACK>
__device__ __forceinline__ void qk_turn(float (&x)[16], const float (&cs)[8], const float (&sn)[8], const QkPieces& pc) {
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const int p = INTER ? 2 * j : j, q = INTER ? 2 * j + 1 : j + 8;
    const bool on = INTER ? (j < 4 ? pc.turn1 : pc.turn2) : pc.turn1;
    if (!on) continue;
    const float a = x[p], b = x[q], s = BACK ? -sn[j] : sn[j];
    x[p] = a * cs[j] - b * s;
    x[q] = a * s + b * cs[j];
  }
}

template <typename T>
__device__ __forceinline__ float qk_lo(uint32_t w);
template <typename T>
__device__ __forceinline__ float qk_hi(uint32_t w);
template <>
__device__ __forceinline__ float qk_lo<__bf16>(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
template <>
__device__ __forceinline__ float qk_hi<__bf16>(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
template <>
__device__ __forceinline__ float qk_lo<_Float16>(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)w); }
template <>
__device__ __forceinline__ float qk_hi<_Float16>(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16)); }

template <typename T>
__device__ __forceinline__ void qk_unpack(float (&x)[16], const u32x4& a, const u32x4& b) {
#pragma unroll
  for (int j = 0; j < 4; j++) {
    x[2 * j] = qk_lo<T>(a[j]);
    x[2 * j + 1] = qk_hi<T>(a[j]);
    x[8 + 2 * j] = qk_lo<T>(b[j]);
    x[8 + 2 * j + 1] = qk_hi<T>(b[j]);
  }
}

template <typename T>
__device__ __forceinline__ void qk_pack(u32x4& a, u32x4& b, const float (&x)[16]) {
#pragma unroll
  for (int j = 0; j < 4; j++) {
    a[j] = Op<T>::pack2(x[2 * j], x[2 * j + 1]);
    b[j] = Op<T>::pack2(x[8 + 2 * j], x[8 + 2 * j + 1]);
  }
}

// Sum over the lanes of a head.
__device__ __forceinline__ float qk_head_sum(float x, int lp2) {
  for (int m = 1; m < lp2; m <<= 1) x += __shfl_xor(x, m, 64);
  return x;
}

__device__ __forceinline__ void qk_gamma(float (&w)[16], const float* __restrict__ gamma, const QkPieces& pc) {
#pragma unroll
  for (int j = 0; j < 2; j++) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(gamma + 8 * pc.one + 4 * j);
    const f32x4 b = *reinterpret_cast<const f32x4*>(gamma + 8 * pc.two + 4 * j);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      w[4 * j + e] = a[e];
      w[8 + 4 * j + e] = b[e];
    }
  }
}

// Position of the lane's token: tokens tok0 .. tok0 + tpw - 1 belong to the wavefront, the lane to number `mine`.
// CACHE: also the sequence.
template <bool CACHE>
__device__ __forceinline__ int qk_position(const QkRows& a, int tok0, int tpw, int mine, int present, int& seq) {
  int pos = 0;
  seq = 0;
  if (!CACHE && a.positions) return mine < present - tok0 ? a.positions[tok0 + mine] : 0;
  if (!a.cu) {
    if (CACHE && mine < present - tok0) {
      seq = tok0 + mine;
      pos = a.seqlens[seq] - 1;
    }
    return pos;
  }
  const int lane = threadIdx.x & 63;
  int begin = 0, end = 0x7fffffff, held = 0;  // of sequence `lane`, where each has a lane
  if (a.batch <= 64 && lane < a.batch) {
    begin = a.cu[lane];
    end = a.cu[lane + 1];
    if (CACHE) held = a.seqlens[lane];
  }
  for (int i = 0; i < min(tpw, present - tok0); i++) {
    const int t = tok0 + i;
    int s, at;
    if (a.batch <= 64) {
      s = min((int)__popcll(__ballot(end <= t)), a.batch - 1);
      at = CACHE ? __builtin_amdgcn_readlane(held, s) - __builtin_amdgcn_readlane(end, s) + t : t - __builtin_amdgcn_readlane(begin, s);
    } else {
      s = qk_sequence(a.cu, a.batch, t);
      at = CACHE ? a.seqlens[s] - a.cu[s + 1] + t : t - a.cu[s];
    }
    if (i == mine) {
      pos = at;
      seq = s;
    }
  }
  return pos;
}

// Forward.  A wavefront takes 64 / (lp2 gs) rows and gs heads of each at a time, `iters` times.  CACHE: keys and values go to
// their place in the cache, the heads being those of q, k and v one after the other.
template <typename T, bool INTER, bool CACHE>
__global__ __launch_bounds__(kQkThreads) void qk_rows_kernel(const QkRows a) {
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (kQkThreads / 64) + (threadIdx.x >> 6);
  const int slots = 64 / a.lp2, tpw = slots / a.gs;
  const int present = qk_present(a);
  const int64_t group = wave / a.parts;
  if (group * tpw >= present) return;
  const int tok0 = __builtin_amdgcn_readfirstlane((int)(group * tpw));
  const int part = (int)(wave - group * a.parts);
  const int c = lane % a.lp2, slot = lane / a.lp2;
  const int mine = slot / a.gs, tok = tok0 + min(mine, present - tok0);  // (= present: no row)
  const bool on = c < a.lph;  // not one of the lanes that a head is padded with
  const QkPieces pc = QkPieces::of<INTER>(c, a.lph, a.rot);
  const int heads = a.nq + a.nk + a.nv;
  const int first = part * a.iters * a.gs + slot % a.gs, last = min(heads, first + a.iters * a.gs);
  auto fetch = [&](u32x4& w1, u32x4& w2, int h) {
    w1 = w2 = u32x4{0u, 0u, 0u, 0u};
    if (!on || tok >= present || h >= last) return;
    const bool is_v = CACHE && h >= a.nq + a.nk;
    const uint16_t* src = h < a.nq ? a.q + tok * a.q_stride + (int64_t)h * a.dim
                          : is_v   ? a.v + tok * a.v_stride + (int64_t)(h - a.nq - a.nk) * a.dim
                                   : a.k + tok * a.k_stride + (int64_t)(h - a.nq) * a.dim;
    w1 = *reinterpret_cast<const u32x4*>(src + 8 * pc.one);
    w2 = *reinterpret_cast<const u32x4*>(src + 8 * pc.two);
  };
  u32x4 w1, w2;
  fetch(w1, w2, first);  // (ahead of all that it takes to know the position)
  int seq;
  const int pos = a.rot || CACHE ? qk_position<CACHE>(a, tok0, tpw, mine, present, seq) : 0;
  if (tok >= present || first >= last) return;  // (here and below control goes by whole heads: what their lanes exchange is there)
  int64_t place = -1;  // of the token in a cache of one head
  if (CACHE) {
    const int page = pos >> a.page_shift;
    if (pos >= 0 && page < a.max_pages) {
      const int g = a.table[(int64_t)seq * a.max_pages + page];
      if (g >= 0 && g < a.num_pages)
        place = g * a.page_stride + (int64_t)(pos & ((1 << a.page_shift) - 1)) * a.dim;
    }
  }
  float cs[8], sn[8];
  if (on) qk_angles<INTER>(cs, sn, pc, a.inv_freq, pos, a.magnitude);
  for (int h = first; h < last; h += a.gs) {
    u32x4 next1, next2;
    fetch(next1, next2, h + a.gs);
    const bool is_q = h < a.nq, is_v = CACHE && h >= a.nq + a.nk;
    const int hk = h - a.nq - (is_v ? a.nk : 0);
    uint16_t* dst = nullptr;  // (null: a token without a place)
    if (is_q)
      dst = a.qo + tok * a.qo_stride + (int64_t)h * a.dim;
    else if (!CACHE)
      dst = a.ko + tok * a.ko_stride + (int64_t)hk * a.dim;
    else if (place >= 0)
      dst = (is_v ? a.vc : a.kc) + place + (((int64_t)hk * a.dim) << a.page_shift);
    if (!is_v) {
      float x[16];
      qk_unpack<T>(x, w1, w2);
      const float* gamma = is_q ? a.gamma_q : a.gamma_k;
      if (gamma) {
        float w[16] = {}, ss = 0.f;
        if (on) qk_gamma(w, gamma, pc);
#pragma unroll
        for (int j = 0; j < 16; j++) ss += x[j] * x[j];
        ss = qk_head_sum(ss, a.lp2);
        const float rstd = 1.f / sqrtf(ss / (float)a.dim + a.eps);
#pragma unroll
        for (int j = 0; j < 16; j++) x[j] *= rstd * w[j];
      }
      if (on) qk_turn<INTER, false>(x, cs, sn, pc);
      qk_pack<T>(w1, w2, x);
    }
    if (on && dst) {
      *reinterpret_cast<u32x4*>(dst + 8 * pc.one) = w1;
      *reinterpret_cast<u32x4*>(dst + 8 * pc.two) = w2;
    }
    w1 = next1;
    w2 = next2;
  }
}

// Backward.  Wavefronts go over the rows in strides, so that the sums for gamma stay in registers to the end; they are
// then added up over the wavefront's heads and rows, over the workgroup, and by qk_gamma_kernel over the
// workgroups, always in the same order.  partial: [workgroups][2][dim].
template <typename T, bool INTER>
__global__ __launch_bounds__(kQkThreads, 3) void qk_rows_bwd_kernel(const QkRows a) {
  __shared__ float sums[kQkThreads / 64][2][256];  // (first gamma: [0][0] of the queries, [0][1] of the keys)
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int slots = 64 / a.lp2, tpw = slots / a.gs;
  const int present = qk_present(a);
  const int c = lane % a.lp2, slot = lane / a.lp2, mine = slot / a.gs;
  const bool on = c < a.lph;
  const QkPieces pc = QkPieces::of<INTER>(c, a.lph, a.rot);
  const int heads = a.nq + a.nk;
  const int items = present > 0 ? ((present - 1) / tpw + 1) * a.parts : 0;
  for (int i = threadIdx.x; i < a.dim; i += kQkThreads) {
    sums[0][0][i] = a.gamma_q ? a.gamma_q[i] : 1.f;
    sums[0][1][i] = a.gamma_k ? a.gamma_k[i] : 1.f;
  }
  __syncthreads();
  struct Raw {
    u32x4 g1, g2, x1, x2;
  };
  // (an empty place, or a lane that its head is padded with, works on zeros)
  auto fetch = [&](Raw& r, int tok, int h, int last) {
    r.g1 = r.g2 = r.x1 = r.x2 = u32x4{0u, 0u, 0u, 0u};
    if (!on || h >= last || tok >= present) return;
    const bool is_q = h < a.nq;
    const int64_t col = (int64_t)(is_q ? h : h - a.nq) * a.dim;
    const uint16_t* dy = is_q ? a.dyq + tok * a.qo_stride + col : a.dyk + tok * a.ko_stride + col;
    r.g1 = *reinterpret_cast<const u32x4*>(dy + 8 * pc.one);
    r.g2 = *reinterpret_cast<const u32x4*>(dy + 8 * pc.two);
    if (is_q ? a.gamma_q : a.gamma_k) {
      const uint16_t* xs = is_q ? a.q + tok * a.q_stride + col : a.k + tok * a.k_stride + col;
      r.x1 = *reinterpret_cast<const u32x4*>(xs + 8 * pc.one);
      r.x2 = *reinterpret_cast<const u32x4*>(xs + 8 * pc.two);
    }
  };
  float sum_q[16] = {}, sum_k[16] = {};
  for (int item = blockIdx.x * (kQkThreads / 64) + w; item < items; item += gridDim.x * (kQkThreads / 64)) {
    const int group = item / a.parts, part = item - group * a.parts;
    const int tok0 = __builtin_amdgcn_readfirstlane(group * tpw), tok = tok0 + min(mine, present - tok0);
    const int first = part * a.iters * a.gs + slot % a.gs, last = min(heads, first + a.iters * a.gs);
    Raw cur;
    fetch(cur, tok, first, last);
    int seq;
    const int pos = a.rot ? qk_position<false>(a, tok0, tpw, mine, present, seq) : 0;
    if (tok >= present) continue;  // (whole heads)
    float cs[8], sn[8];
    if (on) qk_angles<INTER>(cs, sn, pc, a.inv_freq, pos, a.magnitude);
    for (int h = first; h < last; h += a.gs) {
      Raw next;
      fetch(next, tok, h + a.gs, last);  // the next head's rows, ahead of this one's work
      const bool is_q = h < a.nq;
      const bool normed = is_q ? a.gamma_q : a.gamma_k;
      float g[16];
      qk_unpack<T>(g, cur.g1, cur.g2);
      if (on) qk_turn<INTER, true>(g, cs, sn, pc);
      if (normed) {
        float x[16], wt[16] = {}, ss = 0.f, dot = 0.f;
        qk_unpack<T>(x, cur.x1, cur.x2);
        if (on) qk_gamma(wt, sums[0][is_q ? 0 : 1], pc);
#pragma unroll
        for (int j = 0; j < 16; j++) {
          wt[j] *= g[j];
          ss += x[j] * x[j];
          dot += wt[j] * x[j];
        }
        ss = qk_head_sum(ss, a.lp2);
        dot = qk_head_sum(dot, a.lp2);
        const float rstd = 1.f / sqrtf(ss / (float)a.dim + a.eps);
        const float m = dot * rstd / (float)a.dim;  // mean(g gamma xh)
#pragma unroll
        for (int j = 0; j < 16; j++) {
          const float xh = x[j] * rstd;
          if (is_q)
            sum_q[j] += g[j] * xh;
          else
            sum_k[j] += g[j] * xh;
          g[j] = rstd * (wt[j] - xh * m);
        }
      }
      if (on) {
        const int64_t col = (int64_t)(is_q ? h : h - a.nq) * a.dim;
        uint16_t* dx = is_q ? a.dq + tok * a.dq_stride + col : a.dk + tok * a.dk_stride + col;
        u32x4 w1, w2;
        qk_pack<T>(w1, w2, g);
        *reinterpret_cast<u32x4*>(dx + 8 * pc.one) = w1;
        *reinterpret_cast<u32x4*>(dx + 8 * pc.two) = w2;
      }
      cur = next;
    }
  }
  if (!a.gamma_q && !a.gamma_k) return;
  for (int m = a.lp2; m < 64; m <<= 1) {
#pragma unroll
    for (int j = 0; j < 16; j++) {
      sum_q[j] += __shfl_xor(sum_q[j], m, 64);
      sum_k[j] += __shfl_xor(sum_k[j], m, 64);
    }
  }
  __syncthreads();  // gamma is done with
  if (slot == 0 && on) {
#pragma unroll
    for (int j = 0; j < 16; j++) {
      const int at = j < 8 ? 8 * pc.one + j : 8 * pc.two + j - 8;
      sums[w][0][at] = sum_q[j];
      sums[w][1][at] = sum_k[j];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += kQkThreads) {
    const int which = i >= a.dim, at = i - which * a.dim;
    a.partial[(int64_t)blockIdx.x * 2 * a.dim + i] =
        (sums[0][which][at] + sums[1][which][at]) + (sums[2][which][at] + sums[3][which][at]);
  }
}

// dgamma_q[c] and dgamma_k[c] <- the sums of column c over `rows` partial rows.  One workgroup per 64 columns, sixteen
// wavefronts that take every sixteenth row.
constexpr int kQkGammaThreads = 1024;
__global__ __launch_bounds__(kQkGammaThreads) void qk_gamma_kernel(const float* __restrict__ partial, int rows, int dim,
                                                                   float* dgamma_q, float* dgamma_k) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (col < 2 * dim) {
    const float* src = partial + (int64_t)w * 2 * dim + col;
    const int64_t step = (int64_t)16 * 2 * dim;
    for (int r = w; r < rows; r += 16 * 16) {  // sixteen rows in flight: one after the other takes 27 us for 1024 rows of 256
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; i++) x[i] = r + 16 * i < rows ? src[i * step] : 0.f;
#pragma unroll
      for (int i = 0; i < 16; i++) s += x[i];
      src += 16 * step;
    }
  }
  sums[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < 2 * dim) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) s += sums[i][lane];
    float* out = col < dim ? dgamma_q : dgamma_k;
    if (out) out[col < dim ? col : col - dim] = s;
  }
}

}  // namespace fmha
