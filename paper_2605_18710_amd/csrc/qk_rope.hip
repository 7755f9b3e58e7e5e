// What lies between a layer's QKV product and its attention in models that see images and video: a norm over every query
// and key head, then a rotation whose position has several axes, on packed rows [q (H heads) | k (Hkv heads) | v (Hkv heads)].
//
//   xhat = (x - mean) * rstd (mean = 0 for RMS norms), n = gain * xhat + shift, y = R n
//   backward: g = R^T dy, dgain = sum g * xhat, dshift = sum g, w = gain * g, dx = rstd * (w - mean(w) [LayerNorm] - xhat * mean(w * xhat))
//
// R turns pair i of a head by position[axis(i)] * frequency(i).  The angle is formed in double as a number of turns, whose
// whole part is dropped there: a position of any int32 keeps its digits.  rstd is formed again in the backward pass, which reads x anyway.
#include <algorithm>
#include <math.h>
#include "kernels.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxD = 256;
constexpr int kMaxParts = 1024;      // partitions of the gains' gradients
constexpr int kMaxAxes = MOSAIC_MAX_AXES;

// one pair of a head: turns (of 2 pi) for each unit of position on its axis; axis -1: the pair stays
struct PairTurn {
  double turns;
  int axis, unused;
};
static_assert(sizeof(PairTurn) == 16, "an entry of the table");

struct Sections { int32_t n[kMaxAxes]; };

__global__ __launch_bounds__(kThreads) void axes_table_kernel(PairTurn* __restrict__ table, int half, int n_axes, Sections sections, int order, double base) {
  for (int i = blockIdx.x * kThreads + threadIdx.x; i < half; i += gridDim.x * kThreads) {
    PairTurn p = {0.0, -1, 0};
    int nth = 0;                                     // the pair's number among those of its axis
    if (order == MOSAIC_AXES_DEALT) {                // one to each axis in turn while it has room
      int left = i;
      for (int round = 0; p.axis < 0 && round < half; ++round)
        for (int a = 0; a < n_axes; ++a)
          if (round < sections.n[a] && left-- == 0) { p.axis = a; nth = round; break; }
    } else {
      int first = 0;
      for (int a = 0; a < n_axes; ++a) {
        if (i >= first && i < first + sections.n[a]) { p.axis = a; nth = i - first; }
        first += sections.n[a];
      }
    }
    if (p.axis >= 0) {
      const double e = order == MOSAIC_AXES_OWN ? (double)nth / sections.n[p.axis] : (double)i / half;
      p.turns = pow(base, -e) * 0.15915494309189533577;      // 1 / (2 pi)
    }
    table[i] = p;
  }
}

struct Turn { float c, s; };
struct Positions {
  const int32_t* pos;      // [n_axes, T]
  const PairTurn* table;   // null: nothing turns
  int64_t T;
  int n_axes;
};
__device__ __forceinline__ Turn turn_of(const Positions& p, int64_t t, int i) {
  Turn r = {1.f, 0.f};
  if (!p.table) return r;
  const PairTurn e = p.table[i];
  if (e.axis < 0 || e.axis >= p.n_axes) return r;
  double turns = (double)p.pos[e.axis * p.T + t] * e.turns;
  turns -= rint(turns);
  sincospif(2.f * (float)turns, &r.s, &r.c);
  return r;
}

// the elements of pair i of a head
template <bool HALVES> __device__ __forceinline__ int first_of(int i) { return HALVES ? i : 2 * i; }
template <bool HALVES> __device__ __forceinline__ int second_of(int i, int half) { return HALVES ? i + half : 2 * i + 1; }

// Any even head size up to 256 and any alignment: a wave takes a head of a token, a lane up to two of its pairs.
template <typename T, int NORM, bool HALVES>
__global__ __launch_bounds__(kThreads) void qk_fwd_any_kernel(const T* x, T* y, Positions at, int H, int Hkv, int d, int heads, float eps, float sign,
                                                              const T* __restrict__ gq, const T* __restrict__ bq, const T* __restrict__ gk, const T* __restrict__ bk) {
  const int lane = threadIdx.x & 63, half = d / 2;
  const int64_t items = at.T * heads, width = (int64_t)(H + 2 * Hkv) * d;
  for (int64_t item = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * kWaves) {
    const int64_t t = item / heads;
    const int head = (int)(item - t * heads);
    const T* xp = x + t * width + (int64_t)head * d;
    T* yp = y + t * width + (int64_t)head * d;
    if (head >= H + Hkv) {                            // v goes through as it is
      for (int c = lane; c < d; c += 64) yp[c] = xp[c];
      continue;
    }
    float a[2] = {0.f, 0.f}, b[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = lane + 64 * u;
      if (i < half) { a[u] = to_f32(xp[first_of<HALVES>(i)]); b[u] = to_f32(xp[second_of<HALVES>(i, half)]); }
    }
    float mean = 0.f, rstd = 1.f;
    if constexpr (NORM != MOSAIC_NORM_NONE) {
      if constexpr (NORM == MOSAIC_LAYERNORM) mean = wave_sum(a[0] + b[0] + a[1] + b[1]) / (float)d;
      float sq = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < half) sq += (a[u] - mean) * (a[u] - mean) + (b[u] - mean) * (b[u] - mean);
      rstd = 1.f / sqrtf(wave_sum(sq) / (float)d + eps);
    }
    const T* g = head < H ? gq : gk;
    const T* sh = head < H ? bq : bk;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = lane + 64 * u;
      if (i >= half) continue;
      const int ca = first_of<HALVES>(i), cb = second_of<HALVES>(i, half);
      float na = a[u], nb = b[u];
      if constexpr (NORM != MOSAIC_NORM_NONE) {
        na = (na - mean) * rstd * to_f32(g[ca]);
        nb = (nb - mean) * rstd * to_f32(g[cb]);
        if constexpr (NORM == MOSAIC_LAYERNORM) { na += to_f32(sh[ca]); nb += to_f32(sh[cb]); }
      }
      const Turn r = turn_of(at, t, i);
      const float s = sign * r.s;
      yp[ca] = from_f32<T>(na * r.c - nb * s);
      yp[cb] = from_f32<T>(na * s + nb * r.c);
    }
  }
}

// The backward pass for any even head size.  A workgroup takes partitions of rp tokens, its waves their heads in turn; a lane holds the
// gains' sums of its columns, which the four waves add in order: partial[p] = [dgain q | dgain k | dshift q | dshift k].
template <typename T, int NORM, bool HALVES>
__global__ __launch_bounds__(kThreads) void qk_bwd_any_kernel(const T* __restrict__ x, const T* dy, T* dx, Positions at, int H, int Hkv, int d, int heads, float eps,
                                                              const T* __restrict__ gq, const T* __restrict__ gk, float* __restrict__ partial, int rp, int np) {
  __shared__ float sums[kWaves][4 * kMaxD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = d / 2;
  const int64_t width = (int64_t)(H + 2 * Hkv) * d;
  for (int p = blockIdx.x; p < np; p += gridDim.x) {
    float acc[2][2][4] = {};                           // [q or k][pair of the lane][dgain a, dgain b, dshift a, dshift b]
    const int64_t t0 = (int64_t)p * rp, t1 = min(t0 + rp, at.T), items = (t1 - t0) * heads;
    for (int64_t item = wave; item < items; item += kWaves) {
      const int64_t t = t0 + item / heads;
      const int head = (int)(item % heads);
      const int64_t off = t * width + (int64_t)head * d;
      if (head >= H + Hkv) {
        for (int c = lane; c < d; c += 64) dx[off + c] = dy[off + c];
        continue;
      }
      float a[2] = {0.f, 0.f}, b[2] = {0.f, 0.f}, ga[2] = {0.f, 0.f}, gb[2] = {0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = lane + 64 * u;
        if (i >= half) continue;
        const int ca = first_of<HALVES>(i), cb = second_of<HALVES>(i, half);
        a[u] = to_f32(x[off + ca]); b[u] = to_f32(x[off + cb]);
        const float da = to_f32(dy[off + ca]), db = to_f32(dy[off + cb]);
        const Turn r = turn_of(at, t, i);
        ga[u] = da * r.c + db * r.s;                   // turned back
        gb[u] = db * r.c - da * r.s;
      }
      float mean = 0.f, sq = 0.f;
      if constexpr (NORM == MOSAIC_LAYERNORM) mean = wave_sum(a[0] + b[0] + a[1] + b[1]) / (float)d;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < half) { a[u] -= mean; b[u] -= mean; sq += a[u] * a[u] + b[u] * b[u]; }
      const float rstd = 1.f / sqrtf(wave_sum(sq) / (float)d + eps);
      const T* g = head < H ? gq : gk;
      const int set = head < H ? 0 : 1;
      float wsum = 0.f, wx = 0.f, wa[2] = {0.f, 0.f}, wb[2] = {0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = lane + 64 * u;
        if (i >= half) continue;
        a[u] *= rstd; b[u] *= rstd;
        wa[u] = ga[u] * to_f32(g[first_of<HALVES>(i)]);
        wb[u] = gb[u] * to_f32(g[second_of<HALVES>(i, half)]);
        wsum += wa[u] + wb[u];
        wx += wa[u] * a[u] + wb[u] * b[u];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          acc[k][u][0] += k == set ? ga[u] * a[u] : 0.f;
          acc[k][u][1] += k == set ? gb[u] * b[u] : 0.f;
          acc[k][u][2] += k == set ? ga[u] : 0.f;
          acc[k][u][3] += k == set ? gb[u] : 0.f;
        }
      }
      const float mw = NORM == MOSAIC_LAYERNORM ? wave_sum(wsum) / (float)d : 0.f, mx = wave_sum(wx) / (float)d;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = lane + 64 * u;
        if (i >= half) continue;
        dx[off + first_of<HALVES>(i)] = from_f32<T>(rstd * (wa[u] - mw - a[u] * mx));
        dx[off + second_of<HALVES>(i, half)] = from_f32<T>(rstd * (wb[u] - mw - b[u] * mx));
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = lane + 64 * u;
        if (i >= half) continue;
        const int ca = first_of<HALVES>(i), cb = second_of<HALVES>(i, half);
        sums[wave][k * d + ca] = acc[k][u][0];
        sums[wave][k * d + cb] = acc[k][u][1];
        sums[wave][(2 + k) * d + ca] = acc[k][u][2];
        sums[wave][(2 + k) * d + cb] = acc[k][u][3];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < 4 * d; c += kThreads) {
      float v = sums[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += sums[w][c];
      partial[(int64_t)p * 4 * d + c] = v;
    }
    __syncthreads();
  }
}

}  // namespace

size_t rope_axes_table_bytes(int d) { return (size_t)(d / 2) * sizeof(PairTurn); }

mosaic_status launch_rope_axes_table(hipStream_t s, int quota, int d, int n_axes, const int32_t* sections, int order, float base, void* table) {
  Sections n = {};
  for (int a = 0; a < n_axes; ++a) n.n[a] = sections[a];
  axes_table_kernel<<<grid_for(quota, 8, ceil_div(d / 2, kThreads)), kThreads, 0, s>>>((PairTurn*)table, d / 2, n_axes, n, order, (double)base);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

size_t qk_norm_rope_bwd_scratch_bytes(int d) { return (size_t)kMaxParts * 4 * d * sizeof(float); }

mosaic_status launch_qk_norm_rope_fwd(hipStream_t s, int quota, int dtype, int norm, int64_t T, int H, int Hkv, int d, float eps, int pairing, int direction,
                                      int n_axes, const int32_t* pos, const void* table, const void* x, const void* gq, const void* bq,
                                      const void* gk, const void* bk, void* y) {
  const int heads = H + Hkv + (x == y ? 0 : Hkv);      // in place, v lies where it should
  const Positions at = {pos, (const PairTurn*)table, T, n_axes};
  if (T > 0) {
    const int grid = grid_for(quota, 8, ceil_div(T * heads, kWaves));
    auto launch = [&](auto type, auto kind, auto halves) {
      typedef decltype(type) E;
      qk_fwd_any_kernel<E, decltype(kind)::value, decltype(halves)::value><<<grid, kThreads, 0, s>>>(
          (const E*)x, (E*)y, at, H, Hkv, d, heads, eps, (float)direction, (const E*)gq, (const E*)bq, (const E*)gk, (const E*)bk);
    };
    auto of_norm = [&](auto type, auto halves) {
      if (norm == MOSAIC_RMSNORM) launch(type, std::integral_constant<int, MOSAIC_RMSNORM>{}, halves);
      else if (norm == MOSAIC_LAYERNORM) launch(type, std::integral_constant<int, MOSAIC_LAYERNORM>{}, halves);
      else launch(type, std::integral_constant<int, MOSAIC_NORM_NONE>{}, halves);
    };
    auto of_type = [&](auto type) { if (pairing == MOSAIC_PAIR_HALVES) of_norm(type, std::true_type{}); else of_norm(type, std::false_type{}); };
    if (dtype == MOSAIC_BF16) of_type(bf16{}); else of_type(float{});
    MOSAIC_LAUNCH_CHECK();
  }
  return MOSAIC_OK;
}

mosaic_status launch_qk_norm_rope_bwd(hipStream_t s, int quota, int dtype, int norm, int64_t T, int H, int Hkv, int d, float eps, int pairing, int n_axes,
                                      const int32_t* pos, const void* table, const void* x, const void* gq, const void* gk, const void* dy, void* dx,
                                      void* dgq, void* dbq, void* dgk, void* dbk, void* scratch) {
  const int heads = H + Hkv + (dx == dy ? 0 : Hkv);
  const Positions at = {pos, (const PairTurn*)table, T, n_axes};
  // Partitions by the number of tokens alone: the sums' order, and so their bits, do not depend on the quota.
  const int rp = (int)std::max<int64_t>(kWaves, ceil_div(T, kMaxParts)), np = (int)ceil_div(T, rp);
  if (T > 0) {
    const int grid = grid_for(quota, 4, np);
    auto launch = [&](auto type, auto kind, auto halves) {
      typedef decltype(type) E;
      qk_bwd_any_kernel<E, decltype(kind)::value, decltype(halves)::value><<<grid, kThreads, 0, s>>>(
          (const E*)x, (const E*)dy, (E*)dx, at, H, Hkv, d, heads, eps, (const E*)gq, (const E*)gk, (float*)scratch, rp, np);
    };
    auto of_norm = [&](auto type, auto halves) {
      if (norm == MOSAIC_RMSNORM) launch(type, std::integral_constant<int, MOSAIC_RMSNORM>{}, halves);
      else launch(type, std::integral_constant<int, MOSAIC_LAYERNORM>{}, halves);
    };
    auto of_type = [&](auto type) { if (pairing == MOSAIC_PAIR_HALVES) of_norm(type, std::true_type{}); else of_norm(type, std::false_type{}); };
    if (dtype == MOSAIC_BF16) of_type(bf16{}); else of_type(float{});
    MOSAIC_LAUNCH_CHECK();
  }
  const float* partial = (const float*)scratch;
  ColReduceList list;
  list.job[list.n++] = {partial, np, 4 * (int64_t)d, 2 * (int64_t)d, d, INT64_MAX, dgq, dgk, nullptr};
  if (norm == MOSAIC_LAYERNORM) list.job[list.n++] = {partial + 2 * d, np, 4 * (int64_t)d, 2 * (int64_t)d, d, INT64_MAX, dbq, dbk, nullptr};
  return launch_col_reduce(s, quota, dtype, list);
}
