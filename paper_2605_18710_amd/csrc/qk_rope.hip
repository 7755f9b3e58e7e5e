// What lies between a layer's QKV product and its attention in models that see images and video: a norm over every query
// and key head, then a rotation whose position has several axes, on packed rows [q (H heads) | k (Hkv heads) | v (Hkv heads)].
//
//   xhat = (x - mean) * rstd (mean = 0 for RMS norms), n = gain * xhat + shift, y = R n
//   backward: g = R^T dy, dgain = sum g * xhat, dshift = sum g, w = gain * g, dx = rstd * (w - mean(w) [LayerNorm] - xhat * mean(w * xhat))
//
// R turns pair i of a head by position[axis(i)] * frequency(i).  The angle is formed in double as a number of turns, whose
// whole part is dropped there: a position of any int32 keeps its digits.  rstd is formed again in the backward pass, which reads x anyway.
#include <algorithm>
#include <initializer_list>
#include <math.h>
#include "kernels.h"
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kThreadsBwd = 512;
constexpr int kWavesBwd = kThreadsBwd / 64;
constexpr int kMaxD = 256;
constexpr int kMaxParts = 512;      // partitions of the gains' gradients
constexpr int kMaxAxes = MOSAIC_MAX_AXES;

// one pair of a head: turns (of 2 pi) for each unit of position on its axis; axis -1: the pair stays
struct PairTurn {
  double turns;
  int axis, unused;
};
static_assert(kMaxAxes == 4, "positions are chosen from four");
static_assert(sizeof(PairTurn) == 16, "an entry of the table");

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

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

// The sum over the LPH lanes of a head, in every one of them: up to 16 lanes by moves within a row of 16 (DPP), which need no LDS.
// Each step adds the same two numbers in both lanes, so all lanes hold the same bits.
template <int CTRL> __device__ __forceinline__ float from_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LPH> __device__ __forceinline__ float head_sum(float v) {
  if constexpr (LPH >= 2) v += from_lane<0xb1>(v);        // neighbours
  if constexpr (LPH >= 4) v += from_lane<0x4e>(v);        // pairs of a quad
  if constexpr (LPH >= 8) v += from_lane<0x141>(v);       // mirrored within 8
  if constexpr (LPH >= 16) v += from_lane<0x140>(v);      // mirrored within 16
  if constexpr (LPH >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}

// A lane's share of a head: VE elements from ca on and as many from cb = ca + d/2 on, VE whole pairs in either form; LPH lanes (a power of two, the
// last of them idle where d / (2 VE) is none) hold a head, 64 / LPH heads a wave.
template <typename T, int VE, int LPH, bool HALVES> struct Share {
  typedef typename Pack<T, VE>::type vec;
  static constexpr int kHeads = 64 / LPH;
  int half, ca, cb, slot;
  // Bytes of the lane's vectors from a row's first head on.  Rows are read and written through descriptors that end with their heads: lanes behind the
  // last head, and idle ones, read zeros and write nothing, with no branch and no address of their own.
  uint32_t la, lb, step;
  bool active;
  __device__ __forceinline__ explicit Share(int d) {
    const int lane = threadIdx.x & 63;
    half = d / 2;
    ca = lane % LPH * VE;
    cb = ca + half;
    slot = lane / LPH;
    active = ca < half;
    la = active ? (uint32_t)(slot * d + ca) * (uint32_t)sizeof(T) : 0x80000000u;
    lb = la + (uint32_t)half * (uint32_t)sizeof(T);
    step = (uint32_t)(kHeads * d) * (uint32_t)sizeof(T);
  }
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t row(const T* p, int heads, int d) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0, heads * d * (int)sizeof(T), 0x00020000);
  }
  template <bool PAST> static __device__ __forceinline__ vec get(__amdgpu_buffer_rsrc_t row, uint32_t at) {
    if constexpr (sizeof(vec) == 16) return __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b128(row, (int)at, 0, PAST ? 2 : 0));
    else return __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b64(row, (int)at, 0, PAST ? 2 : 0));
  }
  template <bool PAST> static __device__ __forceinline__ void put(__amdgpu_buffer_rsrc_t row, uint32_t at, vec v) {
    if constexpr (sizeof(vec) == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), row, (int)at, 0, PAST ? 2 : 0);
    else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), row, (int)at, 0, PAST ? 2 : 0);
  }
  // The token's turns: each pair's by one lane, through LDS that only this wave uses.
  __device__ __forceinline__ void turns(const Positions& at, const PairTurn (&mine)[2], int64_t t, Turn* lds, float (&c)[VE], float (&s)[VE]) const {
    int pos[kMaxAxes];                                   // wave-wide, and asked for without waiting for the table
#pragma unroll
    for (int a = 0; a < kMaxAxes; ++a) pos[a] = at.pos[min(a, at.n_axes - 1) * at.T + t];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = (threadIdx.x & 63) + 64 * u;
      if (i < half) {
        Turn r = {1.f, 0.f};
        if (mine[u].axis >= 0) {
          const int axis = mine[u].axis;
          double turns = (double)(axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : pos[3]) * mine[u].turns;
          turns -= rint(turns);
          sincospif(2.f * (float)turns, &r.s, &r.c);
        }
        lds[i] = r;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const Turn r = active ? lds[HALVES ? ca + e : e < VE / 2 ? ca / 2 + e : cb / 2 + e - VE / 2] : Turn{1.f, 0.f};
      c[e] = r.c;
      s[e] = r.s;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();                     // the next token's turns are written behind these reads
  }
  // (a, b) turned by +s or, given negative s, back
  static __device__ __forceinline__ void rotate(float (&a)[VE], float (&b)[VE], const float (&c)[VE], const float (&s)[VE]) {
    if constexpr (HALVES) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float x = a[e], y = b[e];
        a[e] = x * c[e] - y * s[e];
        b[e] = x * s[e] + y * c[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < VE / 2; ++e) {
        const float x = a[2 * e], y = a[2 * e + 1], z = b[2 * e], w = b[2 * e + 1];
        a[2 * e] = x * c[e] - y * s[e];
        a[2 * e + 1] = x * s[e] + y * c[e];
        b[2 * e] = z * c[VE / 2 + e] - w * s[VE / 2 + e];
        b[2 * e + 1] = z * s[VE / 2 + e] + w * c[VE / 2 + e];
      }
    }
  }
  __device__ __forceinline__ void own_pairs(const Positions& at, PairTurn (&mine)[2]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = (threadIdx.x & 63) + 64 * u;
      mine[u] = {0.0, -1, 0};
      if (at.table && i < half) mine[u] = at.table[i];
      if (mine[u].axis >= at.n_axes) mine[u].axis = -1;
    }
  }
};

// Rows of whole vectors: a wave takes a token (of few tokens, `per_chunk` of its groups of heads), its lanes 64 / LPH heads at a time.
// Bound by memory: 32768 tokens, 32 + 8 + 8 heads of 128, bf16, RMS norm 139 us (5.8 TB/s; a wave per head and pair by pair 558), on 64 CUs 294; 12000 tokens, 20 heads
// of 64, fp32, LayerNorm 71 (5.2).  Two tokens a wave, one after the other, 148.  Few tokens are a chain of latencies: 24 tokens 3.8 us.
template <typename T, int VE, int LPH, int NORM, bool HALVES, bool PAST>
__global__ __launch_bounds__(kThreads) void qk_fwd_kernel(const T* x, T* y, Positions at, int H, int Hkv, int d, int heads, int per_chunk, int chunks,
                                                          float eps, float sign, const T* __restrict__ gq, const T* __restrict__ bq,
                                                          const T* __restrict__ gk, const T* __restrict__ bk) {
  typedef Share<T, VE, LPH, HALVES> S;
  typedef typename S::vec vec;
  __shared__ Turn lds[kWaves][kMaxD / 2];
  const S sh(d);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), groups = (heads + S::kHeads - 1) / S::kHeads;
  const int64_t width = (int64_t)(H + 2 * Hkv) * d, items = at.T * chunks;
  const float inv_d = 1.f / (float)d;
  PairTurn mine[2];
  sh.own_pairs(at, mine);
  vec ga[2] = {}, gb[2] = {}, sa[2] = {}, sb[2] = {};        // gains and shifts of q and k
  if constexpr (NORM != MOSAIC_NORM_NONE) {
    if (sh.active) {
      ga[0] = *(const vec*)(gq + sh.ca); gb[0] = *(const vec*)(gq + sh.cb);
      ga[1] = *(const vec*)(gk + sh.ca); gb[1] = *(const vec*)(gk + sh.cb);
      if constexpr (NORM == MOSAIC_LAYERNORM) {
        sa[0] = *(const vec*)(bq + sh.ca); sb[0] = *(const vec*)(bq + sh.cb);
        sa[1] = *(const vec*)(bk + sh.ca); sb[1] = *(const vec*)(bk + sh.cb);
      }
    }
  }
  float c[VE], s[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) { c[e] = 1.f; s[e] = 0.f; }
  for (int64_t item = (int64_t)blockIdx.x * kWaves + wave; item < items; item += (int64_t)gridDim.x * kWaves) {
    const int64_t t = chunks == 1 ? item : item / chunks;
    const int g0 = chunks == 1 ? 0 : (int)(item - t * chunks) * per_chunk, g1 = chunks == 1 ? groups : min(g0 + per_chunk, groups);
    const auto in = S::row(x + t * width, heads, d), out = S::row(y + t * width, heads, d);
    auto load = [&](int g, vec& a, vec& b) {
      a = S::template get<PAST>(in, sh.la + g * sh.step);
      b = S::template get<PAST>(in, sh.lb + g * sh.step);
    };
    vec na, nb;
    load(g0, na, nb);
    if (at.table) {
      sh.turns(at, mine, t, lds[wave], c, s);
#pragma unroll
      for (int e = 0; e < VE; ++e) s[e] *= sign;
    }
    for (int g = g0; g < g1; ++g) {
      vec va = na, vb = nb;
      if (g + 1 < g1) load(g + 1, na, nb);
      const int head = g * S::kHeads + sh.slot;
      if (g * S::kHeads < H + Hkv) {                     // the group has more than v
        float a[VE], b[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) { a[e] = (float)va[e]; b[e] = (float)vb[e]; }
        if constexpr (NORM != MOSAIC_NORM_NONE) {
          if constexpr (NORM == MOSAIC_LAYERNORM) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e) sum += a[e] + b[e];
            sum = head_sum<LPH>(sum) * inv_d;             // every lane takes part
            const float mean = sh.active ? sum : 0.f;
#pragma unroll
            for (int e = 0; e < VE; ++e) { a[e] -= mean; b[e] -= mean; }
          }
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < VE; ++e) sq += a[e] * a[e] + b[e] * b[e];
          const float rstd = rsqrtf(head_sum<LPH>(sq) * inv_d + eps);
          const int part = head < H ? 0 : 1;
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            a[e] = a[e] * rstd * (part ? (float)ga[1][e] : (float)ga[0][e]);
            b[e] = b[e] * rstd * (part ? (float)gb[1][e] : (float)gb[0][e]);
            if constexpr (NORM == MOSAIC_LAYERNORM) {
              a[e] += part ? (float)sa[1][e] : (float)sa[0][e];
              b[e] += part ? (float)sb[1][e] : (float)sb[0][e];
            }
          }
        }
        S::rotate(a, b, c, s);
        if (head < H + Hkv) {
#pragma unroll
          for (int e = 0; e < VE; ++e) { va[e] = (T)a[e]; vb[e] = (T)b[e]; }
        }
      }
      S::template put<PAST>(out, sh.la + g * sh.step, va);
      S::template put<PAST>(out, sh.lb + g * sh.step, vb);
    }
  }
}

// The backward pass of rows of whole vectors.  A workgroup takes one part (q, k or, to be copied, v) of a partition of the tokens, its waves every
// (np kWavesBwd)-th token each, so that what the workgroups in flight touch lies side by side.
// A lane holds its columns' sums of the part's gains' (and shifts') gradients, which are joined over the wave's heads and then over the waves, in order.
// Bound by memory and, about as much, by vector instructions (some 25 an element): 32768 tokens, 32 + 8 + 8 heads of 128, bf16, RMS norm 231 us (4.9 TB/s), on 64
// CUs 500, and 5 for the last reduction; 12000 tokens, 20 heads of 64, fp32, LayerNorm 94; bf16 LayerNorm 59, 4096 tokens of 40 + 8 + 8 heads of 72 27.  Workgroups of 256 threads 250, of 640 245, of 1024 241 us; q and k in one
// loop with sums of both 250; partitions of consecutive tokens 260.
template <typename T, int VE, int LPH, int NORM, bool HALVES, bool PAST>
__global__ __launch_bounds__(kThreadsBwd) void qk_bwd_kernel(const T* __restrict__ x, const T* dy, T* dx, Positions at, int H, int Hkv, int d, int parts, float eps,
                                                             const T* __restrict__ gq, const T* __restrict__ gk, float* __restrict__ partial, int np) {
  typedef Share<T, VE, LPH, HALVES> S;
  typedef typename S::vec vec;
  constexpr bool LN = NORM == MOSAIC_LAYERNORM;
  constexpr int kSets = LN ? 2 : 1;                     // gains; shifts
  __shared__ Turn lds[kWavesBwd][kMaxD / 2];
  __shared__ float sums[kWavesBwd][kSets * kMaxD];
  const S sh(d);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t width = (int64_t)(H + 2 * Hkv) * d, stride = (int64_t)np * kWavesBwd;
  const float inv_d = 1.f / (float)d;
  PairTurn mine[2];
  sh.own_pairs(at, mine);
  float c[VE], s[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) { c[e] = 1.f; s[e] = 0.f; }
  for (int item = blockIdx.x; item < parts * np; item += gridDim.x) {
    const int part = item / np, p = item - part * np;
    const int64_t t0 = (int64_t)p * kWavesBwd + wave;
    if (part == 2) {
      const int nv = Hkv * d / VE;
      for (int64_t t = t0; t < at.T; t += stride) {
        const int64_t first = t * width + (int64_t)(H + Hkv) * d;
        const auto grad = S::row(dy + first, Hkv, d), out = S::row(dx + first, Hkv, d);
        for (int i = lane; i < nv; i += 64) S::template put<PAST>(out, (uint32_t)i * (uint32_t)sizeof(vec), S::template get<PAST>(grad, (uint32_t)i * (uint32_t)sizeof(vec)));
      }
      continue;
    }
    const int heads = part ? Hkv : H, groups = (heads + S::kHeads - 1) / S::kHeads;
    const T* gain = part ? gk : gq;
    float ga[VE], gb[VE];
    {
      vec va = {}, vb = {};
      if (sh.active) { va = *(const vec*)(gain + sh.ca); vb = *(const vec*)(gain + sh.cb); }
#pragma unroll
      for (int e = 0; e < VE; ++e) { ga[e] = (float)va[e]; gb[e] = (float)vb[e]; }
    }
    float acc[kSets][2][VE] = {};                     // [gain or shift][a or b]
#pragma unroll 1
    for (int64_t t = t0; t < at.T; t += stride) {
      struct Req { vec xa, xb, da, db; };
      const int64_t first = t * width + (part ? (int64_t)H * d : 0);
      const auto rows = S::row(x + first, heads, d), grad = S::row(dy + first, heads, d), out = S::row(dx + first, heads, d);
      auto load = [&](int g, Req& r) {
        r.xa = S::template get<PAST>(rows, sh.la + g * sh.step);
        r.xb = S::template get<PAST>(rows, sh.lb + g * sh.step);
        r.da = S::template get<PAST>(grad, sh.la + g * sh.step);
        r.db = S::template get<PAST>(grad, sh.lb + g * sh.step);
      };
      Req next;
      load(0, next);
      if (at.table) {
        sh.turns(at, mine, t, lds[wave], c, s);
#pragma unroll
        for (int e = 0; e < VE; ++e) s[e] = -s[e];
      }
#pragma unroll 1
      for (int g = 0; g < groups; ++g) {
        const Req r = next;
        if (g + 1 < groups) load(g + 1, next);
        float a[VE], b[VE], da[VE], db[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) { a[e] = (float)r.xa[e]; b[e] = (float)r.xb[e]; da[e] = (float)r.da[e]; db[e] = (float)r.db[e]; }
        if constexpr (LN) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < VE; ++e) sum += a[e] + b[e];
          sum = head_sum<LPH>(sum) * inv_d;
          const float mean = sh.active ? sum : 0.f;
#pragma unroll
          for (int e = 0; e < VE; ++e) { a[e] -= mean; b[e] -= mean; }
        }
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) sq += a[e] * a[e] + b[e] * b[e];
        const float rstd = rsqrtf(head_sum<LPH>(sq) * inv_d + eps);
        S::rotate(da, db, c, s);
        float wsum = 0.f, wx = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) {                // lanes without a head hold zeros and add nothing
          a[e] *= rstd; b[e] *= rstd;
          acc[0][0][e] += da[e] * a[e]; acc[0][1][e] += db[e] * b[e];
          if constexpr (LN) { acc[1][0][e] += da[e]; acc[1][1][e] += db[e]; }
          da[e] *= ga[e]; db[e] *= gb[e];
          if constexpr (LN) wsum += da[e] + db[e];
          wx += da[e] * a[e] + db[e] * b[e];
        }
        const float mx = head_sum<LPH>(wx) * inv_d, mw = LN ? head_sum<LPH>(wsum) * inv_d : 0.f;
        vec oa, ob;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          oa[e] = (T)(rstd * (da[e] - mw - a[e] * mx));
          ob[e] = (T)(rstd * (db[e] - mw - b[e] * mx));
        }
        S::template put<PAST>(out, sh.la + g * sh.step, oa);
        S::template put<PAST>(out, sh.lb + g * sh.step, ob);
      }
    }
#pragma unroll
    for (int set = 0; set < kSets; ++set)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        float va = acc[set][0][e], vb = acc[set][1][e];
#pragma unroll
        for (int o = LPH; o < 64; o <<= 1) { va += __shfl_xor(va, o, 64); vb += __shfl_xor(vb, o, 64); }
        if (sh.active && sh.slot == 0) {
          sums[wave][set * d + sh.ca + e] = va;
          sums[wave][set * d + sh.cb + e] = vb;
        }
      }
    __syncthreads();
    for (int col = threadIdx.x; col < kSets * d; col += kThreadsBwd) {
      float v = sums[0][col];
#pragma unroll
      for (int w = 1; w < kWavesBwd; ++w) v += sums[w][col];
      const int set = col >= d ? 1 : 0;
      partial[(int64_t)p * 4 * d + (2 * set + part) * d + col - set * d] = v;
    }
    __syncthreads();
  }
}

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

// Past the caches what they do not hold, where a half of a head is whole lines of 128 bytes: a lane's two vectors lie half a head apart, and parts of lines go
// past the caches one by one.  bf16, 32768 tokens of 48 heads of 128: forward 150 -> 139 us, backward 251 -> 237; 36864 tokens of 48 heads of 64 85 -> 94.
template <typename T> bool past_caches(int d, int64_t bytes) { return bytes > kPastCacheBytes && d / 2 * (int)sizeof(T) % 128 == 0; }

// launch(elements of a vector, lanes of a head) where each half of a head is whole vectors and all addresses lie on them.  kBytes: of a vector of bf16; 8 where
// d is no multiple of 16.  The backward pass takes 8 everywhere: with 16 a lane's sums and values leave room for half the waves (12000 tokens, 20 heads
// of 64, LayerNorm 83 us, with 8 62; 32768 tokens of 32 + 8 heads of 128 232 and 237, on 64 CUs 574 and 505).  Forward 16 / 8: 139 / 146 us.
template <typename T, int kBytes, typename F> bool with_vectors(int64_t width, int d, std::initializer_list<const void*> pointers, F launch) {
  constexpr int kWide = (kBytes < 16 && sizeof(T) == 2 ? 8 : 16) / (int)sizeof(T);
  uintptr_t bits = 0;
  for (const void* p : pointers) bits |= (uintptr_t)p;
  if (width * (int64_t)sizeof(T) > (int64_t)1 << 30) return false;      // descriptors and offsets of 32 bits
  auto of_lanes = [&](auto ve) {
    const int lanes = d / (2 * decltype(ve)::value);
    if (lanes <= 2) launch(ve, std::integral_constant<int, 2>{});
    else if (lanes <= 4) launch(ve, std::integral_constant<int, 4>{});
    else if (lanes <= 8) launch(ve, std::integral_constant<int, 8>{});
    else if (lanes <= 16) launch(ve, std::integral_constant<int, 16>{});
    else if constexpr (decltype(ve)::value * 2 * 16 < kMaxD) launch(ve, std::integral_constant<int, 32>{});
  };
  if (d % (2 * kWide) == 0 && bits % (kWide * sizeof(T)) == 0) { of_lanes(std::integral_constant<int, kWide>{}); return true; }
  if (kWide > 4 && d % 8 == 0 && bits % 8 == 0) { of_lanes(std::integral_constant<int, 4>{}); return true; }
  return false;
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
    auto launch = [&](auto type, auto kind, auto halves) {
      typedef decltype(type) E;
      const bool vectors = with_vectors<E, 16>((int64_t)(H + 2 * Hkv) * d, d, {x, y, gq, gk, bq, bk}, [&](auto ve, auto lph) {
        constexpr int VE = decltype(ve)::value, LPH = decltype(lph)::value;
        const int groups = (int)ceil_div(heads, 64 / LPH);
        // Few tokens: their groups of heads apart, as far as there are waves for them (32 + 8 + 8 heads of 128, 1 token 4.3 -> 3.1 us, 200 tokens 4.9 -> 3.8).  In
        // order from 64 MB on (striding / in order: 805 MB 152 / 139 us, 453 MB 90 / 85, 113 MB 25.3 / 26.2, 100 MB 22.6 / 23.0; on 64 CUs 805 MB 324 / 294).
        const int chunks = (int)std::min<int64_t>(groups, std::max<int64_t>(1, (int64_t)quota * 8 / T)), per_chunk = (int)ceil_div(groups, chunks);
        const int64_t items = T * ceil_div(groups, per_chunk), bytes = 2 * T * heads * d * (int64_t)sizeof(E);
        const Sweep sw = sweep_grid(s, quota, ceil_div(items, kWaves), bytes);
        auto with = [&](auto past) {
          qk_fwd_kernel<E, VE, LPH, decltype(kind)::value, decltype(halves)::value, decltype(past)::value><<<sw.grid, kThreads, 0, s>>>(
              (const E*)x, (E*)y, at, H, Hkv, d, heads, per_chunk, (int)ceil_div(groups, per_chunk), eps, (float)direction,
              (const E*)gq, (const E*)bq, (const E*)gk, (const E*)bk);
        };
        if constexpr (VE * LPH * sizeof(E) >= 128) {       // a half of a head may be whole lines
          if (sw.in_order && past_caches<E>(d, bytes)) return with(std::true_type{});
        }
        with(std::false_type{});
      });
      if (vectors) return;
      const int grid = grid_for(quota, 8, ceil_div(T * heads, kWaves));
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
  // Partitions by the number of tokens and the kernel alone: the sums' order, and so their bits, do not depend on the quota.
  int np = 0;
  if (T > 0) {
    auto launch = [&](auto type, auto kind, auto halves) {
      typedef decltype(type) E;
      const bool vectors = with_vectors<E, 8>((int64_t)(H + 2 * Hkv) * d, d, {x, dy, dx, gq, gk}, [&](auto ve, auto lph) {
        constexpr int VE = decltype(ve)::value, LPH = decltype(lph)::value;
        const int64_t bytes = T * (2 * heads + H + Hkv) * d * (int64_t)sizeof(E);
        const int parts = dx == dy ? 2 : 3;            // in place, v lies where it should
        // As many tokens for every wave, and of up to 8192 tokens no more than 256 partitions: a wave then starts, and adds up its sums, for two tokens
        // or more (512 / 256: 8192 tokens of 16 + 4 heads of 128 38.3 / 33.5 us, 4096 of 40 + 8 heads of 72 33.9 / 30.5; 12000 of 20 heads of 64 62.9 / 64.6).
        const int64_t each = ceil_div(T, (T <= 8192 ? kMaxParts / 2 : kMaxParts) * (int64_t)kWavesBwd);
        np = (int)ceil_div(T, each * kWavesBwd);
        const int grid = grid_for(quota, 4, (int64_t)parts * np);
        auto with = [&](auto past) {
          qk_bwd_kernel<E, VE, LPH, decltype(kind)::value, decltype(halves)::value, decltype(past)::value><<<grid, kThreadsBwd, 0, s>>>(
              (const E*)x, (const E*)dy, (E*)dx, at, H, Hkv, d, parts, eps, (const E*)gq, (const E*)gk, (float*)scratch, np);
        };
        if constexpr (VE * LPH * sizeof(E) >= 128) {
          if (past_caches<E>(d, bytes)) return with(std::true_type{});
        }
        with(std::false_type{});
      });
      if (vectors) return;
      const int rp = (int)std::max<int64_t>(kWaves, ceil_div(T, kMaxParts));
      np = (int)ceil_div(T, rp);
      qk_bwd_any_kernel<E, decltype(kind)::value, decltype(halves)::value><<<grid_for(quota, 4, np), kThreads, 0, s>>>(
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
