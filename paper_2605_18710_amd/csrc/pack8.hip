// Activations kept in 8 bits between the forward and the backward pass, and the backward kernels that read them.
//
// A block of 32 consecutive elements has one exponent e, the smallest from -127 on with max |x| <= 127.5 * 2^e, kept as the byte e + 127, and the
// whole numbers q nearest to x / 2^e (ties to even, at most 127 in size): an element is off by half of 2^e at most, and
// q * 2^e is a bf16 number, so that unpacking rounds nothing.  x / 2^e is exact too: the bits do not depend on how it is computed.  A block
// with a NaN or an infinity has the byte 255 and comes back as NaN.
#include <initializer_list>
#include <type_traits>
#include "kernels.h"
#include "activations.h"
#include "pack8.h"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;

// `top`: bits of the block's largest magnitude
__device__ __forceinline__ int scale_byte(unsigned top) {
  if (top >= 0x7f800000u) return 255;
  const int e = (int)(top >> 23) - 6 + ((top & 0x7fffffu) > 0x7f0000u);     // exponent byte of e; 127.5 = 1.9921875 * 2^6
  return e < 0 ? 0 : e;
}
__device__ __forceinline__ float inverse_step(int byte) {     // 2^-e; e is 122 at most (a NaN's numbers are 0)
  return __uint_as_float(byte == 255 ? 0u : (unsigned)(254 - byte) << 23);
}
__device__ __forceinline__ int packed(float x, float inverse) {
  const float v = rintf(x * inverse);
  return v != v ? 0 : (int)fminf(fmaxf(v, -127.f), 127.f);
}

// Eight consecutive elements in fp32: 16 bytes of bf16, 32 of fp32.
template <bool PAST> __device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
  Vec16<bf16> x;
  x.load<PAST>(p);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = x.get(k);
}
template <bool PAST> __device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  Vec16<float> x, y;
  x.load<PAST>(p);
  y.load<PAST>(p + 4);
#pragma unroll
  for (int k = 0; k < 4; ++k) { v[k] = x.get(k); v[4 + k] = y.get(k); }
}
template <bool PAST> __device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  Vec16<bf16> x;
#pragma unroll
  for (int k = 0; k < 8; ++k) x.set(k, v[k]);
  x.store<PAST>(p);
}
template <bool PAST> __device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  Vec16<float> x, y;
#pragma unroll
  for (int k = 0; k < 4; ++k) { x.set(k, v[k]); y.set(k, v[4 + k]); }
  x.store<PAST>(p);
  y.store<PAST>(p + 4);
}
// the same, of an array that ends within the eight
template <bool PAST, typename T> __device__ __forceinline__ void load8(const T* p, int64_t left, float (&v)[8]) {
  if (left >= 8) return load8<PAST>(p, v);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = k < left ? to_f32(p[k]) : 0.f;
}
template <bool PAST, typename T> __device__ __forceinline__ void store8(T* p, int64_t left, const float (&v)[8]) {
  if (left >= 8) return store8<PAST>(p, v);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < left) p[k] = from_f32<T>(v[k]);
}

// Packs the eight elements of each of a block's four lanes (a quad): its exponent byte, and the numbers in two words.  Within 127 the number added to
// 1.5 * 2^23 is rounded to a whole one, ties to even, and stands in the sum's low byte.
__device__ __forceinline__ int pack_quad(const float (&v)[8], u32x2* q) {
  unsigned top = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
  top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));
  top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));
  const int byte = scale_byte(top);
  const float inverse = inverse_step(byte);
  unsigned w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = __float_as_uint(__builtin_amdgcn_fmed3f(v[4 * h + k] * inverse, -127.f, 127.f) + 12582912.f);
    const unsigned lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    w[h] = byte == 255 ? 0u : lo | hi;
  }
  *q = u32x2{w[0], w[1]};
  return byte;
}
__device__ __forceinline__ void put_tail(int8_t* p, int64_t left, u32x2 q) {
  for (int k = 0; k < 8; ++k)
    if (k < left) p[k] = (int8_t)((k < 4 ? q.x : q.y) >> (8 * (k & 3)));
}
__device__ __forceinline__ u32x2 get_tail(const int8_t* p, int64_t left) {
  u32x2 q = {0u, 0u};
  for (int k = 0; k < 8; ++k)
    if (k < left) { if (k < 4) q.x |= (unsigned)(uint8_t)p[k] << (8 * k); else q.y |= (unsigned)(uint8_t)p[k] << (8 * (k - 4)); }
  return q;
}

// 16-byte aligned arrays of any size: a lane takes eight elements, a quad of lanes a block.  `vectors`: eights, rounded up to whole blocks, so that a
// quad's lanes take part together.
template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads) void pack8_kernel(const T* __restrict__ x, int8_t* __restrict__ q, uint8_t* __restrict__ scale, int64_t n, int64_t vectors) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) {
    const int64_t left = n - i * 8;
    float v[8];
    load8<PAST>(x + i * 8, left, v);
    u32x2 w;
    const int byte = pack_quad(v, &w);
    if (left >= 8) store_to<PAST>((u32x2*)(q + i * 8), w);
    else put_tail(q + i * 8, left, w);
    if (i % 4 == 0) scale[i / 4] = (uint8_t)byte;
  }
}

template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads) void unpack8_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, T* __restrict__ x, int64_t n, int64_t vectors) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) {
    const int64_t left = n - i * 8;
    if (left <= 0) continue;
    const u32x2 w = left >= 8 ? load_from<PAST>((const u32x2*)(q + i * 8)) : get_tail(q + i * 8, left);
    float v[8];
    unpack8_of(w, scale[i / 4], v);
    store8<PAST>(x + i * 8, left, v);
  }
}

// any size and alignment: a thread takes an element, 32 lanes a block
template <typename T>
__global__ __launch_bounds__(kThreads) void pack8_any_kernel(const T* __restrict__ x, int8_t* __restrict__ q, uint8_t* __restrict__ scale, int64_t n, int64_t blocks) {
  const int lane = threadIdx.x & (kBlock - 1);
  for (int64_t b = (int64_t)blockIdx.x * (kThreads / kBlock) + threadIdx.x / kBlock; b < blocks; b += (int64_t)gridDim.x * (kThreads / kBlock)) {
    const int64_t i = b * kBlock + lane;
    const float v = i < n ? to_f32(x[i]) : 0.f;
    unsigned top = __float_as_uint(v) & 0x7fffffffu;
#pragma unroll
    for (int o = kBlock / 2; o > 0; o >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, o, kBlock));
    const int byte = scale_byte(top);
    if (i < n) q[i] = (int8_t)packed(v, inverse_step(byte));
    if (lane == 0) scale[b] = (uint8_t)byte;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void unpack8_any_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, T* __restrict__ x, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) x[i] = from_f32<T>((float)q[i] * step_of(scale[i / kBlock]));
}

// e = exp(-z) and s = 1 / (1 + e) of a gate z for results in bf16.  u = 2^-24, of the numbers' own size: the exponential of 2 is off by 2 u, the rest of its rounded
// argument, put right to first order, by 1 u and (for ln 2 in one piece) 1.9e-9 of the argument, 4 u at most: e 7 u, and s 2 u and (1 - s) times that.  A
// third of the instructions of expf and a divide.  s is the approximate reciprocal after one step of Newton's, which makes it the number that the divide gives: its
// last bits decide results that lie near a tie between two bf16 numbers, and of numbers from 8 bits, which repeat, those are many (16384 x 11008 SwiGLU formed
// again: without the step 2.4e-5 of the results were not the nearest number, with it and in the plain form 2.4e-6).
// 1 - s is e s (`rest`), which keeps its digits.  From -88.7 down s is 0 (the reciprocal drops denormal results), so that no size of z brings it back, and
// e stays finite for the step; a NaN reaches the results through the gate itself.
struct Gate {
  float e, s;
  __device__ __forceinline__ float rest() const { return e * s; }
};
__device__ __forceinline__ Gate gate_of(float z) {
  const float x = -__builtin_amdgcn_fmed3f(z, -88.7f, 126.f), hi = x * 1.44269504088896341f;
  const float p = __builtin_amdgcn_exp2f(hi), e = fmaf(p, fmaf(-hi, 0.693147180559945309f, x), p), d = 1.f + e, s = __builtin_amdgcn_rcpf(d);
  return {e, fmaf(s, fmaf(-d, s, 1.f), s)};
}
// The tanh form as a logistic function: (1 + tanh u) / 2 = 1 / (1 + exp(-2u)), which keeps its digits where tanh is near -1 and takes one exponential.
__device__ __forceinline__ float tanh_gelu_arg(float z) { return 1.5957691216057308f * (z + 0.044715f * z * z * z); }
// e = exp(-z^2 / 2) and the normal distribution's phi = (1 + erf(z / sqrt 2)) / 2 for results in bf16.  erf by Hastings' approximation (Abramowitz and Stegun,
// Handbook of Mathematical Functions, 7.1.26: 1 - (a1 t + .. + a5 t^5) exp(-x^2), t = 1 / (1 + p x), off by 1.5e-7), whose exponential GELU's derivative needs anyway:
// phi is off by 1.3 * 2^-24 for it and 3 * 2^-24 for roundings (of 1, not of its own size).  e's rounded argument w costs w exp(-w) * 2^-24, which never passes 0.37.
struct Normal { float e, phi; };
__device__ __forceinline__ Normal normal_of(float z) {
  const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3275911f * 0.70710678118654752f, 1.f));
  const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  const float tail = 0.5f * poly * e;                       // phi(-|z|)
  return {e, z < 0.f ? tail : 1.f - tail};
}
// act(z) and its derivative
template <typename T, int ACT> __device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == MOSAIC_GELU_TANH) return z * (sizeof(T) == 2 ? gate_of(tanh_gelu_arg(z)).s : sigmoid_f(tanh_gelu_arg(z)));
  else if constexpr (sizeof(T) == 2) return z * normal_of(z).phi;
  else return gelu_f(z);
}
template <typename T, int ACT> __device__ __forceinline__ float act_grad_of(float z) {
  if constexpr (ACT == MOSAIC_GELU_TANH) {
    // the argument's derivative; far out the logistic function's is 0, whatever size z has
    const float v = tanh_gelu_arg(z), near = __builtin_amdgcn_fmed3f(z, -1e6f, 1e6f), w = 1.5957691216057308f * (1.0f + 0.134145f * near * near);
    if constexpr (sizeof(T) == 2) {
      const Gate g = gate_of(v);
      return g.s * fmaf(z * g.rest(), w, 1.f);
    } else {                                              // e s is 1 - s with its digits: w z takes what a difference loses up to thirty times
      const float e = expf(-v), s = 1.0f / (1.0f + e);
      return s + z * (s * (fminf(e, 3e38f) * s)) * w;
    }
  } else if constexpr (sizeof(T) == 2) {
    const Normal n = normal_of(z);
    return fmaf(z * 0.39894228040143268f, n.e, n.phi);
  } else {
    return gelu_grad_f(z);
  }
}
template <typename T> __device__ __forceinline__ float glu_of(float gate, float up) {
  if constexpr (sizeof(T) == 2) return gate * gate_of(gate).s * up;
  else return swiglu_f(gate, up);
}
template <typename T> __device__ __forceinline__ void glu_grad_of(float gate, float up, float d, float* dgate, float* dup) {
  if constexpr (sizeof(T) == 2) {
    const Gate g = gate_of(gate);
    *dgate = d * up * (g.s * fmaf(gate, g.rest(), 1.f));
    *dup = d * (gate * g.s);
  } else {
    swiglu_grad_f(gate, up, d, dgate, dup);
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void act_fwd_any_kernel(const T* __restrict__ z, T* __restrict__ a, int64_t rows, int64_t f) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * f; i += (int64_t)gridDim.x * kThreads) {
    if constexpr (ACT == MOSAIC_SWIGLU) {
      const int64_t r = i / f, at = i + r * f;              // row r starts at 2 r f
      a[i] = from_f32<T>(glu_of<T>(to_f32(z[at]), to_f32(z[at + f])));
    } else {
      a[i] = from_f32<T>(act_of<T, ACT>(to_f32(z[i])));
    }
  }
}

// dz = act'(z) da and, where it is asked for, a = act(z), with z from its 8 bits
template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void act_bwd_any_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, const T* da, T* dz, T* __restrict__ a,
                                                               int64_t rows, int64_t f) {
  auto value = [&](int64_t i) { return (float)q[i] * step_of(scale[i / kBlock]); };
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * f; i += (int64_t)gridDim.x * kThreads) {
    const float d = to_f32(da[i]);
    if constexpr (ACT == MOSAIC_SWIGLU) {
      const int64_t r = i / f, at = i + r * f;
      const float gate = value(at), up = value(at + f);
      float dg, du;
      glu_grad_of<T>(gate, up, d, &dg, &du);
      dz[at] = from_f32<T>(dg);
      dz[at + f] = from_f32<T>(du);
      if (a) a[i] = from_f32<T>(glu_of<T>(gate, up));
    } else {
      const float z = value(i);
      dz[i] = from_f32<T>(d * act_grad_of<T, ACT>(z));
      if (a) a[i] = from_f32<T>(act_of<T, ACT>(z));
    }
  }
}

// (row, column) of the i-th eight of rows of fv eights
__device__ __forceinline__ void place(int64_t i, int64_t fv, int64_t* r, int64_t* c) {
  if ((uint64_t)(i | fv) >> 32 == 0) {                    // the same for all lanes but where an array passes 2^32 eights
    const uint32_t q = (uint32_t)i / (uint32_t)fv;
    *r = q;
    *c = (uint32_t)i - q * (uint32_t)fv;
  } else {
    *r = i / fv;
    *c = i - *r * fv;
  }
}

// Bound by memory: 16384 x 11008 SwiGLU 239 us forward (6.1 TB/s; 281 with expf and a divide for the gate) and 295 backward (6.2), 32768 x 5120 GELU 135 (6.2) and
// 185 (6.4; 236 with erf from a table in LDS, which keeps workgroups from starting in order).  fp32, with expf, erff and a divide: 9216 x 4096 GELU 64 (5.4) and
// 93 (5.3), its tanh form 67 (5.1) and 98 (5.0), 4096 x 5632 SwiGLU 58 (5.6) and 82 (5.1).
// a = act(z) and z in 8 bits.  GELU forms: flat, any size.  SwiGLU: rows of f = 8 fv, f a multiple of 32, so that no block has elements of both halves.
template <typename T, int ACT, bool PAST>
__global__ __launch_bounds__(kThreads) void act_fwd_kernel(const T* __restrict__ z, T* __restrict__ a, int8_t* __restrict__ q, uint8_t* __restrict__ scale,
                                                           int64_t n, int64_t vectors, int64_t fv) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) {
    float v[8], o[8];
    u32x2 w;
    if constexpr (ACT == MOSAIC_SWIGLU) {
      int64_t r, c;
      place(i, fv, &r, &c);
      const int64_t at = (r * 2 * fv + c) * 8, up = at + fv * 8;
      float u[8];
      load8<PAST>(z + at, v);
      load8<PAST>(z + up, u);
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = glu_of<T>(v[k], u[k]);
      store8<PAST>(a + i * 8, o);
      u32x2 wu;
      const int bg = pack_quad(v, &w), bu = pack_quad(u, &wu);
      store_to<PAST>((u32x2*)(q + at), w);
      store_to<PAST>((u32x2*)(q + up), wu);
      if (c % 4 == 0) { scale[at / kBlock] = (uint8_t)bg; scale[up / kBlock] = (uint8_t)bu; }
    } else {
      const int64_t left = n - i * 8;
      load8<PAST>(z + i * 8, left, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = act_of<T, ACT>(v[k]);
      store8<PAST>(a + i * 8, left, o);
      const int byte = pack_quad(v, &w);
      if (left >= 8) store_to<PAST>((u32x2*)(q + i * 8), w);
      else put_tail(q + i * 8, left, w);
      if (i % 4 == 0) scale[i / 4] = (uint8_t)byte;
    }
  }
}

// SwiGLU whose halves are no whole blocks (f = 8 fv): lanes walk z as it lies, and those of gate numbers ask for their up numbers too, which another
// workgroup packs and the caches hold.  8192 x 5608 75 us (activation and packing in a pass each 101; halves of whole blocks, 8192 x 5632, 61), 16384 x 11000 280 (373),
// 333 x 1000 4.2 (8.4); fp32 4096 x 5624 62 (82), but on 64 CUs 176 (168).
template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads) void swiglu_fwd_flat_kernel(const T* __restrict__ z, T* __restrict__ a, int8_t* __restrict__ q, uint8_t* __restrict__ scale,
                                                                   int64_t n, int64_t vectors, int64_t fv) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) {
    const bool any = i * 8 < n;                            // the last block's lanes take part together
    int64_t r, c;
    place(i, 2 * fv, &r, &c);
    float v[8] = {}, u[8], o[8];
    if (any) load8<false>(z + i * 8, v);
    if (any && c < fv) {
      load8<false>(z + (i + fv) * 8, u);
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = glu_of<T>(v[k], u[k]);
      store8<PAST>(a + (r * fv + c) * 8, o);
    }
    u32x2 w;
    const int byte = pack_quad(v, &w);
    if (any) store_to<PAST>((u32x2*)(q + i * 8), w);
    if (i % 4 == 0) scale[i / 4] = (uint8_t)byte;
  }
}

// dz = act'(z) da and, where asked for, a = act(z), with z from its 8 bits; SwiGLU: rows of f = 8 fv
template <typename T, int ACT, bool PAST, bool AGAIN>
__global__ __launch_bounds__(kThreads) void act_bwd_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, const T* da, T* dz, T* __restrict__ a,
                                                           int64_t n, int64_t vectors, int64_t fv) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += (int64_t)gridDim.x * kThreads) {
    float z[8], d[8], o[8];
    if constexpr (ACT == MOSAIC_SWIGLU) {
      int64_t r, c;
      place(i, fv, &r, &c);
      const int64_t at = (r * 2 * fv + c) * 8, up = at + fv * 8;
      float u[8], og[8], ou[8];
      const u32x2 wg = load_from<PAST>((const u32x2*)(q + at)), wu = load_from<PAST>((const u32x2*)(q + up));
      const int bg = scale[at / kBlock], bu = scale[up / kBlock];
      load8<PAST>(da + i * 8, d);
      unpack8_of(wg, bg, z);
      unpack8_of(wu, bu, u);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        glu_grad_of<T>(z[k], u[k], d[k], &og[k], &ou[k]);
        if constexpr (AGAIN) o[k] = glu_of<T>(z[k], u[k]);
      }
      store8<PAST>(dz + at, og);
      store8<PAST>(dz + up, ou);
      if constexpr (AGAIN) store8<PAST>(a + i * 8, o);
    } else {
      const int64_t left = n - i * 8;
      if (left <= 0) continue;
      const u32x2 w = left >= 8 ? load_from<PAST>((const u32x2*)(q + i * 8)) : get_tail(q + i * 8, left);
      const int byte = scale[i / 4];
      load8<PAST>(da + i * 8, left, d);
      unpack8_of(w, byte, z);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        d[k] *= act_grad_of<T, ACT>(z[k]);
        if constexpr (AGAIN) o[k] = act_of<T, ACT>(z[k]);
      }
      store8<PAST>(dz + i * 8, left, d);
      if constexpr (AGAIN) store8<PAST>(a + i * 8, left, o);
    }
  }
}

// Workgroups in order from 64 MB on (sweep_grid), striding / in order, us: 2^27 bf16 elements packed 76 / 73, unpacked 75 / 67; GELU of 12000 x 5120, forward 61 / 51
// and backward 84 / 68, on 64 CUs 182 / 153 and 206 / 166; SwiGLU of 8192 x 5632 72 / 61 and 89 / 76, of 2048 x 5632 (93 and 116 MB) 19.3 / 20.0 and
// 23.5 / 23.9, on 64 CUs 44.4 / 44.3 and 55.0 / 52.2.
// Past the caches what they do not hold, of bf16: 16384 x 11008 SwiGLU 270 us forward and 330 backward -> 240 and 294, on 64 CUs 648 and 778 -> 635 and 754,
// unpacking 2^27 elements 70 -> 67.  An fp32 lane's 32 bytes
// are two instructions' halves of a line, which past the caches are written one by one: unpacking 2^26 elements 61 us, past them 91.
template <typename T> bool past_caches(const Sweep& sw, int64_t bytes) { return sizeof(T) == 2 && sw.in_order && bytes > kPastCacheBytes; }

bool on16(std::initializer_list<const void*> pointers) {
  uintptr_t bits = 0;
  for (const void* p : pointers) bits |= (uintptr_t)p;
  return bits % 16 == 0;
}

}  // namespace

size_t pack8_scale_bytes(int64_t n) { return (size_t)ceil_div(n, kBlock); }

mosaic_status launch_pack8(hipStream_t s, int quota, int dtype, int64_t n, const void* x, void* q, void* scale) {
  if (n == 0) return MOSAIC_OK;
  const int64_t blocks = ceil_div(n, kBlock);
  auto launch = [&](auto type) {
    typedef decltype(type) E;
    if (!on16({x, q})) {
      pack8_any_kernel<E><<<grid_for(quota, 8, ceil_div(n, kThreads)), kThreads, 0, s>>>((const E*)x, (int8_t*)q, (uint8_t*)scale, n, blocks);
      return;
    }
    const int64_t vectors = blocks * (kBlock / 8), bytes = n * (int64_t)(sizeof(E) + 1);
    const Sweep sw = sweep_grid(s, quota, ceil_div(vectors, kThreads), bytes);
    if (past_caches<E>(sw, bytes)) pack8_kernel<E, true><<<sw.grid, kThreads, 0, s>>>((const E*)x, (int8_t*)q, (uint8_t*)scale, n, vectors);
    else pack8_kernel<E, false><<<sw.grid, kThreads, 0, s>>>((const E*)x, (int8_t*)q, (uint8_t*)scale, n, vectors);
  };
  if (dtype == MOSAIC_BF16) launch(bf16{}); else launch(float{});
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

mosaic_status launch_unpack8(hipStream_t s, int quota, int dtype, int64_t n, const void* q, const void* scale, void* x) {
  if (n == 0) return MOSAIC_OK;
  auto launch = [&](auto type) {
    typedef decltype(type) E;
    if (!on16({x, q})) {
      unpack8_any_kernel<E><<<grid_for(quota, 8, ceil_div(n, kThreads)), kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (E*)x, n);
      return;
    }
    const int64_t vectors = ceil_div(n, 8), bytes = n * (int64_t)(sizeof(E) + 1);
    const Sweep sw = sweep_grid(s, quota, ceil_div(vectors, kThreads), bytes);
    if (past_caches<E>(sw, bytes)) unpack8_kernel<E, true><<<sw.grid, kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (E*)x, n, vectors);
    else unpack8_kernel<E, false><<<sw.grid, kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (E*)x, n, vectors);
  };
  if (dtype == MOSAIC_BF16) launch(bf16{}); else launch(float{});
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

namespace {
// launch(type, act) for the pair at hand
template <typename F> void of_type_and_act(int dtype, int act, F launch) {
  auto of_act = [&](auto type) {
    if (act == MOSAIC_GELU) launch(type, std::integral_constant<int, MOSAIC_GELU>{});
    else if (act == MOSAIC_SWIGLU) launch(type, std::integral_constant<int, MOSAIC_SWIGLU>{});
    else launch(type, std::integral_constant<int, MOSAIC_GELU_TANH>{});
  };
  if (dtype == MOSAIC_BF16) of_act(bf16{}); else of_act(float{});
}
}  // namespace

mosaic_status launch_act_fwd_pack8(hipStream_t s, int quota, int dtype, int act, int64_t T, int64_t f, const void* z, void* a, void* q, void* scale) {
  if (T * f == 0) return MOSAIC_OK;
  const bool glu = act == MOSAIC_SWIGLU, whole = !glu || f % kBlock == 0;
  const int64_t m = T * f, n = glu ? 2 * m : m;
  if (whole && on16({z, a, q})) {
    of_type_and_act(dtype, act, [&](auto type, auto kind) {
      typedef decltype(type) E;
      constexpr int ACT = decltype(kind)::value;
      const int64_t vectors = glu ? m / 8 : ceil_div(n, kBlock) * (kBlock / 8), blocks = ceil_div(vectors, kThreads), bytes = (n + m) * (int64_t)sizeof(E) + n;
      const Sweep sw = sweep_grid(s, quota, blocks, bytes);
      auto with = [&](auto past) {
        act_fwd_kernel<E, ACT, decltype(past)::value><<<sw.grid, kThreads, 0, s>>>((const E*)z, (E*)a, (int8_t*)q, (uint8_t*)scale, n, vectors, f / 8);
      };
      if (past_caches<E>(sw, bytes)) with(std::true_type{}); else with(std::false_type{});
    });
    MOSAIC_LAUNCH_CHECK();
    return MOSAIC_OK;
  }
  if (glu && f % 8 == 0 && on16({z, a, q})) {
    auto launch = [&](auto type) {
      typedef decltype(type) E;
      const int64_t vectors = ceil_div(n, kBlock) * (kBlock / 8), bytes = (n + m) * (int64_t)sizeof(E) + n;
      const Sweep sw = sweep_grid(s, quota, ceil_div(vectors, kThreads), bytes);
      auto with = [&](auto past) {
        swiglu_fwd_flat_kernel<E, decltype(past)::value><<<sw.grid, kThreads, 0, s>>>((const E*)z, (E*)a, (int8_t*)q, (uint8_t*)scale, n, vectors, f / 8);
      };
      if (past_caches<E>(sw, bytes)) with(std::true_type{}); else with(std::false_type{});
    };
    if (dtype == MOSAIC_BF16) launch(bf16{}); else launch(float{});
    MOSAIC_LAUNCH_CHECK();
    return MOSAIC_OK;
  }
  const int grid = grid_for(quota, 8, ceil_div(m, kThreads));
  of_type_and_act(dtype, act, [&](auto type, auto kind) {
    typedef decltype(type) E;
    act_fwd_any_kernel<E, decltype(kind)::value><<<grid, kThreads, 0, s>>>((const E*)z, (E*)a, T, f);
  });
  MOSAIC_LAUNCH_CHECK();
  return launch_pack8(s, quota, dtype, n, z, q, scale);
}

mosaic_status launch_act_bwd_pack8(hipStream_t s, int quota, int dtype, int act, int64_t T, int64_t f, const void* q, const void* scale, const void* da,
                                   void* dz, void* a) {
  if (T * f == 0) return MOSAIC_OK;
  const bool glu = act == MOSAIC_SWIGLU, whole = !glu || f % 8 == 0;
  const int64_t m = T * f, n = glu ? 2 * m : m;
  of_type_and_act(dtype, act, [&](auto type, auto kind) {
    typedef decltype(type) E;
    constexpr int ACT = decltype(kind)::value;
    if (!whole || !on16({q, da, dz, a})) {
      act_bwd_any_kernel<E, ACT><<<grid_for(quota, 8, ceil_div(m, kThreads)), kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (const E*)da, (E*)dz, (E*)a, T, f);
      return;
    }
    const int64_t vectors = ceil_div(m, 8), blocks = ceil_div(vectors, kThreads), bytes = n + (n + (a ? 2 : 1) * m) * (int64_t)sizeof(E);
    const Sweep sw = sweep_grid(s, quota, blocks, bytes);
    auto with = [&](auto past, auto again) {
      act_bwd_kernel<E, ACT, decltype(past)::value, decltype(again)::value><<<sw.grid, kThreads, 0, s>>>(
          (const int8_t*)q, (const uint8_t*)scale, (const E*)da, (E*)dz, (E*)a, n, vectors, f / 8);
    };
    auto of_past = [&](auto past) { if (a) with(past, std::true_type{}); else with(past, std::false_type{}); };
    if (past_caches<E>(sw, bytes)) of_past(std::true_type{}); else of_past(std::false_type{});
  });
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

// scratch: the input as numbers of `dtype`, then what the weight gradient of a linear layer wants
size_t linear_wgrad_pack8_scratch_bytes(int dtype, int64_t T, int64_t k, int64_t n) {
  return align_up((size_t)T * k * dtype_size(dtype), 256) + align_up(gemm_splitk_scratch_bytes(k, n, T), 256) + colsum_scratch_bytes(n);
}

mosaic_status launch_linear_wgrad_pack8(hipStream_t s, int quota, int dtype, int64_t T, int64_t k, int64_t n, const void* q, const void* scale, const void* dY,
                                        void* dW, void* db, void* scratch) {
  if (dtype == MOSAIC_BF16 && wgrad_pack8_small(T, k, n, q, dY, dW)) return launch_wgrad_pack8_small(s, quota, T, k, n, q, scale, dY, dW, db);
  char* x = (char*)scratch;
  char* splitk = x + align_up((size_t)T * k * dtype_size(dtype), 256);
  MOSAIC_TRY(launch_unpack8(s, quota, dtype, T * k, q, scale, x));
  MOSAIC_TRY(launch_gemm(s, quota, dtype, false, false, k, n, T, x, k, dY, n, dW, n, nullptr, nullptr, splitk));
  if (db) MOSAIC_TRY(launch_colsum(s, quota, dtype, T, n, dY, db, splitk + align_up(gemm_splitk_scratch_bytes(k, n, T), 256)));
  return MOSAIC_OK;
}
