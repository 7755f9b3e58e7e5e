// Activations kept in 8 bits between the forward and the backward pass, and the backward kernels that read them.
//
// A block of 32 consecutive elements has one exponent e, the smallest from -127 on with max |x| <= 127.5 * 2^e, kept as the byte e + 127, and the
// whole numbers q nearest to x / 2^e (ties to even, at most 127 in size): an element is off by half of 2^e at most, and
// q * 2^e is a bf16 number, so that unpacking rounds nothing.  x / 2^e is exact too: the bits do not depend on how it is computed.  A block
// with a NaN or an infinity has the byte 255 and comes back as NaN.
#include "kernels.h"
#include "activations.h"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;

// `top`: bits of the block's largest magnitude
__device__ __forceinline__ int scale_byte(unsigned top) {
  if (top >= 0x7f800000u) return 255;
  const int e = (int)(top >> 23) - 6 + ((top & 0x7fffffu) > 0x7f0000u);     // exponent byte of e; 127.5 = 1.9921875 * 2^6
  return e < 0 ? 0 : e;
}
__device__ __forceinline__ float step_of(int byte) {          // 2^e
  return __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x400000u : (unsigned)byte << 23);
}
__device__ __forceinline__ float inverse_step(int byte) {     // 2^-e; e is 122 at most (a NaN's numbers are 0)
  return __uint_as_float(byte == 255 ? 0u : (unsigned)(254 - byte) << 23);
}
__device__ __forceinline__ int packed(float x, float inverse) {
  const float v = rintf(x * inverse);
  return v != v ? 0 : (int)fminf(fmaxf(v, -127.f), 127.f);
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

template <int ACT> __device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == MOSAIC_GELU) return gelu_f(z);
  else return tanh_gelu_f(z);
}
template <int ACT> __device__ __forceinline__ float act_grad_of(float z) {
  if constexpr (ACT == MOSAIC_GELU) return gelu_grad_f(z);
  else return tanh_gelu_grad_f(z);
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void act_fwd_any_kernel(const T* __restrict__ z, T* __restrict__ a, int64_t rows, int64_t f) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * f; i += (int64_t)gridDim.x * kThreads) {
    if constexpr (ACT == MOSAIC_SWIGLU) {
      const int64_t r = i / f, at = i + r * f;              // row r starts at 2 r f
      a[i] = from_f32<T>(swiglu_f(to_f32(z[at]), to_f32(z[at + f])));
    } else {
      a[i] = from_f32<T>(act_of<ACT>(to_f32(z[i])));
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
      swiglu_grad_f(gate, up, d, &dg, &du);
      dz[at] = from_f32<T>(dg);
      dz[at + f] = from_f32<T>(du);
      if (a) a[i] = from_f32<T>(swiglu_f(gate, up));
    } else {
      const float z = value(i);
      dz[i] = from_f32<T>(d * act_grad_of<ACT>(z));
      if (a) a[i] = from_f32<T>(act_of<ACT>(z));
    }
  }
}

}  // namespace

size_t pack8_scale_bytes(int64_t n) { return (size_t)ceil_div(n, kBlock); }

mosaic_status launch_pack8(hipStream_t s, int quota, int dtype, int64_t n, const void* x, void* q, void* scale) {
  if (n == 0) return MOSAIC_OK;
  const int64_t blocks = ceil_div(n, kBlock);
  const int grid = grid_for(quota, 8, ceil_div(n, kThreads));
  if (dtype == MOSAIC_BF16) pack8_any_kernel<bf16><<<grid, kThreads, 0, s>>>((const bf16*)x, (int8_t*)q, (uint8_t*)scale, n, blocks);
  else pack8_any_kernel<float><<<grid, kThreads, 0, s>>>((const float*)x, (int8_t*)q, (uint8_t*)scale, n, blocks);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

mosaic_status launch_unpack8(hipStream_t s, int quota, int dtype, int64_t n, const void* q, const void* scale, void* x) {
  if (n == 0) return MOSAIC_OK;
  const int grid = grid_for(quota, 8, ceil_div(n, kThreads));
  if (dtype == MOSAIC_BF16) unpack8_any_kernel<bf16><<<grid, kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (bf16*)x, n);
  else unpack8_any_kernel<float><<<grid, kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (float*)x, n);
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
  const int grid = grid_for(quota, 8, ceil_div(T * f, kThreads));
  of_type_and_act(dtype, act, [&](auto type, auto kind) {
    typedef decltype(type) E;
    act_fwd_any_kernel<E, decltype(kind)::value><<<grid, kThreads, 0, s>>>((const E*)z, (E*)a, T, f);
  });
  MOSAIC_LAUNCH_CHECK();
  return launch_pack8(s, quota, dtype, act == MOSAIC_SWIGLU ? 2 * T * f : T * f, z, q, scale);
}

mosaic_status launch_act_bwd_pack8(hipStream_t s, int quota, int dtype, int act, int64_t T, int64_t f, const void* q, const void* scale, const void* da,
                                   void* dz, void* a) {
  if (T * f == 0) return MOSAIC_OK;
  const int grid = grid_for(quota, 8, ceil_div(T * f, kThreads));
  of_type_and_act(dtype, act, [&](auto type, auto kind) {
    typedef decltype(type) E;
    act_bwd_any_kernel<E, decltype(kind)::value><<<grid, kThreads, 0, s>>>((const int8_t*)q, (const uint8_t*)scale, (const E*)da, (E*)dz, (E*)a, T, f);
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
  char* x = (char*)scratch;
  char* splitk = x + align_up((size_t)T * k * dtype_size(dtype), 256);
  MOSAIC_TRY(launch_unpack8(s, quota, dtype, T * k, q, scale, x));
  MOSAIC_TRY(launch_gemm(s, quota, dtype, false, false, k, n, T, x, k, dY, n, dW, n, nullptr, nullptr, splitk));
  if (db) MOSAIC_TRY(launch_colsum(s, quota, dtype, T, n, dY, db, splitk + align_up(gemm_splitk_scratch_bytes(k, n, T), 256)));
  return MOSAIC_OK;
}
