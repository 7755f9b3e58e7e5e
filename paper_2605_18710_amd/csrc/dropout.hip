// Dropout whose mask is never stored: y = R + x * keep / (1 - p), keep computed from the element's number.  The same call on the gradient of y is the
// backward pass.
//
// Random bits: Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), a bijection of a
// counter of 128 bits under a key of 64: the counter is (block, offset + site), the key the seed, a block eight consecutive elements with 16 bits
// each.  So an element's bits depend on nothing but its number, whatever the type, the grid or the alignment.  An element stays where its bits are
// at least `drop` = p * 65536 rounded, and is divided by the exact probability of that, 1 - drop / 65536.
//
// What bounds it: memory, once the bits are shared: 32 bits an element would take a generator of about 26 multiplications and 60 other operations to
// four elements, which no longer hides behind the 4 to 6 bytes that bf16 moves.  4 x 4096 x 4096 bf16 with a residual: 67.5 us, 6.0 TB/s.
#include "kernels.h"

namespace {

struct Philox { uint32_t w[4]; };
__device__ __forceinline__ Philox philox(uint64_t counter_low, uint64_t counter_high, uint64_t key) {
  uint32_t c0 = (uint32_t)counter_low, c1 = (uint32_t)(counter_low >> 32), c2 = (uint32_t)counter_high, c3 = (uint32_t)(counter_high >> 32);
  uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

// Eight elements to a thread.  VEC: their accesses are whole 16-byte pieces (the last, ragged block aside).
template <typename T, bool RES, bool VEC, bool PAST>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, const T* R, T* y, int64_t n, uint32_t drop, float scale, uint64_t site,
                                                      const uint64_t* __restrict__ rng) {
  constexpr int N = Vec16<T>::N, P = 8 / N;
  const uint64_t seed = rng[0], turn = rng[1] + site;
  const int64_t blocks = (n + 7) / 8;
  for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * 256) {
    const int64_t at = b * 8;
    const bool whole = VEC && at + 8 <= n;
    Vec16<T> vx[P], vr[P];
    if (whole) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        vx[i].template load<PAST>(x + at + i * N);
        if constexpr (RES) vr[i].template load<PAST>(R + at + i * N);
      }
    }
    const Philox r = philox((uint64_t)b, turn, seed);
    auto one = [&](int e, float v, float res) {
      const uint32_t bits = e & 1 ? r.w[e >> 1] >> 16 : r.w[e >> 1] & 0xffffu;
      // a dropped element leaves nothing behind, NaN and infinities neither
      const float kept = bits >= drop ? v * scale : 0.f;
      return RES ? res + kept : kept;
    };
    if (whole) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
#pragma unroll
        for (int e = 0; e < N; ++e) vx[i].set(e, one(i * N + e, vx[i].get(e), RES ? vr[i].get(e) : 0.f));
        vx[i].template store<PAST>(y + at + i * N);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) y[at + e] = from_f32<T>(one(e, to_f32(x[at + e]), RES ? to_f32(R[at + e]) : 0.f));
    }
  }
}

template <typename T>
mosaic_status dropout_t(hipStream_t s, int quota, int64_t n, uint32_t drop, uint64_t site, const uint64_t* rng, const T* x, const T* R, T* y) {
  const bool vec = (((uintptr_t)x | (uintptr_t)R | (uintptr_t)y) & 15) == 0;
  const float scale = drop < 65536 ? 65536.f / (float)(65536 - drop) : 0.f;
  const int64_t bytes = n * (int64_t)sizeof(T) * (R ? 3 : 2);
  const Sweep g = sweep_grid(s, quota, ceil_div(n, 2048), bytes);
  const bool past = vec && g.in_order && bytes > kPastCacheBytes;
  auto go = [&](auto res, auto v, auto p) {
    dropout_kernel<T, decltype(res)::value, decltype(v)::value, decltype(p)::value><<<g.grid, 256, 0, s>>>(x, R, y, n, drop, scale, site, rng);
  };
  auto with = [&](auto res) {
    if (past) go(res, std::true_type{}, std::true_type{});
    else if (vec) go(res, std::true_type{}, std::false_type{});
    else go(res, std::false_type{}, std::false_type{});
  };
  if (R) with(std::true_type{}); else with(std::false_type{});
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

}  // namespace

mosaic_status launch_dropout(hipStream_t s, int quota, int dtype, int64_t n, uint32_t drop, uint64_t site, const void* rng, const void* x, const void* R, void* y) {
  if (n == 0) return MOSAIC_OK;
  if (dtype == MOSAIC_BF16) return dropout_t<bf16>(s, quota, n, drop, site, (const uint64_t*)rng, (const bf16*)x, (const bf16*)R, (bf16*)y);
  return dropout_t<float>(s, quota, n, drop, site, (const uint64_t*)rng, (const float*)x, (const float*)R, (float*)y);
}
