// Products of few rows, or of few tiles over a long contraction, on the matrix cores: 64 columns of up to 64 rows to a workgroup, whose eight waves share
// the contraction.  (The four-wave kernel's tiles of 128 or 256 rows and 256 columns take 1.3 us for 64 k-values when they have a CU each
// to themselves, however few their rows are.)
#pragma once
#include <math.h>
#include "gemm_w4.h"

namespace {

constexpr int kFewStep = 64, kFewWaves = 8, kFewNT = 64 * kFewWaves;
// two workgroups to a CU for items of 16 rows: four waves to a SIMD
constexpr int few_waves(int RB) { return RB == 1 ? 4 : 2; }
// bytes of LDS: the waves' own 8 KB for every operand whose contraction is the strided index, or then their sums
template <bool A_KC, bool B_KC, int RB> constexpr int few_lds() {
  return std::max(kFewWaves * 16 * RB * 64 * 4, kFewWaves * 8192 * ((A_KC ? 0 : 1) + (B_KC ? 0 : 1)));
}

// 64 k-rows x 64 columns of an operand [K, X] as rows of 128 bytes, 32-byte chunks XOR-swizzled by bits 1 and 3 of the row, and out again by the
// transposing read: both touch every bank alike.
__device__ __forceinline__ void few_put(lds_byte* area, const bf16x8 (&v)[8]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 8 * i + (lane >> 3), c = lane & 7, f = ((row >> 1) & 1) | (((row >> 3) & 1) << 1);
    *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>(area + row * 128 + (((c >> 1) ^ f) << 5) + 16 * (c & 1)) = v[i];
  }
}
// columns 16j .. 16j+15, k-values 32 half .. 32 half + 31
__device__ __forceinline__ bf16x8 few_get(const lds_byte* area, int j, int half) {
  typedef __attribute__((ext_vector_type(8))) short s16x8;
  const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4, q = lr >> 2, f = (q >> 1) | ((g & 1) << 1);
  const lds_byte* const at = area + (32 * half + 8 * g + q) * 128 + ((j ^ f) << 5) + 8 * (lr & 3);
  const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
  const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 4 * 128));
  return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
}

// C[m0 .. m0 + 16 RB - 1, n0 .. n0 + 63] of C[M,N] = op(A) op(B): finish(row, col, v) for eight columns v[8] of a row, by eight lanes side by side for a row's 64, rows
// and columns past M and N too.  A [M, K] (A_KC) or [K, M] (RB 4), B [N, K] (B_KC) or [K, N]; lda, ldb, M or N where they are a row's length rounded up, and K
// where it is, multiples of 8, zeros or readable up to there.  K = 0: zeros.  LO: A is the sum of two, the other one a_lo elements behind it, whose product is added
// (16 rows with a contiguous contraction: in the same step, so that B is read once).
// Step i of 64 k-values is wave i % 8's, so the waves read on side by side; a wave has two steps on their way in registers, 16 KB of B.  An operand
// whose contraction is contiguous goes straight to the matrix instructions: of a row's 128-byte line 32 bytes to a lane where
// both are, else the k-values that the transposing read gives.  The waves' sums meet in LDS and are added in wave order.
template <bool A_KC, bool B_KC, int RB, bool LO = false, typename FINISH>
__device__ __forceinline__ void few_tile(const bf16* __restrict__ A, int64_t lda, int m0, int M, const bf16* __restrict__ B, int64_t ldb, int n0, int N, int K,
                                         unsigned char* smem, FINISH finish, int64_t a_lo = 0) {
  static_assert(A_KC || RB == 4, "a strided row operand comes in 64 columns");
  constexpr int kRows = 16 * RB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, g = lane >> 4;
  constexpr bool BOTH = LO && A_KC && RB == 1;
  const int once = (K + kFewStep - 1) / kFewStep, steps = LO && !BOTH ? 2 * once : once;
  lds_byte* const mine_b = (lds_byte*)smem + wave * 8192 * ((A_KC ? 0 : 1) + (B_KC ? 0 : 1));
  lds_byte* const mine_a = mine_b + (B_KC ? 0 : 8192);
  float* const sums = reinterpret_cast<float*>(smem);                    // [wave][row][64]
  const bf16* a_row[RB];
#pragma unroll
  for (int i = 0; i < RB; ++i) a_row[i] = A + (int64_t)min(m0 + 16 * i + lr, M - 1) * lda;      // A_KC: rows past the last one repeat it
  constexpr int NA = A_KC ? 2 * RB : 8;
  bf16x8 a[2][NA], b[2][8], more[2][BOTH ? NA : 1];
  auto request = [&](auto buf, int s) {
    constexpr int U = decltype(buf)::value;
    const bool low = LO && !BOTH && s >= once;
    const int k0 = (low ? s - once : s) * kFewStep;
    const int64_t lo = low ? a_lo : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      b[U][i] = bf16x8{};
      if constexpr (B_KC) {                      // [2j + half]: row 16j + lr
        const int k = k0 + (A_KC ? 16 * g + 8 * (i & 1) : 32 * (i & 1) + 8 * g), row = n0 + 16 * (i >> 1) + lr;
        if (k < K && row < N) b[U][i] = *reinterpret_cast<const bf16x8*>(B + (int64_t)row * ldb + k);
      } else {
        const int k = k0 + 8 * i + (lane >> 3), c = n0 + 8 * (lane & 7);
        if (k < K && c < N) b[U][i] = *reinterpret_cast<const bf16x8*>(B + (int64_t)k * ldb + c);
      }
    }
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      a[U][i] = bf16x8{};
      if constexpr (A_KC) {                      // [2i + half]
        const int k = k0 + (B_KC ? 16 * g + 8 * (i & 1) : 32 * (i & 1) + 8 * g);
        if (k < K) a[U][i] = *reinterpret_cast<const bf16x8*>(a_row[i >> 1] + lo + k);
        if constexpr (BOTH) {
          more[U][i] = bf16x8{};
          if (k < K) more[U][i] = *reinterpret_cast<const bf16x8*>(a_row[i >> 1] + a_lo + k);
        }
      } else {
        const int k = k0 + 8 * i + (lane >> 3), c = m0 + 8 * (lane & 7);
        if (k < K && c < M) a[U][i] = *reinterpret_cast<const bf16x8*>(A + lo + (int64_t)k * lda + c);
      }
    }
  };
  f32x4 acc[RB][4];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto meet = [] {                               // of one wave's own accesses to LDS
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  auto multiply = [&](auto buf) {
    constexpr int U = decltype(buf)::value;
    if constexpr (!B_KC) few_put(mine_b, b[U]);
    if constexpr (!A_KC) few_put(mine_a, a[U]);
    if constexpr (!A_KC || !B_KC) meet();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      bf16x8 x[RB];
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        if constexpr (A_KC) x[i] = a[U][2 * i + half];
        else x[i] = few_get(mine_a, i, half);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 y;
        if constexpr (B_KC) y = b[U][2 * j + half];
        else y = few_get(mine_b, j, half);
#pragma unroll
        for (int i = 0; i < RB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x[i], acc[i][j], 0, 0, 0);
        if constexpr (BOTH) acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, more[U][half], acc[0][j], 0, 0, 0);
      }
    }
    if constexpr (!A_KC || !B_KC) meet();        // read before the next step is written
  };
  typedef std::integral_constant<int, 0> B0;
  typedef std::integral_constant<int, 1> B1;
  request(B0{}, wave);
  for (int s = wave; s < steps; s += 2 * kFewWaves) {
    request(B1{}, s + kFewWaves);                // past the contraction: zeros
    multiply(B0{});
    request(B0{}, s + 2 * kFewWaves);
    multiply(B1{});
  }
  __syncthreads();                               // the waves' parts of LDS become the sums'
  // acc[i][j][e] is row 16i + lr, column 16j + 4g + e
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(sums + (wave * kRows + 16 * i + lr) * 64 + ((16 * j + 4 * g) ^ ((lr & 7) << 3))) = acc[i][j];
  __syncthreads();
  for (int i = threadIdx.x; i < (kRows * 8 + 63) / 64 * 64; i += kFewNT) {
    const int r = i >> 3, c = (i & 7) * 8;
    float v[8] = {};
#pragma unroll
    for (int u = 0; u < kFewWaves; ++u) {
      const float* const at = sums + (u * kRows + r) * 64 + (c ^ ((r & 7) << 3));
      const f32x4 low = *reinterpret_cast<const f32x4*>(at), high = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] += low[e]; v[4 + e] += high[e]; }
    }
    finish(m0 + r, n0 + c, v);
  }
  __syncthreads();                               // and the waves' again
}

template <typename KERN>
mosaic_status few_allow_lds(KERN kern, int bytes, std::once_flag* once, hipError_t* rc) {
  std::call_once(*once, [&] { *rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
  MOSAIC_HIP(*rc);
  return MOSAIC_OK;
}

// Prices in microseconds on the whole device, of the shape alone since the order of the sums goes by the way taken.  A tile of the four-wave kernel takes 1.3 (128 rows;
// 256: 1.5) for 64 k-values while it has its CU to itself.  Workgroups of few_tile read their operands through the caches at 6.3 TB/s together, or wait 1.45
// for a step of each wave; two of them share a CU where their LDS allows.
inline double w4_price(double tiles, double K, bool low) { return 4.0 + std::ceil(tiles / 256.0) * std::max(2.0, std::ceil(K / 64.0)) * (low ? 1.3 : 1.5); }
// items and operands of a group whose rows are its contraction are taken as the average, but the longest chain as 2.5 times that: experts are not chosen evenly
constexpr double kUneven = 2.5;
inline double few_price(double items, double K, int blocks, bool twice) {
  const double waits = std::ceil(items / (twice ? 512.0 : 256.0)) * (2.0 + std::ceil(std::ceil(K / 64.0) / kFewWaves) * 1.45);
  return 4.0 + std::max(waits, items * K * 2.0 * (64.0 + 16.0 * blocks) / 6.3e6);
}

}  // namespace
