// Products of rows sorted by group with their group's matrix, the form that the MLPs of experts take: rows offsets[g] .. offsets[g + 1] - 1 are
// group g's, and offsets lie on the device, where a router left them.
//   forward          Y_r  = X_r W_g(r)        W [groups, k, n]
//   input gradient   dX_r = dY_r W_g(r)^T
//   weight gradient  dW_g = X_g^T dY_g        zero for a group without rows
//
// bf16: the four-wave kernel (gemm_w4.h), whose workgroups find the tiles of all groups from the offsets at their start, one list in the order of the
// groups; no tile holds rows of two groups.  Few rows to a group, or few tiles: grouped_few_kernel.  fp32, and bf16 sizes or alignments that
// neither takes: gemm_f32_grouped_kernel.
// Every output is a sum over its contraction in an order that T, groups, k and n fix: its bits do not depend on where the groups end.
#include <math.h>
#include "gemm_plan.h"
#include "gemm_w4.h"
#include "kernels.h"

mosaic_status launch_grouped_f32(hipStream_t s, int quota, int dtype, bool a_kc, bool b_kc, int M, int N, int K, const void* A, int64_t lda, const void* B,
                                 int64_t ldb, void* C, int64_t ldc, const void* R, const int32_t* offsets, int groups, int bound, int64_t stride, int split_k = 0, int splits = 1);

namespace {

// Tiles of 256 rows, or of 128 where the groups have no more on average: an expert's rows seldom fill a tile, and half a tile less is computed for nothing.
template <bool A_KC, bool B_KC>
mosaic_status launch_rows(hipStream_t s, int quota, W4Args p) {
  auto go = [&](auto mi) -> mosaic_status {
    constexpr int MI = decltype(mi)::value;
    p.tiles_m = (int)ceil_div(p.M, 32 * MI);
    const int64_t most = (p.tiles_m + (int64_t)std::min(p.groups, p.M)) * p.tiles_n;
    if (most > INT32_MAX / 2) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "too many output tiles");
    p.tile_count = (int)most;
    p.row_block = row_block_for(p.K, p.M, 32 * MI);
    return launch_w4_epi<A_KC, B_KC, W4_PLAIN, MI, W4_GROUPED>(s, quota, p);
  };
  return p.M <= 128 * (int64_t)p.groups ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 8>{});
}

// Few rows to a group, or few tiles: an item is 64 columns of up to 16 RB rows of a group, its contraction dealt to eight waves in steps of 64 k-values (step i to
// wave i % 8, so the waves read on side by side), whose sums meet in LDS in wave order.  A wave keeps two steps in registers on their way, 16 KB of W.
//   W [N, K] rows (input gradient): straight to the matrix instructions, of a row's 128-byte line 32 bytes to a lane; the rows' k-values lie alike.
//   W [K, N] (forward): k-rows of 128 bytes into the wave's own 8 KB of LDS, 32-byte chunks XOR-swizzled by bits 1 and 3 of the row, and out
//     again by the transposing read.
// What bounds it: W, read once from memory for up to 16 RB rows.  48 rows of 8 experts, 4096 x 1408 (93 MB): 20 us, four-wave kernel 86.
constexpr int kStep = 64, kFewWaves = 8;
template <bool B_KC, int RB>
__global__ __launch_bounds__(64 * kFewWaves) void grouped_few_kernel(const bf16* __restrict__ A, const bf16* __restrict__ W, bf16* __restrict__ C, int T, int groups,
                                                                     int K, int N, const int32_t* __restrict__ offsets) {
  constexpr int kRows = 16 * RB;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int starts[kMaxGroups + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, g = lane >> 4;
  const W4GroupTiles tiles_of = {starts, groups};
  tiles_of.fill(offsets, T, kRows);
  __syncthreads();
  const int cols = (N + 63) / 64, items = starts[groups] * cols, steps = (K + kStep - 1) / kStep;
  const int64_t ldw = B_KC ? K : N;
  lds_byte* const mine = (lds_byte*)smem + wave * 8192;
  float* const sums = reinterpret_cast<float*>(smem);                    // [wave][row][64]
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int tile = item / cols, n0 = (item - tile * cols) * 64;
    const int group = tiles_of.group_of(tile);
    const int lo = min(max(offsets[group], 0), T), hi = max(lo, min(max(offsets[group + 1], 0), T));
    const int r0 = lo + (tile - starts[group]) * kRows;
    const bf16* const Wg = W + (int64_t)group * K * N;
    const bf16* a_row[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) a_row[i] = A + (int64_t)min(r0 + 16 * i + lr, hi - 1) * K;      // rows past the last one repeat it, and are not stored
    bf16x8 w[2][8], x[2][RB][2];
    // step s: w[.][2j + half] is 16 columns' (j) k-values 16g + 8 half of it, or k-row lane / 8 + 8i, columns 8 (lane % 8)
    auto request = [&](auto buf, int s) {
      constexpr int B = decltype(buf)::value;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[B][i] = bf16x8{};
        if constexpr (B_KC) {
          const int k = s * kStep + 16 * g + 8 * (i & 1), row = n0 + 16 * (i >> 1) + lr;
          if (k < K && row < N) w[B][i] = *reinterpret_cast<const bf16x8*>(Wg + (int64_t)row * ldw + k);
        } else {
          const int k = s * kStep + 8 * i + (lane >> 3), c = n0 + 8 * (lane & 7);
          if (k < K && c < N) w[B][i] = *reinterpret_cast<const bf16x8*>(Wg + (int64_t)k * ldw + c);
        }
      }
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int k = s * kStep + (B_KC ? 16 * g + 8 * half : 32 * half + 8 * g);
          x[B][i][half] = bf16x8{};
          if (k < K) x[B][i][half] = *reinterpret_cast<const bf16x8*>(a_row[i] + k);
        }
    };
    f32x4 acc[RB][4];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](auto buf) {
      constexpr int B = decltype(buf)::value;
      if constexpr (!B_KC) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = 8 * i + (lane >> 3), c = lane & 7, f = ((row >> 1) & 1) | (((row >> 3) & 1) << 1);
          *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>(mine + row * 128 + (((c >> 1) ^ f) << 5) + 16 * (c & 1)) = w[B][i];
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bf16x8 b;
          if constexpr (B_KC) {
            b = w[B][2 * j + half];
          } else {
            const int q = lr >> 2, f = (q >> 1) | ((g & 1) << 1);
            const lds_byte* const at = mine + (32 * half + 8 * g + q) * 128 + ((j ^ f) << 5) + 8 * (lr & 3);
            const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
            const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 4 * 128));
            typedef __attribute__((ext_vector_type(8))) short s16x8;
            b = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
          }
#pragma unroll
          for (int i = 0; i < RB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, x[B][i][half], acc[i][j], 0, 0, 0);
        }
      if constexpr (!B_KC) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();                     // read before the next step is written
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    };
    typedef std::integral_constant<int, 0> B0;
    typedef std::integral_constant<int, 1> B1;
    request(B0{}, wave);
    for (int s = wave; s < steps; s += 2 * kFewWaves) {
      request(B1{}, s + kFewWaves);                          // past the contraction: zeros
      multiply(B0{});
      request(B0{}, s + 2 * kFewWaves);
      multiply(B1{});
    }
    __syncthreads();                                         // the waves' parts of LDS become the sums'
    // acc[i][j][e] is row 16i + lr, column 16j + 4g + e
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(sums + (wave * kRows + 16 * i + lr) * 64 + ((16 * j + 4 * g) ^ ((lr & 7) << 3))) = acc[i][j];
    __syncthreads();
    // eight columns to a lane
    for (int i = threadIdx.x; i < kRows * 8; i += 64 * kFewWaves) {
      const int r = i >> 3, c = (i & 7) * 8;
      float v[8] = {};
#pragma unroll
      for (int u = 0; u < kFewWaves; ++u) {
        const float* const at = sums + (u * kRows + r) * 64 + (c ^ ((r & 7) << 3));
        const f32x4 low = *reinterpret_cast<const f32x4*>(at), high = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] += low[e]; v[4 + e] += high[e]; }
      }
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (bf16)v[e];
      if (r0 + r < hi && n0 + c < N) *reinterpret_cast<bf16x8*>(C + (int64_t)(r0 + r) * N + n0 + c) = o;
    }
    __syncthreads();                                         // and the waves' again
  }
}

template <bool B_KC, int RB>
mosaic_status launch_few(hipStream_t s, int quota, int T, int groups, int K, int N, const int32_t* offsets, const void* A, const void* W, void* C) {
  constexpr int kLds = std::max(kFewWaves * 16 * RB * 64 * 4, B_KC ? 0 : kFewWaves * 8192);
  auto kern = grouped_few_kernel<B_KC, RB>;
  static std::once_flag attr_once;
  static hipError_t attr_rc = hipSuccess;
  std::call_once(attr_once, [&] { attr_rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kLds); });
  MOSAIC_HIP(attr_rc);
  const int64_t items = (ceil_div(T, 16 * RB) + std::min(groups, T)) * ceil_div(N, 64);
  kern<<<grid_for(quota, RB <= 2 ? 2 : 1, items), 64 * kFewWaves, kLds, s>>>((const bf16*)A, (const bf16*)W, (bf16*)C, T, groups, K, N, offsets);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

// Row blocks of 16 in an item of grouped_few_kernel, or 0: the four-wave kernel.  By the shape alone, since the order of the sums differs: prices in microseconds on the whole
// device, half a tile more for every group than its rows fill.  The four-wave kernel takes 1.3 (tiles of 128 rows; 256: 1.5) for 64 k-values of a tile, alone on
// its CU.  Items read W and their rows through the caches at 6.3 TB/s, or wait 1.45 for a step of each wave.  Measured, four-wave kernel / items of 16, 32, 64 rows:
//   4 experts, 4096 x 4096, forward, 8 rows each 86 / 32 33 37, 32 rows 85 / 57 51 41, 64 rows 86 / 90 66 63, 200 rows 84 / - 130 107
//   16 experts, 2048 x 1408, forward, 8 rows 46 / 24 26 32, 64 rows 47 / 70 51 47, 128 rows 49 / - 81 70;  16 of 4096 x 4096, 8 rows 111 / 122 125 133
//   64 experts, 512 x 512, input gradient, 8 rows 16.8 / 10.3 13.6 15.2, 64 rows 17.6 / 25.9 26.2 22.2;  one, 200 rows, 17 / - 7 9
inline int few_blocks(int64_t T, int64_t groups, int64_t K, int64_t N) {
  const double with = (double)std::min(groups, T), ktiles = (double)ceil_div(K, 64);
  auto tiles = [&](double rows) { return std::max(with, (double)T / rows + 0.5 * with); };
  const bool low = T <= 128 * groups;
  double least = 4.0 + std::ceil(tiles(low ? 128 : 256) * (double)ceil_div(N, 256) / 256.0) * std::max(2.0, ktiles) * (low ? 1.3 : 1.5);
  int best = 0;
  for (int blocks = 1; blocks <= 4; blocks *= 2) {
    const double items = tiles(16.0 * blocks) * (double)ceil_div(N, 64), slots = blocks <= 2 ? 512.0 : 256.0;
    const double waits = std::ceil(items / slots) * (2.0 + std::ceil(ktiles / kFewWaves) * 1.45), reads = items * (double)K * 2.0 * (64.0 + 16.0 * blocks) / 6.3e6;
    const double us = 4.0 + std::max(waits, reads);
    if (us < least) { least = us; best = blocks; }
  }
  return best;
}

}  // namespace

mosaic_status launch_grouped(hipStream_t s, int quota, int dtype, GroupedForm form, int64_t T, int groups, int64_t k, int64_t n, const int32_t* offsets,
                             const void* A, const void* B, void* C) {
  if (groups == 0 || (T == 0 && form != GROUPED_WGRAD)) return MOSAIC_OK;
  const bool dgrad = form == GROUPED_DGRAD, wgrad = form == GROUPED_WGRAD;
  // contraction and columns; W [k, n] of a group is B, or C
  const int64_t K = wgrad ? T : dgrad ? n : k, N = dgrad ? k : n, M = wgrad ? k : T, lda = dgrad ? n : k, ldb = n, ldc = dgrad ? k : n;
  const bool w4 = dtype == MOSAIC_BF16 && k % 8 == 0 && n % 8 == 0 && (((uintptr_t)A | (uintptr_t)B | (uintptr_t)C) & 15) == 0 && k * n < ((int64_t)1 << 31) - 8 &&
                  k < (1 << 22) && n < (1 << 22);
  if (!w4)
    return launch_grouped_f32(s, quota, dtype, !wgrad, dgrad, (int)M, (int)N, (int)K, A, lda, B, ldb, C, ldc, nullptr, offsets, groups, (int)T, k * n);
  if (const int blocks = wgrad ? 0 : few_blocks(T, groups, K, N)) {
    auto go = [&](auto kc) -> mosaic_status {
      constexpr bool KC = decltype(kc)::value;
      if (blocks == 1) return launch_few<KC, 1>(s, quota, (int)T, groups, (int)K, (int)N, offsets, A, B, C);
      if (blocks == 2) return launch_few<KC, 2>(s, quota, (int)T, groups, (int)K, (int)N, offsets, A, B, C);
      return launch_few<KC, 4>(s, quota, (int)T, groups, (int)K, (int)N, offsets, A, B, C);
    };
    return dgrad ? go(std::true_type{}) : go(std::false_type{});
  }
  W4Args p = {};
  p.A = (const bf16*)A; p.B = (const bf16*)B; p.C = (bf16*)C;
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.lda = lda; p.ldb = ldb; p.ldc = ldc;
  p.offsets = offsets; p.groups = groups; p.bound = (int)T; p.stride = k * n;
  p.b_bytes = (uint32_t)(k * n * 2);
  p.tiles_n = (int)ceil_div(N, 256);
  if (wgrad) {
    p.tiles_m = (int)ceil_div(M, 256);
    const int64_t all = (int64_t)p.tiles_m * p.tiles_n * groups;
    if (all > INT32_MAX / 2) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "too many output tiles");
    p.tile_count = (int)all;
    p.row_block = row_block_for(K, M, 256);
    return launch_w4_epi<false, false, W4_PLAIN, 8, W4_GROUPED>(s, quota, p, true);
  }
  return dgrad ? launch_rows<true, true>(s, quota, p) : launch_rows<true, false>(s, quota, p);
}
