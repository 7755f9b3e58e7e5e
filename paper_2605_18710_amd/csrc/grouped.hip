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
#include "gemm_few.h"
#include "gemm_plan.h"
#include "gemm_w4.h"
#include "kernels.h"

namespace {

// Tiles of 256, 224, 192 or 160 rows, whichever fill the rounds of 256 CUs best, half a tile more for every group than its rows fill (a round of lower ones takes
// 0.9, 0.8, 0.73 of the time: they read the weight side's fragments for fewer instructions); of 128 where the groups have no more rows on average.
// 16384 rows of 16 experts, 2048 x 5632: 338 us by 256 rows (6.2 rounds), 331 by 224 (7.0); 41794 rows of 4, 1840 x 1064 214, 200 by 192.
inline int tile_rows(int64_t T, int64_t groups, int64_t tiles_n) {
  if (T <= 128 * groups) return 4;
  const double with = (double)std::min(groups, T), cost[] = {3.5, 3.15, 2.8, 2.57};
  double least = 1e30;
  int best = 8;
  for (int i = 0; i < 4; ++i) {
    // uneven ends of the groups: half a tile each on average, give or take sqrt(groups / 12) in all
    const double per = (double)tiles_n / 256.0, rounds = ((double)T / (32.0 * (8 - i)) + 0.5 * with) * per, spread = std::sqrt(with / 12.0) * per;
    const double us = (std::ceil(rounds - spread) + std::ceil(rounds) + std::ceil(rounds + spread)) / 3.0 * cost[i];
    if (us < least - 1e-9) { least = us; best = 8 - i; }
  }
  return best;
}
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
  switch (tile_rows(p.M, p.groups, p.tiles_n)) {
    case 4: return go(std::integral_constant<int, 4>{});
    case 5: return go(std::integral_constant<int, 5>{});
    case 6: return go(std::integral_constant<int, 6>{});
    case 7: return go(std::integral_constant<int, 7>{});
    default: return go(std::integral_constant<int, 8>{});
  }
}

// Few rows to a group, or few tiles: items of 64 columns and up to 16 RB rows of a group (few_tile).
// What bounds it: W, read once from memory for up to 16 RB rows.  48 rows of 8 experts, 4096 x 1408 (93 MB): 20 us, four-wave kernel 86.
template <bool B_KC, int RB>
__global__ __launch_bounds__(kFewNT, few_waves(RB)) void grouped_few_kernel(const bf16* __restrict__ A, const bf16* __restrict__ W, bf16* __restrict__ C, int T, int groups,
                                                             int K, int N, const int32_t* __restrict__ offsets) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int starts[kMaxGroups + 1];
  const W4GroupTiles tiles_of = {starts, groups};
  tiles_of.fill(offsets, T, 16 * RB);
  __syncthreads();
  const int cols = (N + 63) / 64, items = starts[groups] * cols;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int tile = item / cols, n0 = (item - tile * cols) * 64, group = tiles_of.group_of(tile);
    const int lo = min(max(offsets[group], 0), T), rows = max(0, min(max(offsets[group + 1], 0), T) - lo);
    bf16* const out = C + (int64_t)lo * N;
    few_tile<true, B_KC, RB>(A + (int64_t)lo * K, K, (tile - starts[group]) * 16 * RB, rows, W + (int64_t)group * K * N, B_KC ? K : N, n0, N, K, smem,
                             [&](int row, int col, const float (&v)[8]) {
                               bf16x8 o;
#pragma unroll
                               for (int e = 0; e < 8; ++e) o[e] = (bf16)v[e];
                               if (row < rows && col < N) *reinterpret_cast<bf16x8*>(out + (int64_t)row * N + col) = o;
                             });
  }
}

// Weight gradients of few tiles: items of 64 x 64 of a group's matrix, the group's rows shared by eight waves.
// 11749 rows of 3 experts, 104 x 136: 32 us, four-wave kernel 106.
__global__ __launch_bounds__(kFewNT) void grouped_few_wgrad_kernel(const bf16* __restrict__ X, const bf16* __restrict__ dY, bf16* __restrict__ dW, int T, int groups, int k,
                                                                   int n, const int32_t* __restrict__ offsets) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int rows_of = (k + 63) / 64, cols = (n + 63) / 64;
  const int64_t items = (int64_t)groups * rows_of * cols;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int group = (int)(item / (rows_of * cols)), tile = (int)(item - (int64_t)group * (rows_of * cols)), m0 = tile / cols * 64, n0 = tile % cols * 64;
    const int lo = min(max(offsets[group], 0), T), rows = max(0, min(max(offsets[group + 1], 0), T) - lo);
    bf16* const out = dW + (int64_t)group * k * n;
    few_tile<false, false, 4>(X + (int64_t)lo * k, k, m0, k, dY + (int64_t)lo * n, n, n0, n, rows, smem, [&](int row, int col, const float (&v)[8]) {
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (bf16)v[e];
      if (row < k && col < n) *reinterpret_cast<bf16x8*>(out + (int64_t)row * n + col) = o;
    });
  }
}

template <bool B_KC, int RB>
mosaic_status launch_few(hipStream_t s, int quota, int T, int groups, int K, int N, const int32_t* offsets, const void* A, const void* W, void* C) {
  static std::once_flag once;
  static hipError_t rc = hipSuccess;
  constexpr int kLds = few_lds<true, B_KC, RB>();
  MOSAIC_TRY(few_allow_lds(grouped_few_kernel<B_KC, RB>, kLds, &once, &rc));
  const int64_t items = (ceil_div(T, 16 * RB) + std::min(groups, T)) * ceil_div(N, 64);
  grouped_few_kernel<B_KC, RB><<<grid_for(quota, RB == 1 ? 2 : 1, items), kFewNT, kLds, s>>>((const bf16*)A, (const bf16*)W, (bf16*)C, T, groups, K, N, offsets);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

// Row blocks of 16 in an item of grouped_few_kernel, or 0: the four-wave kernel.  Half a tile more for every group than its rows fill.  Measured, four-wave
// kernel / items of 16, 32, 64 rows:
//   4 experts, 4096 x 4096, forward, 8 rows each 86 / 32 33 37, 32 rows 85 / 57 51 41, 64 rows 86 / 90 66 63, 200 rows 84 / - 130 107
//   16 experts, 2048 x 1408, forward, 8 rows 46 / 24 26 32, 64 rows 47 / 70 51 47, 128 rows 49 / - 81 70;  16 of 4096 x 4096, 8 rows 111 / 122 125 133
//   64 experts, 512 x 512, input gradient, 8 rows 16.8 / 10.3 13.6 15.2, 64 rows 17.6 / 25.9 26.2 22.2;  one, 200 rows, 17 / - 7 9
inline int few_blocks(int64_t T, int64_t groups, int64_t K, int64_t N) {
  const double with = (double)std::min(groups, T);
  auto tiles = [&](double rows) { return std::max(with, (double)T / rows + 0.5 * with); };
  const bool low = T <= 128 * groups;
  double least = w4_price(tiles(low ? 128 : 256) * (double)ceil_div(N, 256), (double)K, low);
  int best = 0;
  for (int blocks = 1; blocks <= 4; blocks *= 2) {
    const double us = few_price(tiles(16.0 * blocks) * (double)ceil_div(N, 64), (double)K, blocks, blocks == 1);
    if (us < least) { least = us; best = blocks; }
  }
  return best;
}
// Weight gradients.  14419 rows of 10 experts, some of many rows, 216 x 976: four-wave kernel 103 us, items of 64 x 64 42.
inline bool few_wgrad(int64_t T, int64_t groups, int64_t k, int64_t n) {
  const double K = (double)T / (double)groups, longest = groups > 1 ? std::min((double)T, kUneven * K) : K;
  const double items = (double)(groups * ceil_div(k, 64) * ceil_div(n, 64)), tiles = (double)(groups * ceil_div(k, 256) * ceil_div(n, 256));
  return std::max(few_price(items, K, 4, false), few_price(1, longest, 4, false)) < std::max(w4_price(tiles, K, false), w4_price(1, longest, false));
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
  if (wgrad && few_wgrad(T, groups, k, n)) {
    static std::once_flag once;
    static hipError_t rc = hipSuccess;
    constexpr int kLds = few_lds<false, false, 4>();
    MOSAIC_TRY(few_allow_lds(grouped_few_wgrad_kernel, kLds, &once, &rc));
    grouped_few_wgrad_kernel<<<grid_for(quota, 1, groups * ceil_div(k, 64) * ceil_div(n, 64)), kFewNT, kLds, s>>>(p.A, p.B, p.C, (int)T, groups, (int)k, (int)n, offsets);
    MOSAIC_LAUNCH_CHECK();
    return MOSAIC_OK;
  }
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
