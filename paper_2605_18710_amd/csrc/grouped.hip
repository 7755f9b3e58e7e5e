// Products of rows sorted by group with their group's matrix, the form that the MLPs of experts take: rows offsets[g] .. offsets[g + 1] - 1 are
// group g's, and offsets lie on the device, where a router left them.
//   forward          Y_r  = X_r W_g(r)        W [groups, k, n]
//   input gradient   dX_r = dY_r W_g(r)^T
//   weight gradient  dW_g = X_g^T dY_g        zero for a group without rows
//
// bf16: the four-wave kernel (gemm_w4.h), whose workgroups find the tiles of all groups from the offsets at their start, one list in the order of the
// groups; no tile holds rows of two groups.  fp32, and bf16 sizes or alignments that it does not take: gemm_f32_grouped_kernel.
// Every output is the sum over its contraction in ascending order, by one wave: its bits depend on the sizes of the
// groups in nothing.
#include "gemm_plan.h"
#include "gemm_w4.h"
#include "kernels.h"

mosaic_status launch_grouped_f32(hipStream_t s, int quota, int dtype, bool a_kc, bool b_kc, int M, int N, int K, const void* A, int64_t lda, const void* B,
                                 int64_t ldb, void* C, int64_t ldc, const void* R, const int32_t* offsets, int groups, int bound, int64_t stride);

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
