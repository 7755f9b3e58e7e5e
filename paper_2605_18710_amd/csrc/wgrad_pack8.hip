// Weight gradient dW[k,n] = X^T dY of a linear layer whose input X[T,k] was kept in 8 bits, in one launch: the numbers become bf16 on their way into
// LDS, the matrix cores take them with dY from there, and the first row of tiles adds up dY's columns (db) as they pass.
#include <type_traits>
#include "kernels.h"
#include "pack8.h"

namespace {

constexpr int kTokens = 64;       // of a step
constexpr int kTile = 64;
constexpr unsigned kOut = 0x80000000u;

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)bytes, 0x00020000);
}

// A tile in LDS: kTokens rows of kTile bf16 numbers, 128 bytes each.  The two 64-byte pieces of every other pair of rows are swapped, so that the four
// consecutive rows that a transposing read takes lie on different banks (256 bytes of them).
__device__ __forceinline__ int lds_at(int row, int col) { return row * (kTile * 2) + (((col >> 5) ^ (row >> 1 & 1)) << 6) + (col & 31) * 2; }
// 32 columns from c0 on and 16 tokens from t0 on as a matrix operand: lane l has column c0 + l % 32 and tokens t0 + 8 (l / 32) .. + 7
__device__ __forceinline__ bf16x8 fragment(const lds_byte* tile, int t0, int c0) {
  const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
  const int row = t0 + 8 * (g >> 1) + (i >> 2), col = c0 + 16 * (g & 1) + 4 * (i & 3);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tile + lds_at(row, col)));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tile + lds_at(row + 4, col)));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The eight values of two words, a quarter of them: (number + 128) * step - 128 * step in one operation, where the whole step would overflow in blocks of the
// largest numbers.
__device__ __forceinline__ bf16x8 quarters(uint32_t lo, uint32_t hi, int byte) {
  const float step = 0.25f * step_of(byte), shift = -128.f * step;
  bf16x8 v;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t w = (h ? hi : lo) ^ 0x80808080u;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * h + k] = (bf16)fmaf((float)(w >> (8 * k) & 0xffu), step, shift);
  }
  return v;
}

struct Args {
  const int8_t* q;
  const uint8_t* scale;
  const bf16* dy;
  bf16* dw;
  bf16* db;
  int T, k, n, tiles_m, tiles_n;
};

// 64 x 64 of dW for a workgroup.  G groups of four waves take every G-th step of 64 tokens, a quarter of the tile for each wave, and the groups' sums are added
// in order at the end.  A step is a chain (barrier, 16 reads from LDS, conversion of 16 numbers, writes, four products that wait for each other) of 0.39 us
// where a CU has one workgroup of four waves; the second group fills its gaps (0.57 us for both steps).
// Steps are requested kAhead rounds ahead, in registers; a group's two tiles in LDS take turns, and the next round's numbers are converted while
// these operands are on their way from LDS.
// SHARED: one tile holds columns 0 to 15 and the last block, which T k ends within.
template <int G, bool SHARED>
__global__ __launch_bounds__(256 * G) void wgrad_pack8_kernel(Args p) {
  constexpr int kAhead = 4, kSteps = kTokens / 16;
  constexpr int kTileBytes = kTile * kTokens * 2, kStage = 2 * kTileBytes;
  __shared__ __attribute__((aligned(128))) unsigned char smem[G * 2 * kStage];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave >> 2, lane = threadIdx.x & 63, tid = threadIdx.x & 255;
  lds_byte* const lds = (lds_byte*)smem + group * 2 * kStage;
  const int wm = (wave >> 1 & 1) * 32, wn = (wave & 1) * 32;
  const auto rq = rsrc(p.q, (int64_t)p.T * p.k), ry = rsrc(p.dy, (int64_t)p.T * p.n * 2);
  const unsigned numbers = (unsigned)p.T * (unsigned)p.k;
  const int rounds = (p.T + G * kTokens - 1) / (G * kTokens);
  const int row_a = tid >> 2, col_a = (tid & 3) * 16, row_b = tid >> 3, col_b = (tid & 7) * 8;
  for (int item = blockIdx.x; item < p.tiles_m * p.tiles_n; item += gridDim.x) {
    const int m0 = item / p.tiles_n * kTile, n0 = item % p.tiles_n * kTile;
    const bool with_db = p.db && m0 == 0;
    // Where this thread reads next.  Past the last token an offset is past its descriptor's end, and so is every offset of a column that the matrix does not
    // have: such requests give zeros, with no branch.  (Offsets stay below 2^31 + 2^31: wgrad_pack8_small.)
    // So do those of exponent bytes but for one: where T k ends within a block, columns 0 to 15 behind the last token would get that block's byte, a NaN's
    // perhaps, which makes NaN of zeros.  The tile that holds these columns holds none of that block's from 80 columns on: its bytes end before the block.  With fewer
    // (SHARED) offsets are compared (2048 tokens 1024 x 1024 13.1 us, compared 14.2).
    const auto rs = rsrc(p.scale, (numbers + (SHARED || m0 > 0 ? 31u : 0u)) / 32u);
    unsigned at_a = (m0 + col_a < p.k ? 0u : kOut) + (unsigned)(group * kTokens + row_a) * (unsigned)p.k + (unsigned)(m0 + col_a);
    unsigned at_b = (n0 + col_b < p.n ? 0u : kOut) + ((unsigned)(group * kTokens + row_b) * (unsigned)p.n + (unsigned)(n0 + col_b)) * 2u;
    struct Step { u32x4 q; unsigned s; u32x4 y[2]; } in[kAhead];
    auto request = [&](Step& r) {
      r.q = __builtin_amdgcn_raw_buffer_load_b128(rq, (int)at_a, 0, 0);
      r.s = __builtin_amdgcn_raw_buffer_load_b8(rs, (int)(SHARED && at_a >= numbers ? kOut : at_a >> 5), 0, 0);
      r.y[0] = __builtin_amdgcn_raw_buffer_load_b128(ry, (int)at_b, 0, 0);
      r.y[1] = __builtin_amdgcn_raw_buffer_load_b128(ry, (int)(at_b + 64u * (unsigned)p.n), 0, 0);
      at_a += (unsigned)(G * kTokens) * (unsigned)p.k;
      at_b += (unsigned)(G * kTokens * 2) * (unsigned)p.n;
    };
    f32x16 acc = {};
    float sums[8] = {};
    auto convert = [&](const Step& r, lds_byte* ta) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *(__attribute__((address_space(3))) bf16x8*)(ta + lds_at(row_a, col_a + 8 * h)) = quarters(r.q[2 * h], r.q[2 * h + 1], (int)r.s);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        *(__attribute__((address_space(3))) u32x4*)(ta + kTileBytes + lds_at(row_b + 32 * j, col_b)) = r.y[j];
        if (with_db) {
          const bf16x8 y = __builtin_bit_cast(bf16x8, r.y[j]);
#pragma unroll
          for (int e = 0; e < 8; ++e) sums[e] += (float)y[e];
        }
      }
    };
#pragma unroll
    for (int a = 0; a < kAhead; ++a) request(in[a]);
    convert(in[0], lds);
    request(in[0]);
    auto work = [&](auto slot) {
      constexpr int a = decltype(slot)::value;
      const lds_byte* const ta = lds + (a & 1) * kStage;
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");        // this turn's numbers are written, the last turn's read; loads stay in flight
      bf16x8 fa[kSteps], fb[kSteps];
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        fa[ks] = fragment(ta, 16 * ks, wm);
        fb[ks] = fragment(ta + kTileBytes, 16 * ks, wn);
      }
      convert(in[(a + 1) % kAhead], lds + (a + 1 & 1) * kStage);              // zeros behind the last round
      request(in[(a + 1) % kAhead]);
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[ks], fa[ks], acc, 0, 0, 0);
    };
    // Whole turns of the four slots without a way out in between: the compiler then knows how many requests are younger than the one it waits for
    // (with one it waited for all of them, and a step took 0.77 us).
    int left = rounds;
    for (; left >= kAhead; left -= kAhead) {
      work(std::integral_constant<int, 0>{}); work(std::integral_constant<int, 1>{});
      work(std::integral_constant<int, 2>{}); work(std::integral_constant<int, 3>{});
    }
    if (left > 0) work(std::integral_constant<int, 0>{});
    if (left > 1) work(std::integral_constant<int, 1>{});
    if (left > 2) work(std::integral_constant<int, 2>{});
    __syncthreads();                                  // the tiles in LDS have been read
    if constexpr (G > 1) {                            // [group - 1][wave of the group][register][lane]
      float* const part = (float*)smem;
      if (group > 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) part[(((group - 1) * 4 + (wave & 3)) * 16 + i) * 64 + lane] = acc[i];
      }
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int g = 0; g < G - 1; ++g)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[i] += part[((g * 4 + wave) * 16 + i) * 64 + lane];
      }
      __syncthreads();
    }
    if (group == 0) {                                 // lane l of a 32 x 32 block has row l % 32 of dW and columns 8 g + 4 (l / 32) + 0..3
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int row = m0 + wm + (lane & 31), col = n0 + wn + 8 * g + 4 * (lane >> 5);
        bf16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (bf16)(4.f * acc[4 * g + e]);
        if (row < p.k && col < p.n) *(bf16x4*)(p.dw + (int64_t)row * p.n + col) = o;
      }
    }
    if (with_db) {                                    // uniform: a thread's sums over its rows, then the threads in order
      float* const part = (float*)smem;
#pragma unroll
      for (int e = 0; e < 8; ++e) part[(threadIdx.x >> 3) * kTile + col_b + e] = sums[e];
      __syncthreads();
      if (threadIdx.x < kTile && n0 + (int)threadIdx.x < p.n) {
        float v = 0.f;
        for (int r = 0; r < 32 * G; ++r) v += part[r * kTile + threadIdx.x];
        p.db[n0 + threadIdx.x] = (bf16)v;
      }
      __syncthreads();
    }
  }
}

}  // namespace

// Where this kernel is the faster road: small outputs, whose time the other one (unpack, product, column sums) spends between its launches.  A pure rule on the
// shape: the two add in different orders, and results must not depend on the quota.  us, this / the other one: 64 tokens 256 x 256 4.3 / 11.7, 512 tokens
// 1024 x 1024 6.6 / 11.0, 1500 tokens 1280 x 1280 with db 18 / 26, 4096 tokens 1024 x 1024 with db 24 / 37; but 9216 tokens 1024 x 1024 48 / 48, 16384 tokens 256 x 256
// 76 / 35 (one workgroup's chain of steps), 1024 tokens 2048 x 2048 23 / 19, 256 tokens 4096 x 4096 39 / 20.
// X's rows are whole 16-byte pieces within blocks of 32, and descriptors hold 32 bits.
bool wgrad_pack8_small(int64_t T, int64_t k, int64_t n, const void* q, const void* dY, const void* dW) {
  const int64_t most = (int64_t)1 << 30;              // bytes; 5 rounds more stay below 2^31
  if (k % 16 || n % 8 || k >= (1 << 20) || n >= (1 << 19) || T * k >= most || T * n * 2 >= most) return false;
  if ((((uintptr_t)q | (uintptr_t)dY) & 15) || ((uintptr_t)dW & 7)) return false;
  const int64_t tiles = ceil_div(k, kTile) * ceil_div(n, kTile), steps = ceil_div(T, kTokens);
  return tiles <= 256 ? steps <= 64 : tiles * steps <= 10240;
}

mosaic_status launch_wgrad_pack8_small(hipStream_t s, int quota, int64_t T, int64_t k, int64_t n, const void* q, const void* scale, const void* dY, void* dW,
                                       void* db) {
  const Args p = {(const int8_t*)q, (const uint8_t*)scale, (const bf16*)dY, (bf16*)dW, (bf16*)db, (int)T, (int)k, (int)n, (int)ceil_div(k, kTile), (int)ceil_div(n, kTile)};
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  // Two groups where a CU would have a workgroup to itself (1568 tokens 768 x 768 13.1 -> 11.5 us, 4096 tokens 1024 x 1024 28.8 -> 24.5; but 1500 tokens
  // 1280 x 1280, 400 tiles, 18.2 -> 19.6), and more than one step to share.
  auto launch = [&](auto shared) {
    if (tiles <= 256 && T > kTokens) wgrad_pack8_kernel<2, decltype(shared)::value><<<grid_for(quota, 2, tiles), 512, 0, s>>>(p);
    else wgrad_pack8_kernel<1, decltype(shared)::value><<<grid_for(quota, 2, tiles), 256, 0, s>>>(p);
  };
  if (k <= kTile && T * k % 32) launch(std::true_type{}); else launch(std::false_type{});
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}
