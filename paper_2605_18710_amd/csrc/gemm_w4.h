// What the matrix-core kernels of gemm.hip, grouped.hip and linear_ce.hip share: the order of a product's tiles, and the four-wave kernel.
#pragma once
#include "activations.h"
#include "common.h"
#include "tile_queue.h"
#include <algorithm>
#include <mutex>
#include <type_traits>

namespace {

#pragma clang diagnostic ignored "-Winline-asm"   // m0 is named as a clobber on purpose

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

constexpr unsigned kOob = 0xFFFFFFF0u;   // byte offset beyond any descriptor's range

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;

// Position `tile` of the tile list -> (tile row, tile column).  The list is panel-major: panels
// of 8 tile columns, row-major inside a panel, so 32 consecutive entries form a 4 x 8 patch that
// shares operand panels in one XCD's L2.  Above that, tile rows are taken in super-blocks of
// `row_block` rows (all panels of a super-block before the next super-block), sized on the
// host so that the row operand of a super-block (row_block x 256 rows x K) stays in the
// last-level cache: it is then re-read from there, not from HBM, once per panel (measured on
// the 7B-shaped products: +3 % forward, +4 % input gradient; the board is power-bound and HBM
// reads cost energy).  Both kernels and both launches of a mixed plan use this one order.
__device__ __forceinline__ void tile_coords(int tile, int tiles_m, int tiles_n, int row_block, int* row, int* col) {
  const int per_sb = row_block * tiles_n;
  const int sb = tile / per_sb, rem = tile - sb * per_sb;
  const int rows_sb = min(row_block, tiles_m - sb * row_block);
  const int panel = rem / (rows_sb * 8);
  const int pw = min(8, tiles_n - panel * 8);
  const int in_panel = rem - panel * rows_sb * 8;
  *row = sb * row_block + in_panel / pw;
  *col = panel * 8 + in_panel % pw;
}

// Where row r of the activation goes in that input (24000 x 1280 from 240 k-values: product 59 us and gather 35 -> 82): tap 1 of output r / 2 (even rows), or tap 2 of it and tap 0 of the next one; the last row
// of a sample, which has no next one, clears tap 0 of the sample's first output.  Element offsets of its first column, -1: none.
struct TapRows { int64_t first, second; bool zero; };
// r mod r_rows with r_magic = 2^32 / r_rows + 1: exact as long as r * r_rows < 2^32 (checked by the launcher)
__device__ __forceinline__ int table_row(int r, uint32_t r_rows, uint32_t r_magic) { return r - (int)(__umulhi((uint32_t)r, r_magic) * r_rows); }
__device__ __forceinline__ TapRows tap_rows(int r, int M, int64_t n, uint32_t lo, uint32_t magic) {
  const int t = r >> 1;
  TapRows o = {-1, -1, false};
  if (r < M) {
    o.first = (3 * (int64_t)t + 1 + (r & 1)) * n;
    if (r & 1) {
      o.zero = table_row(t + 1, lo, magic) == 0;
      o.second = 3 * (int64_t)(o.zero ? t + 1 - (int)lo : t + 1) * n;
    }
  }
  return o;
}

// ------------------------------------------------------------------ four-wave kernel
// 256x256x64 tiles, four waves of 128x128, v_mfma_f32_16x16x32_bf16, for every form whose
// K-contiguous operands have a contraction of whole K-tiles (K a multiple of 64).  Where the row operand is
// K-contiguous the tile may be 32 * MI rows high, MI = 8, 7, 6 or 5 (launch_mfma_shape says when).
//
// What bounds it: on the whole chip the board's power.  Registers only, random data, the
// 16x16x32 instruction delivers 1830 TFLOP/s and the 32x32x16 one 1760 (it reads and writes twice
// the accumulator bytes per flop); around it the kernel spends as little as it can: a wave tile of
// 128x128 reads 1 LDS byte per 64 flops (two thirds of what 128x64 wave tiles read), a K-tile of 64
// brings whole 128-byte lines, operands go HBM -> LDS without passing registers, 128 matrix instructions
// come with about 135 others per K-tile.
//   LDS: two stages of 64 KB.  The fragments of a K-tile's second half are read under its first 16
//     matrix instructions; after a barrier (slot 24 of 128) the stage is free and the K-tile after the
//     next is requested into it, one request per six matrix instructions: requests made faster than
//     the CU's vector cache takes them (16 cycles each, four waves) hold up the wave that makes
//     them.  The next K-tile has to be there, behind a second barrier, at slot 88, when its first
//     fragments are read.  Measured on 32768 x 4096 x 22016 input gradient / 12000 x 5120 x 1280
//     forward: a request per two slots, one barrier in the middle 4697 / 118 us; per four 4734 / 112;
//     two barriers and one per six 3960 / 112; without any requests the K loop takes 20 % less than
//     the first of these.
//   The stream of K-tiles runs on across output tiles; the epilogue passes through 4 KB per
//     wave behind the stages, so the next tile's first K-tiles land under it.
//   K-contiguous operand: rows of 128 bytes, 16-byte chunks XOR-swizzled by (row/2)%8, a fragment is
//     one ds_read_b128.  K-strided operand: k-rows of 512 bytes as in HBM, 32-byte chunks XOR-swizzled
//     by 2*(k%4) + (k/8)%2, a fragment is two ds_read_b64_tr_b16.  Both touch every bank once.
//   Requests take a constant offset per lane; the K-tile moves the descriptor (base and remaining
//     bytes: scalar instructions), which also bounds it: rows past the end read zeros, columns past
//     the end read the next row's values and only reach outputs that are not stored.
//   The matrix instruction is written in assembly to tie the result to its accumulator: left to
//     itself the compiler copied 400 accumulator registers per K-tile.
// Each output element is accumulated in ascending k: same bits as gemm_bf16_kernel's.
// Measured, whole device, eight-wave kernel (input gradient: a four-wave kernel that staged through
// registers) -> this: forward 32768 x 4096 x 12288 2525 -> 2300 us (1434 TFLOP/s), 8192 x 5632 x 2048
// 149 -> 129; with GELU 12000 x 1280 x 5120 199 -> 151, with SwiGLU 8192 x 2048 x 11264 365 -> 338;
// input gradient 32768 x 4096 x 22016 4433 -> 3960 (1492 TFLOP/s), 9216 x 4096 x 1024 77 -> 70;
// weight gradient 4096 x 32768 x 22016 4268 -> 4000, 2048 x 8192 x 11264 339 -> 331.
struct W4Args {
  const bf16 *A, *B, *bias, *R;
  bf16 *C, *C2;
  int M, N, K;
  int64_t lda, ldb, ldc, ldc2;
  uint32_t a_bytes, b_bytes, c_bytes, c2_bytes;
  int tiles_m, tiles_n, tile_begin, tile_count, row_block, gu_f;
  uint32_t r_rows, r_magic;        // W4_TABLE, W4_TAPS: see ActArgs
  // W4_GROUPED
  const int32_t* offsets;          // [groups + 1], on the device: group g is rows offsets[g] .. offsets[g + 1] - 1 of A (and of B, where A is K-strided)
  int groups, bound;               // offsets are held to 0 .. bound
  int64_t stride;                  // elements between two groups' B (C, where A is K-strided)
  int splits, split_k;             // W4_PIECES, K-strided A: the contraction in `splits` pieces (K-contiguous: as the kernel cuts it, split_k k-values each)
  const int32_t* rows;             // W4_PIECES, K-contiguous A: where a row of the product goes in C.  W4_SOFTMAX: its target, a column or -1
  float* sums;                     // W4_PIECES: [pieces][rows][N], rows M, or those of the tiles that there are; W4_ADD: what is there already, [M][N]
  const float* scale;              // null, or on the device: a factor of the sums that leave for C
  int first;                       // W4_ADD: nothing is there yet
  const int32_t* piece;            // null, or [2], on the device: a row that the operands of all rows are counted from (A: W4_SOFTMAX, B: K-strided A, and
                                   // `rows`), and (W4_ADD) whether the sum is complete with this launch and goes to C
  // W4_SOFTMAX: see there
  float* at_target;
  float2* stats;
  float* totals;
};
enum { W4_PLAIN, W4_BIAS, W4_RES, W4_GELU, W4_SWIGLU, W4_TABLE, W4_TAPS, W4_PIECES, W4_ADD, W4_SOFTMAX };
// W4_GROUPED: products of groups of rows with a matrix each; how many rows a group has is known on the device only.  The tiles of a group's
// product follow those of the one before; tiles of a K-contiguous A are cut at the ends of its groups, a K-strided A has all tiles of
// C for every group.  Group sizes bound the descriptors, so no tile reads or writes another group's rows.
enum { W4_WHOLE, W4_GROUPED };
constexpr int kMaxGroups = 1024;

// W4_PIECES, K-contiguous A: into how many pieces the contraction of `tiles` tiles is cut, by the shape alone (256: CUs of the device that the kernels are written
// for).  Nanoseconds: 1450 for 64 k-values of a tile, 8000 around them; the sums of a tile written and read at 5 TB/s, 5000 for the pass that adds them.  Whole
// numbers, so that the product and that pass come to the same cut.  Measured: 6144 x 4096 of 128000, 384 tiles: 5600 us in two rounds, 4400 as
// three rounds of half the length; 187 x 216 of 85501, one tile: 106 us in 16 pieces, 29 in 122.
constexpr int kMostPieces = 128, kMostPieceTiles = 2048, kLeastPiece = 256, kCuts = 40;
struct W4Cut { int pieces, k; };
// candidate i: 1 to 16, then eight of even steps up to every doubling
__device__ __host__ __forceinline__ int w4_cut_pieces(int i) { return i < 16 ? i + 1 : (18 + 2 * ((i - 16) & 7)) << ((i - 16) >> 3); }
__device__ __host__ __forceinline__ W4Cut w4_cut_of(int i, int K) {
  const int n = w4_cut_pieces(i), k = ((K + n - 1) / n + 63) / 64 * 64;
  return {(K + k - 1) / k, k};
}
__device__ __host__ __forceinline__ int64_t w4_cut_ns(int i, int tiles, int K) {
  const W4Cut cut = w4_cut_of(i, K);
  if (i && (cut.k < kLeastPiece || (int64_t)w4_cut_pieces(i) * tiles > kMostPieceTiles)) return INT64_MAX >> 8;
  return ((int64_t)tiles * cut.pieces + 255) / 256 * (cut.k / 64 * (int64_t)1450 + 8000) + (i ? (int64_t)tiles * (8 * cut.pieces + 2) * 13 + 5000 : 0);
}
inline float w4_cut_us(int tiles, int K) {
  int64_t best = INT64_MAX;
  for (int i = 0; i < kCuts; ++i) best = std::min(best, w4_cut_ns(i, tiles, K));
  return (float)best * 1e-3f;
}
// all lanes of a wave together, a candidate to a lane
__device__ __forceinline__ W4Cut w4_cut(int tiles, int K) {
  const int lane = threadIdx.x & 63;
  int64_t best = lane < kCuts ? w4_cut_ns(lane, tiles, K) << 6 | lane : INT64_MAX;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) best = min(best, (int64_t)__shfl_xor((long long)best, o, 64));
  const int i = __builtin_amdgcn_readfirstlane((int)best & 63);
  const W4Cut cut = w4_cut_of(i, K);
  return {__builtin_amdgcn_readfirstlane(cut.pieces), __builtin_amdgcn_readfirstlane(cut.k)};
}
constexpr int kW4Stage = 2 * 256 * 64 * 2;                         // both operands of a K-tile
constexpr int kW4Pitch = 68;                                       // floats per row of the epilogue's patch: 16 rows of 64
constexpr int kW4Patch = 4 * 16 * kW4Pitch * 4;
constexpr int w4_lds(int epi) { return 2 * kW4Stage + kW4Patch + (epi == W4_GELU || epi == W4_TAPS ? ErfTable::kEntries * 4 : 0); }

// One operand: what a lane requests of a K-tile, and where its fragments are.
template <bool KC, bool GU, int NF = 8>
struct W4Operand {
  unsigned voff[NF];                       // byte offset of request j from the K-tile's first byte
  int kofs[KC ? 2 : 1];                    // KC: first k-value of request j % 2's 16 bytes in the K-tile
  int frag[KC ? 2 : 8];                    // LDS offsets: KC: of k-half 0 / 1, + 2048 per 16 rows; else of 16 columns each, + 16384 per k-half
  __device__ __forceinline__ void init(int wave, int w0, int64_t ld, int gu_f) {
    const int lane = threadIdx.x & 63, lr = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      if constexpr (KC) {
        const int r = 8 * NF * wave + 8 * j + (lane >> 3), ch = (lane & 7) ^ ((r >> 1) & 7);
        voff[j] = (unsigned)((int64_t)r * ld * 2 + ch * 16);
        if (j < 2) kofs[j & 1] = 8 * ch;
      } else {
        const int kr = 16 * wave + 2 * j + (lane >> 5), pos = lane & 31;
        const int c32 = (pos >> 1) ^ (((kr & 3) << 1) | ((kr >> 3) & 1));
        // GU: 16-column group c32 of the tile belongs to the gate half (even) or the up half (odd)
        const int64_t byte = GU ? (c32 >> 1) * 32 + (int64_t)(c32 & 1) * gu_f * 2 : c32 * 32;
        voff[j] = (unsigned)((int64_t)kr * ld * 2 + byte + (pos & 1) * 16);
      }
    }
    if constexpr (KC) {
      const int sw = (lr >> 1) & 7;
      frag[0] = (w0 + lr) * 128 + ((g ^ sw) << 4);
      frag[1] = (w0 + lr) * 128 + (((4 + g) ^ sw) << 4);
    } else {
      const int q = lr >> 2, f = (q << 1) | (g & 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) frag[i] = (8 * g + q) * 512 + (((w0 >> 4) + (i ^ f)) << 5) + 8 * (lr & 3);
    }
  }
  // the same for a K-tile of which only the first `left` k-values are the row's own (the others lie in the next row, and read zeros)
  __device__ __forceinline__ unsigned within(int j, int left) const {
    if constexpr (KC) return kofs[j & 1] < left ? voff[j] : kOob;
    else return voff[j];
  }
  __device__ __forceinline__ u32x4 read(const lds_byte* area, int i, int half) const {
    if constexpr (KC) {
      return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(area + frag[half] + 2048 * i);
    } else {
      const lds_byte* p = area + frag[i] + 16384 * half;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 2048));
      typedef __attribute__((ext_vector_type(8))) short s16x8;
      return __builtin_bit_cast(u32x4, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Where an operand's next K-tile starts and how many bytes of the tensor lie behind that point.
// SIZE: 64 bits for tensors of any size, of which a descriptor shows what 32 bits reach (a K-tile's requests reach less: the host checks that).
template <typename SIZE>
struct W4Cursor {
  uint64_t at;
  SIZE left;
  __device__ __forceinline__ void set(const void* base, uint64_t off, SIZE bytes) {
    at = (uint64_t)(uintptr_t)base + off;
    left = off < bytes ? (SIZE)(bytes - off) : (SIZE)0;
  }
  __device__ __forceinline__ void advance(uint32_t step) { at += step; left = left > step ? left - step : (SIZE)0; }
  __device__ __forceinline__ i32x4 desc(bool live) const {
    const uint32_t seen = sizeof(SIZE) == 8 && (uint64_t)left > 0xfffffff0u ? 0xfffffff0u : (uint32_t)left;
    i32x4 d;
    d.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)at); d.y = __builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffffu));
    d.z = __builtin_amdgcn_readfirstlane((int)(live ? seen : 0u)); d.w = 0x00020000;
    return d;
  }
};

// Where the row tiles of every group start, in LDS, and which group a tile belongs to: the last one that starts at or before it (a group
// without rows starts where the next one does).
struct W4GroupTiles {
  int* starts;                     // [groups + 1]
  int groups;
  // by the first wave, `height` rows a tile; the workgroup has to meet before the others read
  __device__ __forceinline__ void fill(const int32_t* offsets, int bound, int height) const {
    if (threadIdx.x >= 64) return;
    const int lane = threadIdx.x & 63;
    int run = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
      const int g = g0 + lane;
      int n = 0;
      if (g < groups) {
        const int lo = min(max(offsets[g], 0), bound), hi = min(max(offsets[g + 1], 0), bound);
        n = hi > lo ? (hi - lo + height - 1) / height : 0;
      }
      int scan = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(scan, o, 64);
        if (lane >= o) scan += v;
      }
      if (g < groups) starts[g] = run + scan - n;
      run += __shfl(scan, 63, 64);
    }
    if (lane == 0) starts[groups] = run;
  }
  __device__ __forceinline__ int group_of(int tile) const {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) n += __popcll(__ballot(g0 + lane < groups && starts[g0 + lane] <= tile));
    return __builtin_amdgcn_readfirstlane(n - 1);
  }
};

// W4_SOFTMAX: the product is a tile of logits.  What leaves is, for each row and block of kCeBlock columns, the largest logit m and the sum of
// exp(z - m): stats[block][row], p.M rows; the sum of the logits where totals is given; the logit of the row's target; and, where C is given,
// exp(z - m) rounded to fp16 (0 past the last column, up to ldc).
// From 0 to 1, relative to its block's largest: an fp16 number is within 2^-11 of it relative to itself, or within 2^-25 of the largest.  The logits
// themselves in 16 bits would be off by that share of the logit, which the exponential turns into that much of a probability times the logit.
// A block whose largest logit is -infinity has a sum of 0, or NaN where it holds one, and m stays -infinity: a 0 in its place would be the largest of a row whose
// logits all lie below.  +infinity makes the sum NaN.
// The exponent is (z - m) log2 e, of a difference that is exact next to m.  With m log2 e rounded by itself what is left of that rounding is an exponent: at 200 it is 10^-5 of
// every probability, and blocks that are masked by a large finite value leave fp16's range where m log2 e passes 2^28, fp32's from 2^31 on.  (One fused operation
// a logit instead of two: 13004 tokens, 25 % ignored, h 104, V 65996 419 us, this 438; 3063 tokens, h 2048, V 50021 405 to 414 either way.)
// Here for one row of two blocks side by side, a lane's sixteen values v[h][j][e] of each, columns col + 64h + 16j + 4g + e; the four lanes of a row lie 16 apart
// (g = 0 .. 3).  Two at once, because a wave is alone on its SIMD and every step waits for the one before (12288 x 4096 x 128000 9790 -> 9450 us).
constexpr int kCeBlock = 64;
// what the four lanes of a row make of their values together
template <typename F> __device__ __forceinline__ float across_rows(float x, F f) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);       // the low half's in both halves, and the high half's
  x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);       // the same by 16 lanes
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ void w4_softmax(const W4Args& p, f32x4 (&v)[2][4], int row, int col, int g, int target, bool in) {
  constexpr float kLog2e = 1.44269504088896340736f;
  auto add = [](float a, float b) { return a + b; };
  auto high = [](float a, float b) { return fmaxf(a, b); };
  const int hit = target - col;
  const bool mine = in && hit >= 0 && hit < 2 * kCeBlock && target < p.N && ((hit >> 2) & 3) == g;
  if (__ballot(mine)) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const f32x4& x = v[j >> 2][j & 3];
      const float a = hit & 1 ? x[1] : x[0], b = hit & 1 ? x[3] : x[2];
      t = hit >> 4 == j ? (hit & 2 ? b : a) : t;
    }
    if (mine) p.at_target[row] = t;
  }
  const bool first = g == 0 && in;
  const int64_t slot = (int64_t)(col / kCeBlock) * p.M + row;
  if (p.totals) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float total = 0.f;                           // rows of the table past its end read zeros
#pragma unroll
      for (int j = 0; j < 4; ++j) total += (v[h][j][0] + v[h][j][1]) + (v[h][j][2] + v[h][j][3]);
      total = across_rows(total, add);
      if (first && col + 64 * h < p.N) p.totals[slot + h * p.M] = total;
    }
  }
  if (col + 2 * kCeBlock > p.N) {
    int left = p.N - col - 4 * g;
    asm volatile("" : "+v"(left));                 // compared here, for these rows: kept for all of a tile's the masks take more scalar registers than there are
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[h][j][e] = 64 * h + 16 * j + e < left ? v[h][j][e] : -INFINITY;
  }
  float m[2], ref[2], sum[2], part[2][4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) part[h][j] = fmaxf(fmaxf(v[h][j][0], v[h][j][1]), fmaxf(v[h][j][2], v[h][j][3]));
#pragma unroll
  for (int h = 0; h < 2; ++h) m[h] = fmaxf(fmaxf(part[h][0], part[h][1]), fmaxf(part[h][2], part[h][3]));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    m[h] = across_rows(m[h], high);
    ref[h] = m[h] == -INFINITY ? 0.f : m[h];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[h][j][e] = __builtin_amdgcn_exp2f((v[h][j][e] - ref[h]) * kLog2e);
      part[h][j] = (v[h][j][0] + v[h][j][1]) + (v[h][j][2] + v[h][j][3]);
    }
#pragma unroll
  for (int h = 0; h < 2; ++h) sum[h] = across_rows((part[h][0] + part[h][1]) + (part[h][2] + part[h][3]), add);
#pragma unroll
  for (int h = 0; h < 2; ++h) if (first && col + 64 * h < p.N) p.stats[slot + h * p.M] = make_float2(m[h], sum[h]);
}

template <bool A_KC, bool B_KC, int EPI, int MI, int MAP = W4_WHOLE>
__global__ __launch_bounds__(256, 1) void gemm_bf16_w4_kernel(W4Args p, TileQueueArgs tq) {
  constexpr int OPB = kW4Stage / 2;
  constexpr bool GROUPED = MAP == W4_GROUPED;
  static_assert(MI == 8 || A_KC, "a K-strided row operand fills whole requests with 256 rows only");
  extern __shared__ __align__(16) unsigned char smem[];
  lds_byte* const lds = (lds_byte*)smem;
  const unsigned lds0 = (unsigned)(uintptr_t)lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave >> 1) * (16 * MI), wn = (wave & 1) * 128;
  // at least two, the depth of the request stream (WHOLE: the host sees to it)
  const int nk_all = GROUPED ? max(2, (p.K + 63) / 64) : (p.K + 63) / 64;
  const uint32_t astep = A_KC ? 128u : (uint32_t)(64 * p.lda * 2), bstep = B_KC ? 128u : (uint32_t)(64 * p.ldb * 2);
  W4Operand<A_KC, false, MI> oa;
  W4Operand<B_KC, EPI == W4_SWIGLU> ob;
  oa.init(wave, wm, p.lda, 0);
  ob.init(wave, wn, p.ldb, p.gu_f);

  // GROUPED: rows lo .. hi - 1 are the group's, g its number; m0 counts from lo; K-tiles from k0 on (W4_PIECES: piece `split`)
  struct Item { int m0, n0, nk, g, lo, hi, k0, split; };
  __shared__ int starts[GROUPED && A_KC ? kMaxGroups + 1 : 1];
  const W4GroupTiles tiles_of = {starts, GROUPED ? p.groups : 0};
  if constexpr (GROUPED && A_KC) {
    tiles_of.fill(p.offsets, p.bound, 32 * MI);
    __syncthreads();
    // the list is as long as the groups make it; the host's length is that of the longest
    tq.n_items = tiles_of.starts[p.groups] * p.tiles_n;
    if constexpr (EPI == W4_PIECES) {
      const W4Cut cut = w4_cut(tq.n_items, p.K);
      p.splits = cut.pieces;
      p.split_k = cut.k;
      p.M = tiles_of.starts[p.groups] * 32 * MI;
      tq.n_items *= cut.pieces;
    }
    tq.n_full = tq.n_items / (8 * tq.chunk) * (8 * tq.chunk);
    tq.tail_per = (tq.n_items - tq.n_full + 7) / 8;
  }
  const int start = GROUPED && p.piece ? __builtin_amdgcn_readfirstlane(p.piece[0]) : 0;
  const float scale = GROUPED && p.scale ? *p.scale : 1.f;
  const bool last = EPI == W4_ADD && p.piece && __builtin_amdgcn_readfirstlane(p.piece[1]);
  if (EPI == W4_ADD && !p.first && !last && p.offsets[1] <= p.offsets[0]) { tq.n_items = tq.n_full = tq.tail_per = 0; }      // nothing to add
  auto decode = [&](int item) -> Item {
    int trow, tcol;
    if constexpr (GROUPED) {
      Item r = {};
      r.nk = nk_all;
      if constexpr (A_KC) {
        if constexpr (EPI == W4_PIECES) {
          const int all = tiles_of.starts[p.groups] * p.tiles_n;
          r.split = item / all;
          item -= r.split * all;
          r.k0 = r.split * p.split_k;
          r.nk = max(2, (min(p.K - r.k0, p.split_k) + 63) / 64);
        }
        r.g = tiles_of.group_of(item / p.tiles_n);
        const int at = starts[r.g];
        tile_coords(item - at * p.tiles_n, starts[r.g + 1] - at, p.tiles_n, p.row_block, &trow, &tcol);
      } else {
        const int all = p.tiles_m * p.tiles_n;
        r.g = item / all;
        tile_coords(item - r.g * all, p.tiles_m, p.tiles_n, p.row_block, &trow, &tcol);
        if constexpr (EPI == W4_PIECES) { r.split = r.g; r.g = 0; }          // of one group
      }
      r.lo = __builtin_amdgcn_readfirstlane(min(max(p.offsets[r.g], 0), p.bound));
      r.hi = __builtin_amdgcn_readfirstlane(max(r.lo, min(max(p.offsets[r.g + 1], 0), p.bound)));
      if constexpr (!A_KC && EPI == W4_PIECES) {
        const int per = ((r.hi - r.lo + p.splits - 1) / p.splits + 63) / 64 * 64;          // the rows that there are, in equal pieces
        r.lo = min(r.lo + r.split * per, r.hi);
        r.hi = min(r.lo + per, r.hi);
      }
      if constexpr (!A_KC) r.nk = max(2, (r.hi - r.lo + 63) / 64);
      r.m0 = trow * (32 * MI);
      r.n0 = tcol * 256;
      return r;
    } else {
      tile_coords(p.tile_begin + item, p.tiles_m, p.tiles_n, p.row_block, &trow, &tcol);
      return {trow * (32 * MI), tcol * 256, nk_all};
    }
  };
  W4Cursor<typename std::conditional<GROUPED, uint64_t, uint32_t>::type> ca, cb;
  int k_left = 0;                              // GROUPED: k-values from the cursors' K-tile on
  auto point = [&](const Item& it) {
    k_left = p.K - it.k0;
    if constexpr (GROUPED && A_KC) {
      const bf16* B = p.B + it.g * p.stride;
      ca.set(p.A + (int64_t)(it.lo + (EPI == W4_SOFTMAX ? start : 0)) * p.lda, ((uint64_t)it.m0 * p.lda + it.k0) * 2,
             ((uint64_t)(it.hi - it.lo - 1) * p.lda + p.K) * 2);
      cb.set(B, ((uint64_t)it.n0 * (B_KC ? p.ldb : 1) + (uint64_t)it.k0 * (B_KC ? 1 : p.ldb)) * 2, p.b_bytes);
    } else if constexpr (GROUPED) {
      const uint64_t n = (uint64_t)(it.hi - it.lo);
      ca.set(p.A + (int64_t)it.lo * p.lda, (uint64_t)it.m0 * 2, n ? ((n - 1) * p.lda + (p.M + 7) / 8 * 8) * 2 : 0);      // whole 16-byte pieces: a row has them
      cb.set(p.B + (int64_t)(it.lo + start) * p.ldb, (uint64_t)it.n0 * 2, n ? ((n - 1) * p.ldb + p.N) * 2 : 0);
    } else {
      ca.set(p.A, A_KC ? (uint64_t)it.m0 * p.lda * 2 : (uint64_t)it.m0 * 2, p.a_bytes);
      cb.set(p.B, B_KC ? (uint64_t)it.n0 * p.ldb * 2 : (uint64_t)(EPI == W4_SWIGLU ? it.n0 : it.n0 * 2), p.b_bytes);
    }
  };
  const unsigned wdst = lds0 + (unsigned)wave * 8192, adst = lds0 + (unsigned)wave * (MI * 1024);
  auto request = [&](const i32x4& d, unsigned off, unsigned dst) {
    // m0 = LDS address of lane 0's 16 bytes; lane l lands at m0 + 16*l.  Completion is waited for by hand.
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(dst), "v"(off), "s"(d) : "m0");
  };
  auto request_tile = [&](int st) {
    i32x4 da = ca.desc(true), db = cb.desc(true);
    // A memory instruction may read a scalar register that the vector unit wrote (v_readfirstlane) five wait
    // states later at the earliest, and the compiler does not see the requests: both descriptors
    // pass through these five, so that no part of them is formed later.
    asm volatile("s_nop 4" : "+s"(da), "+s"(db));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < MI; ++j) request(da, GROUPED ? oa.within(j, k_left) : oa.voff[j], adst + (unsigned)(st * kW4Stage + j * 1024));
#pragma unroll
    for (int j = 0; j < 8; ++j) request(db, GROUPED ? ob.within(j, k_left) : ob.voff[j], wdst + (unsigned)(st * kW4Stage + OPB + j * 1024));
    ca.advance(astep);
    cb.advance(bstep);
    k_left -= 64;
  };

  __shared__ int mail;
  TileQueueCursor qc;
  int item = tq_first(tq, qc, &mail);
  if (item < 0) { tq_done(tq); return; }
  Item it = decode(item);
  point(it);
  request_tile(0);
  request_tile(1);
  // 256 values of a tile to a thread: seven erff to fill the table instead of 256 (the epilogue of 12000 x 1280 x 5120
  // takes 10 us of 150; with erff in it, four waves a CU, 83 of 239)
  float* const erf_table = reinterpret_cast<float*>(smem + 2 * kW4Stage + kW4Patch);
  if constexpr (EPI == W4_GELU || EPI == W4_TAPS) {
    ErfTable::fill(erf_table, threadIdx.x, 256);
    __syncthreads();
  }
  f32x4 acc[MI][8];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 ax[MI], bx[8], ay[MI], by[8];          // fragments of the first and of the second half
  __builtin_amdgcn_s_waitcnt(((MI + 8) & 15) | (7 << 4) | (15 << 8) | (((MI + 8) >> 4) << 14));      // vmcnt: the first K-tile has landed
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i < MI) ax[i] = oa.read(lds, i, 0);
    bx[i] = ob.read(lds + OPB, i, 0);
  }
  int st = 0;
  bool live = true;
  // Tiles of 128 rows leave it half of the accumulators' registers free: it moves them between two sets around the K loop, so there the instruction is
  // its own, whose latency it knows.
  auto mfma = [](f32x4& c, const u32x4& b, const u32x4& a) {
    if constexpr (MI <= 4) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
    else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
  };
  // The compiler knows nothing of the latency of an assembly instruction: this stands between the
  // matrix instructions and other reads or writes of their registers (more than the 19 wait
  // states that the longest of those dependencies wants).
  auto settle = [] { asm volatile("s_nop 15\n\ts_nop 15"); __builtin_amdgcn_sched_barrier(0); };
  // One K-tile: 128 slots of one matrix instruction, the rest placed between them (see above).
  constexpr int NR = MI + 8;                  // requests of a K-tile, fragments of half of it
  constexpr int kFree = NR + 8, kLanded = 16 * MI - 2 * NR - 8, kRequest = kFree + 1, kEvery = MI == 8 ? 6 : MI - 1;
  constexpr int kBefore = (kLanded - kRequest + kEvery - 1) / kEvery;        // requests made before kLanded
  static_assert(kFree <= 8 * MI && kLanded >= 8 * MI && kRequest + (NR - 1) * kEvery < 16 * MI, "slots of a K-tile");
  auto step = [&]() {
    const lds_byte* const here = lds + st * kW4Stage;
    const lds_byte* const there = lds + (st ^ 1) * kW4Stage;
    // formed here, ahead of the scheduling barrier, and first read kRequest matrix instructions on: far beyond the
    // five wait states that request_tile waits out
    const i32x4 da = ca.desc(live), db = cb.desc(live);
    const unsigned dst = wdst + (unsigned)(st * kW4Stage), dsta = adst + (unsigned)(st * kW4Stage);
    __builtin_amdgcn_sched_barrier(0);
    auto half = [&](auto first) {
      constexpr int t0 = decltype(first)::value;
#pragma unroll
      for (int q = 0; q < 8 * MI; ++q) {
        const int t = t0 + q, i = q % MI, j = q / MI;
        if constexpr (t0 == 0) mfma(acc[i][j], bx[j], ax[i]);
        else mfma(acc[i][j], by[j], ay[i]);
        if (t < MI) ay[t] = oa.read(here, t, 1);
        else if (t < NR) by[t - MI] = ob.read(here + OPB, t - MI, 1);
        if (t == kFree) {
          __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));                                       // lgkmcnt(0)
          __builtin_amdgcn_s_barrier();
        }
        if (t == kLanded) {
          __builtin_amdgcn_s_waitcnt((kBefore & 15) | (7 << 4) | (15 << 8) | ((kBefore >> 4) << 14));             // vmcnt(kBefore)
          __builtin_amdgcn_s_barrier();
        }
        if (t >= kRequest && (t - kRequest) % kEvery == 0 && (t - kRequest) / kEvery < NR) {
          const int r = (t - kRequest) / kEvery;
          if (r < MI) request(da, GROUPED ? oa.within(r, k_left) : oa.voff[r], dsta + (unsigned)(r * 1024));
          else request(db, GROUPED ? ob.within(r - MI, k_left) : ob.voff[r - MI], dst + (unsigned)(OPB + (r - MI) * 1024));
        }
        if (t >= kLanded && (t - kLanded) % 2 == 0 && t < kLanded + 2 * NR) {
          const int r = (t - kLanded) / 2;
          if (r < MI) ax[r] = oa.read(there, r, 0);
          else bx[r - MI] = ob.read(there + OPB, r - MI, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    half(std::integral_constant<int, 0>{});
    half(std::integral_constant<int, 8 * MI>{});
    ca.advance(astep);
    cb.advance(bstep);
    k_left -= 64;
    st ^= 1;
  };
  const __amdgpu_buffer_rsrc_t rc_all = make_rsrc(p.C, p.c_bytes), rc2 = make_rsrc(p.C2, p.C2 ? p.c2_bytes : 0u);
  const __amdgpu_buffer_rsrc_t rr = make_rsrc(p.R, !p.R ? 0u : EPI == W4_TABLE ? (uint32_t)(p.r_rows * p.ldc * 2) : p.c_bytes), rbias = make_rsrc(p.bias, p.bias ? (uint32_t)p.N * 2u : 0u);
  // W4_PIECES, K-contiguous A: where this lane's rows go; W4_SOFTMAX: their targets.  Requested ahead of the K loop: behind it they would wait for the requests of the
  // next item's K-tiles, and the epilogue for them (loss of 2450 tokens, 2048 x 50021, 455 -> 431 us).
  constexpr bool TO_ROWS = EPI == W4_PIECES && A_KC;
  constexpr int kOfRow = TO_ROWS ? 2 * MI : EPI == W4_SOFTMAX ? MI : 0;
  int of_row[kOfRow ? kOfRow : 1];
  while (true) {
#pragma unroll
    for (int i = 0; i < kOfRow; ++i) {
      const int row = wm + (EPI == W4_SOFTMAX ? 16 * i + (lane & 15) : 8 * i + (lane >> 3));
      of_row[i] = row < it.hi - it.lo - it.m0 ? p.rows[start + it.lo + it.m0 + row] : -1;
    }
    settle();
    for (int n = it.nk - 2; n > 0; --n) step();
    // the last K-tile of this item has been requested: the requests move on to the next item
    const unsigned entry = tq_claim_ahead(tq, qc);
    const int next = tq_next(tq, qc, entry, &mail);
    live = next >= 0;
    const Item nit = decode(live ? next : item);
    point(nit);
    for (int n = 2; n > 0; --n) step();
    settle();
    // Epilogue, 16 rows x 64 columns at a time through the patch, leaving row-contiguous.
    // acc[i][j][e] is output (row m0+wm+16i+lr, column n0+wn+16j+4g+e).
    {
      float* const patch = reinterpret_cast<float*>(smem + 2 * kW4Stage) + wave * (16 * kW4Pitch);
      int ln = lane;
      asm volatile("" : "+v"(ln));           // write-back offsets are formed here, not kept across the K loop
      // GROUPED: rows of C are counted from the tile's first
      const int m0 = GROUPED ? 0 : it.m0, rows = (A_KC ? it.hi - it.lo : p.M) - it.m0;
      const __amdgpu_buffer_rsrc_t rc = GROUPED ? make_rsrc(p.C + (A_KC ? (int64_t)(it.lo + it.m0) * p.ldc : it.g * p.stride + (int64_t)it.m0 * p.ldc),
                                                            (uint32_t)(((int64_t)(min(rows, 32 * MI) - 1) * p.ldc + (EPI == W4_SOFTMAX ? p.ldc : p.N)) * 2))
                                                : rc_all;
      const int elr = ln & 15, eg = ln >> 4;
      constexpr bool GU = EPI == W4_SWIGLU;
      // a lane writes 8 columns: of rows prow and prow + 8, or (SwiGLU) of gate, up and activation of row prow
      const int prow = GU ? ln >> 2 : ln >> 3, pcol = GU ? 32 * ((ln >> 1) & 1) + 8 * (ln & 1) : 8 * (ln & 7);
      auto out_col = [&](int h) { return GU ? (it.n0 >> 1) + ((wn + 64 * h) >> 1) + (pcol >> 5) * 16 + (pcol & 15) : it.n0 + wn + 64 * h + pcol; };
      const int ncols = GU ? p.gu_f : p.N;
      auto off = [&](int row, int col, int64_t ld, bool ok) -> int { return ok ? (int)(unsigned)(((int64_t)row * ld + col) * 2) : (int)kOob; };
      u32x4 bias_[2] = {}, bias_up[2] = {};
      constexpr bool HAS_BIAS = EPI != W4_PLAIN && EPI < W4_PIECES;
      if constexpr (HAS_BIAS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int col = out_col(h);
          bias_[h] = __builtin_amdgcn_raw_buffer_load_b128(rbias, col < ncols ? col * 2 : (int)kOob, 0, 0);
          if constexpr (GU) bias_up[h] = __builtin_amdgcn_raw_buffer_load_b128(rbias, col < ncols ? (col + p.gu_f) * 2 : (int)kOob, 0, 0);
        }
      }
      auto patch_sync = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      };
      // What is added to block b, requested RAHEAD blocks before: one block's stores and its way through the patch take less than the latency of
      // memory (a table of positions comes from the caches).  Forward with a residual, requested in its own block -> three ahead: 32768 x 4096 x 4096
      // 863 -> 822 us, 32768 x 11008 x 4096 2091 -> 2056, 12000 x 5120 x 1280 120.2 -> 117.3, 9216 x 1024 x 1024 24.4 -> 23.8.
      constexpr bool HAS_R = EPI == W4_RES || EPI == W4_TABLE;
      constexpr int RAHEAD = EPI == W4_RES ? 3 : EPI == W4_TABLE ? 1 : 0;
      u32x4 ring[RAHEAD + 1][2] = {};
      auto request_res = [&](int b) {
        const int col = out_col(b & 1);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int row = m0 + wm + 16 * (b >> 1) + prow + 8 * q;
          ring[b % (RAHEAD + 1)][q] = __builtin_amdgcn_raw_buffer_load_b128(rr, off(EPI == W4_TABLE ? table_row(row, p.r_rows, p.r_magic) : row, col, p.ldc, col < ncols), 0, 0);
        }
      };
      if constexpr (HAS_R) {
#pragma unroll
        for (int b = 0; b < RAHEAD; ++b) request_res(b);
      }
      // Groups of rows, no sums: 16 rows x 128 columns are rounded where they are and pass through two patches of 2 KB (64 columns each, rows of 128
      // bytes, 16-byte chunks XOR-swizzled by the row); they are stored once the next are worked on.
      if constexpr (GROUPED && (EPI == W4_PLAIN || EPI == W4_SOFTMAX || EPI == W4_PIECES)) {
        unsigned char* const half = reinterpret_cast<unsigned char*>(smem + 2 * kW4Stage) + wave * (64 * kW4Pitch);
        u32x4 leaving[2][2];
        const int last_col = EPI == W4_SOFTMAX ? (int)p.ldc : p.N;
        auto leave = [&](int b) {
          const int col = it.n0 + wn + 64 * (b & 1) + 8 * (ln & 7);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int row = wm + 16 * (b >> 1) + prow + 8 * q;
            if constexpr (TO_ROWS) {
              const int to = of_row[2 * (b >> 1) + q];
              if (col < last_col && to >= 0) *reinterpret_cast<u32x4*>(p.C + (int64_t)to * p.ldc + col) = leaving[b & 1][q];
            } else {
              __builtin_amdgcn_raw_buffer_store_b128(leaving[b & 1][q], rc, off(row, col, p.ldc, col < last_col), 0, 0);
            }
          }
        };
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          f32x4 v[2][4];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            // moved here and not before: left to itself the compiler moves all 256 accumulators at once, to registers that there are not
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float x;
              asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[i][j][e]));
              v[j >> 2][j & 3][e] = x;
            }
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
          if constexpr (EPI == W4_SOFTMAX) {
            const int row = wm + 16 * i + elr;
            w4_softmax(p, v, it.m0 + row, it.n0 + wn, eg, of_row[i], row < rows);
          }
          if (EPI == W4_PIECES && p.splits > 1) {        // a piece's sums, in fp32
            const int row = wm + 16 * i + elr, col = it.n0 + wn + 4 * eg;
            float* const at = p.sums + ((int64_t)it.split * p.M + (A_KC ? it.lo : 0) + it.m0 + row) * p.N + col;
#pragma unroll
            for (int j = 0; j < 8; ++j) if (row < rows && col + 16 * j < p.N) *reinterpret_cast<f32x4*>(at + 16 * j) = v[j >> 2][j & 3];
          } else if (EPI != W4_SOFTMAX || p.C) {
            if (i > 0) { leave(2 * i - 2); leave(2 * i - 1); }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int jj = 0; jj < 4; ++jj) {
                typedef typename std::conditional<EPI == W4_SOFTMAX, _Float16, bf16>::type E;
                typedef __attribute__((ext_vector_type(4))) E vec4;
                vec4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (E)(EPI == W4_SOFTMAX ? v[h][jj][e] : v[h][jj][e] * scale);
                *reinterpret_cast<vec4*>(half + 2048 * h + elr * 128 + (((2 * jj + (eg >> 1)) ^ (elr & 7)) << 4) + 8 * (eg & 1)) = o;
              }
            patch_sync();
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int q = 0; q < 2; ++q)
                leaving[h][q] = *reinterpret_cast<const u32x4*>(half + 2048 * h + (prow + 8 * q) * 128 + (((ln & 7) ^ (prow & 7)) << 4));
            patch_sync();
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (EPI == W4_PIECES ? p.splits == 1 : EPI != W4_SOFTMAX || p.C) { leave(2 * MI - 2); leave(2 * MI - 1); }
      } else {
      // W4_ADD: the sums so far, requested a block ahead
      float4 before[EPI == W4_ADD ? 2 : 1][2][2];
      auto sum_at = [&](int b, int q) -> float4* {
        const int row = it.m0 + wm + 16 * (b >> 1) + prow + 8 * q, col = out_col(b & 1);
        return row < p.M && col < ncols ? reinterpret_cast<float4*>(p.sums + (int64_t)row * p.N + col) : nullptr;
      };
      auto request_sums = [&](int b) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float4* at = p.first ? nullptr : sum_at(b, q);
#pragma unroll
          for (int u = 0; u < 2; ++u) before[b & 1][q][u] = at ? at[u] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      };
      if constexpr (EPI == W4_ADD) request_sums(0);
#pragma unroll
      for (int b = 0; b < 2 * MI; ++b) {
        const int i = b >> 1, h = b & 1, row0 = m0 + wm + 16 * i, col = out_col(h);
        const bool ok = col < ncols;
        if constexpr (HAS_R) if (b + RAHEAD < 2 * MI) request_res(b + RAHEAD);
        if constexpr (EPI == W4_ADD) if (b + 1 < 2 * MI) request_sums(b + 1);
        const u32x4* const res = ring[b % (RAHEAD + 1)];
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          f32x4& a = acc[i][4 * h + jj];
          *reinterpret_cast<float4*>(patch + elr * kW4Pitch + 16 * jj + 4 * eg) = make_float4(a[0], a[1], a[2], a[3]);
          a = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        patch_sync();
        auto row8 = [&](int r, int c, float* v) {
          const float4 x = *reinterpret_cast<const float4*>(patch + r * kW4Pitch + c), y = *reinterpret_cast<const float4*>(patch + r * kW4Pitch + c + 4);
          v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        };
        if constexpr (GU) {
          float gv[8], uv[8];
          row8(prow, pcol, gv);
          row8(prow, pcol + 16, uv);
          const bf16x8 bg = __builtin_bit_cast(bf16x8, bias_[h]), bu = __builtin_bit_cast(bf16x8, bias_up[h]);
          bf16x8 og, ou, oc;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            og[e] = (bf16)(gv[e] + (float)bg[e]);
            ou[e] = (bf16)(uv[e] + (float)bu[e]);
            oc[e] = (bf16)swiglu_f((float)og[e], (float)ou[e]);     // of the values as stored
          }
          const int row = row0 + prow;
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, og), rc, off(row, col, p.ldc, ok), 0, 0);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, ou), rc, off(row, col + p.gu_f, p.ldc, ok), 0, 0);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, oc), rc2, off(row, col, p.ldc2, ok), 0, 0);
        } else {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int row = row0 + prow + 8 * q;
            float v[8];
            row8(prow + 8 * q, pcol, v);
            if constexpr (EPI == W4_ADD) {
              const float4 x = before[b & 1][q][0], y = before[b & 1][q][1];
              const float old[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = (v[e] + old[e]) * (last ? scale : 1.f);
              if (!last) {
                if (float4* at = sum_at(b, q)) {
                  at[0] = make_float4(v[0], v[1], v[2], v[3]);
                  at[1] = make_float4(v[4], v[5], v[6], v[7]);
                }
                continue;
              }
            }
            const bf16x8 bv = __builtin_bit_cast(bf16x8, bias_[h]), rv = __builtin_bit_cast(bf16x8, res[q]);
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float x = v[e];
              if constexpr (HAS_BIAS) x += (float)bv[e];
              if constexpr (EPI == W4_RES || EPI == W4_TABLE) x += (float)rv[e];
              o[e] = (bf16)x;
            }
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rc, off(row, col, p.ldc, ok), 0, 0);
            if constexpr (EPI == W4_GELU || EPI == W4_TAPS) {
              bf16x8 a2;
#pragma unroll
              for (int e = 0; e < 8; ++e) a2[e] = (bf16)ErfTable::gelu(erf_table, (float)o[e]);     // of the value as stored
              const u32x4 av = __builtin_bit_cast(u32x4, a2);
              if constexpr (EPI == W4_TAPS) {
                const TapRows t = tap_rows(row, p.M, p.N, p.r_rows, p.r_magic);
                __builtin_amdgcn_raw_buffer_store_b128(av, rc2, ok && t.first >= 0 ? (int)(unsigned)((t.first + col) * 2) : (int)kOob, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b128(t.zero ? u32x4{0u, 0u, 0u, 0u} : av, rc2, ok && t.second >= 0 ? (int)(unsigned)((t.second + col) * 2) : (int)kOob, 0, 0);
              } else {
                __builtin_amdgcn_raw_buffer_store_b128(av, rc2, off(row, col, p.ldc2, ok), 0, 0);
              }
            }
          }
        }
        patch_sync();
      }
      }
    }
    if (!live) break;
    item = next;
    it = nit;
  }
  __builtin_amdgcn_s_waitcnt(0);
  tq_done(tq);
}

// prefer_queue: items of unequal cost (tile_queue.h)
template <bool A_KC, bool B_KC, int EPI, int MI = 8, int MAP = W4_WHOLE>
mosaic_status launch_w4_epi(hipStream_t s, int quota, const W4Args& p, bool prefer_queue = false) {
  auto kern = gemm_bf16_w4_kernel<A_KC, B_KC, EPI, MI, MAP>;
  static std::once_flag attr_once;
  static hipError_t attr_rc = hipSuccess;
  std::call_once(attr_once, [&] {
    attr_rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, w4_lds(EPI));
  });
  MOSAIC_HIP(attr_rc);
  TileQueueArgs tq;
  int grid;
  MOSAIC_TRY(tile_queue_plan(s, quota, 1, p.tile_count, 0, prefer_queue, &tq, &grid));
  kern<<<grid, 256, w4_lds(EPI), s>>>(p, tq);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}

}  // namespace
