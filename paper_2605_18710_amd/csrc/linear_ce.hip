// Softmax cross entropy behind a linear layer, without the logits: z_t = x_t table^T over the V rows of a table [V, h], and for every
// token whose target lies in the table
//   l_t = log sum_v exp(z_tv) - (1 - s) z_t,target - s mean_v z_tv          (s: label smoothing)
//   loss = sum l_t / D;  dz_tv = (softmax(z_t)_v - (1 - s) [v = target] - s / V) / D;  dX = dz table;  dtable = dz^T X
// with D given, or the number of such tokens.  The others take no part: their rows of X are not multiplied (they may hold anything).
//
//   1. The tokens that count are listed in order, and their rows copied side by side (list_kernel, place_kernel): how many there are
//      stays on the device, where the products' workgroups read it.
//   2. In pieces of tokens (kPieceElems): the product with the table, whose epilogue leaves exp(z - m) in fp16 and, for each row and 64 columns, the
//      largest logit m and the sum (w4_softmax in gemm_w4.h); or only these, when the loss alone is asked for.
//   3. lse_kernel joins a row's blocks to the largest logit, the sum and the loss; grad_kernel turns what lies there into dz, in place (and joins short rows itself).
//   4. dX = dz table, into the rows of X that the tokens came from; dtable = dz^T X, summed in fp32 over the pieces.
// So the gradients take three products of 2 T h V operations, where pieces of the vocabulary would want the logits twice: their softmax needs the whole
// row.  Few tokens or a small table: the products by few_tile.  fp32: the same on fp32 logits, in rows that a workgroup or a wave holds (rows_f32_kernel), or in blocks
// of columns that lse_kernel joins (wide_f32_kernel).
//
// What bounds it: the matrix cores.  12288 tokens that count of 16384, h 4096, V 128000, bf16: 29.5 ms, 1.31 PFLOP/s over all; the pass over the logits in
// step 3 takes 1.35 ms of it at 4.7 TB/s.  Of one token or a few: the table's bytes (few_kernel).  Of small workloads: four to seven launches.
//
// All sums have an order that the sizes and the targets fix.
#include "gemm_few.h"
#include "gemm_plan.h"
#include "gemm_w4.h"
#include "kernels.h"

namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// ------------------------------------------------------------------------- the tokens that count
struct CeHead { int count; float per_token; };      // their number, and 1 / D
struct CeSpan { int zero, live, start, last; };     // of a piece: 0, how many tokens it has, the first of them, whether none follow

struct CeList {
  const int32_t* targets;
  int T, V, piece, pieces;
  float denom;
  int balanced;            // pieces of equal size, as few as hold the tokens (else `piece` tokens each)
  CeHead* head;
  CeSpan* spans;
  int32_t *rows, *target;  // in order: the token, and its target
  int32_t* slot;           // of a token: its place in that order, or -1
};

// One workgroup: 16 waves in order, 512 tokens of a turn each, eight to a lane (with one to a lane a barrier for every 1024 tokens: 15 us of 14313, now 7).
// `write`: to memory; each(t, at) for every token a thread looks at, at < 0 where it does not count.
constexpr int kListThreads = 1024, kListEach = 8;
template <typename F>
__device__ __forceinline__ void list_tokens(const CeList& l, bool write, F each) {
  constexpr int kWaves = kListThreads / 64;
  __shared__ int wave_count[2][kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int run = 0, y[kListEach];
  auto look = [&](int t0) {
#pragma unroll
    for (int j = 0; j < kListEach; ++j) {
      const int64_t t = (int64_t)t0 + 64 * (kListEach * wave + j) + lane;
      y[j] = t < l.T ? l.targets[t] : -1;
    }
  };
  look(0);
  for (int64_t t0 = 0, turn = 0; t0 < l.T; t0 += kListThreads * kListEach, turn ^= 1) {
    int here[kListEach], mine[kListEach], all = 0;       // tokens of the wave that count: before the lane's own, all
#pragma unroll
    for (int j = 0; j < kListEach; ++j) {
      here[j] = y[j] >= 0 && y[j] < l.V ? y[j] : -1;
      const unsigned long long m = __ballot(here[j] >= 0);
      mine[j] = all + __popcll(m & ((1ull << lane) - 1ull));
      all += __popcll(m);
    }
    look((int)min(t0 + kListThreads * kListEach, (int64_t)l.T));         // its latency passes under this turn
    if (lane == 0) wave_count[turn][wave] = all;
    __syncthreads();                             // the other half of wave_count was read before the barrier of the turn before
    int before = run;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int n = wave_count[turn][w];
      if (w < wave) before += n;
      run += n;
    }
#pragma unroll
    for (int j = 0; j < kListEach; ++j) {
      const int64_t t = t0 + 64 * (kListEach * wave + j) + lane;
      const int at = here[j] >= 0 ? before + mine[j] : -1;
      if (write && at >= 0) { l.rows[at] = (int)t; l.target[at] = here[j]; }
      if (t < l.T) each((int)t, at);
    }
  }
  if (!write) return;
  const int n = l.balanced ? max(1, (int)(((int64_t)run + l.piece - 1) / l.piece)) : l.pieces;
  const int size = l.balanced ? min(l.piece, ((run + n - 1) / n + 255) / 256 * 256) : l.piece;
  for (int p = threadIdx.x; p < l.pieces; p += kListThreads) {
    const int start = (int)min((int64_t)p * size, (int64_t)run);
    l.spans[p] = {0, p < n ? min(size, run - start) : 0, start, p == n - 1};
  }
  if (threadIdx.x == 0) *l.head = {run, l.denom > 0.f ? 1.f / l.denom : run ? 1.f / (float)run : 0.f};
}

// A token's row of X to its place, or zeros to its gradient and loss; by one wave
template <typename T, int V>
__device__ __forceinline__ void place_row(int64_t t, int at, const T* X, int64_t h, T* Xc, T* dX, float* losses) {
  typedef typename Pack<T, V>::type vec;
  const int lane = threadIdx.x & 63;
  if (at >= 0) {
    for (int64_t c = lane * V; c < h; c += 64 * V) *reinterpret_cast<vec*>(Xc + at * h + c) = *reinterpret_cast<const vec*>(X + t * h + c);
  } else {
    if (dX) for (int64_t c = lane * V; c < h; c += 64 * V) *reinterpret_cast<vec*>(dX + t * h + c) = vec{};
    if (lane == 0) losses[t] = 0.f;
  }
}
__global__ __launch_bounds__(kListThreads) void list_kernel(CeList l) {
  list_tokens(l, true, [&](int t, int at) { l.slot[t] = at; });
}
template <typename T, int V>
__global__ __launch_bounds__(256) void place_kernel(const int32_t* __restrict__ slot, int tokens, const T* __restrict__ X, int64_t h, T* __restrict__ Xc,
                                                    T* __restrict__ dX, float* __restrict__ losses) {
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < tokens; t += (int64_t)gridDim.x * 4) place_row<T, V>(t, slot[t], X, h, Xc, dX, losses);
}
// Both in one launch up to kListMax tokens: every workgroup makes the list for itself (one turn, where a launch takes four microseconds), the first one
// writes it.
constexpr int kListMax = 8192;
template <typename T, int V>
__global__ __launch_bounds__(kListThreads) void list_place_kernel(CeList l, const T* __restrict__ X, int64_t h, T* __restrict__ Xc, T* __restrict__ dX,
                                                                  float* __restrict__ losses) {
  __shared__ int slot[kListMax];
  list_tokens(l, blockIdx.x == 0, [&](int t, int at) { slot[t] = at; });
  __syncthreads();
  for (int t = blockIdx.x * 16 + (threadIdx.x >> 6); t < l.T; t += gridDim.x * 16) place_row<T, V>(t, slot[t], X, h, Xc, dX, losses);
}

// -------------------------------------------------------------------------- rows of the softmax
struct CePiece {
  const CeSpan* span;
  const int32_t *rows, *target;      // of all tokens
  const float* at_target;
  int capacity, V;
  float smoothing;
  float *top, *inverse;        // of each row: the largest logit, which the sum's exponentials are relative to, and 1 / the sum
  float* losses;
};

// (m, sum) of two sets of columns.  One of which nothing has come, or nothing but -infinity, has m = -infinity and adds its sum, 0 or NaN; infinities and NaN go into the
// sum as they are
__device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ void join_sums(float& top, float& sum, float m, float s) {
  const float before = top;
  top = fmaxf(top, m);
  const float ref = reference(top);
  sum = sum * exp_of(before - ref) + s * exp_of(m - ref);
}
// A row's (m, sum) and totals over its blocks, by 64 groups of 16 lanes, a lane to a row; in the first group on return.
struct RowSums { float (*top)[16], (*sum)[16], (*total)[16]; };       // [16][16] each, in LDS
__device__ __forceinline__ void row_sums(const float2* stats, const float* totals, int blocks, int64_t pitch, int row, RowSums lds, float& top, float& sum, float& total) {
  const int r = threadIdx.x & 15, wave = threadIdx.x >> 6;
  top = -INFINITY; sum = 0.f; total = 0.f;
  for (int b0 = threadIdx.x >> 4; b0 < blocks; b0 += 64 * 8) {
    float2 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = b0 + 64 * u < blocks ? stats[(b0 + 64 * u) * pitch + row] : make_float2(-INFINITY, 0.f);
    float high = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) high = fmaxf(high, v[u].x);
    if (high != top) { sum *= exp_of(top - high); top = high; }
    const float ref = reference(top);
#pragma unroll
    for (int u = 0; u < 8; ++u) if (b0 + 64 * u < blocks) sum = fmaf(v[u].y, exp_of(v[u].x - ref), sum);
    if (totals) {
#pragma unroll
      for (int u = 0; u < 8; ++u) if (b0 + 64 * u < blocks) total += totals[(b0 + 64 * u) * pitch + row];
    }
  }
#pragma unroll
  for (int o = 16; o < 64; o <<= 1) {
    const float m = __shfl_xor(top, o, 64), s = __shfl_xor(sum, o, 64);
    // in the same order on both sides
    if (threadIdx.x & o) { float a = m, b = s; join_sums(a, b, top, sum); top = a; sum = b; }
    else join_sums(top, sum, m, s);
    total += __shfl_xor(total, o, 64);
  }
  if ((threadIdx.x & 63) < 16) { lds.top[wave][r] = top; lds.sum[wave][r] = sum; lds.total[wave][r] = total; }
  __syncthreads();
  if (threadIdx.x < 16) {
#pragma unroll
    for (int w = 1; w < 16; ++w) { join_sums(top, sum, lds.top[w][r], lds.sum[w][r]); total += lds.total[w][r]; }
  }
  __syncthreads();
}
// differences of logits first: next to them the logarithm keeps its digits
__device__ __forceinline__ float token_loss(float top, float sum, float at_target, float total, float smoothing, int V) {
  float ahead = fmaf(-(1.f - smoothing), at_target, top);
  if (smoothing > 0.f) ahead -= smoothing * (total / (float)V);
  return ahead + logf(sum);
}

// 16 rows to a workgroup: their statistics lie side by side.
__global__ __launch_bounds__(1024) void lse_kernel(CePiece p, const float2* __restrict__ stats, const float* __restrict__ totals, int blocks) {
  __shared__ float top_of[16][16], sum_of[16][16], total_of[16][16];
  const int live = p.span->live, start = p.span->start;
  for (int r0 = blockIdx.x * 16; r0 < live; r0 += gridDim.x * 16) {
    const int row = r0 + (threadIdx.x & 15);     // below capacity, a multiple of 16
    float top, sum, total;
    row_sums(stats, totals, blocks, p.capacity, row, {top_of, sum_of, total_of}, top, sum, total);
    if (threadIdx.x < 16 && row < live) {
      p.top[row] = top;
      p.inverse[row] = 1.f / sum;
      p.losses[p.rows[start + row]] = token_loss(top, sum, p.at_target[row], total, p.smoothing, p.V);
    }
  }
}

// exp(z - m) in fp16 -> D dz in bf16, in place (the products' results are divided by D: a target of small probability, the largest term of its row, is then
// -1 and not rounded at all): a strip of 16 rows and 1024 columns to a workgroup, 16 bytes to a lane and row pair.  PAST: tensors that no cache holds.
// LO: what that rounding leaves goes behind it, `lo` elements on.  The rounding of dz is one error of up to half a step beside the results' own; over many
// values it makes sqrt(2) of the plain form's error, over the few of a small vocabulary and few tokens up to 2.1 times (1 x 64 to 64 x 3), and of up to 16 tokens
// up to 2.2 times whatever the vocabulary, where it is cheap to take it away.
constexpr int kStrip = 1024;
constexpr int kLowTokens = 512, kLowColumns = 512, kFewRows = 16;
template <bool PAST, bool JOIN, bool LO>
__global__ __launch_bounds__(256, 4) void grad_kernel(CePiece p, const float2* __restrict__ stats, const float* __restrict__ totals, bf16* __restrict__ E, int64_t ld, int64_t lo) {
  // JOIN: every workgroup joins its rows' blocks itself, of which there are at most kJoinBlocks, and no launch does before
  __shared__ float top_of[4][16], sum_of[4][16], total_of[4][16], row_top[16], row_inverse[16];
  const int live = p.span->live, start = p.span->start, strips = (int)((ld + kStrip - 1) / kStrip);
  const float even = p.smoothing / (float)p.V;
  const int64_t items = (int64_t)((live + 15) / 16) * strips;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int r0 = (int)(item / strips) * 16, c0 = (int)(item % strips) * kStrip;
    const int col = c0 + 8 * (threadIdx.x & 127);
    f16x8 v[8];
    float scale[8], top_of_row[8], inverse[8];
    int hit[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = r0 + 2 * i + (threadIdx.x >> 7);
      if (row >= live || col >= ld) continue;
      v[i] = load_from<PAST>(reinterpret_cast<const f16x8*>(E + (int64_t)row * ld + col));
      if constexpr (!JOIN) { top_of_row[i] = p.top[row]; inverse[i] = p.inverse[row]; }
      scale[i] = stats[(int64_t)(col / kCeBlock) * p.capacity + row].x;
      hit[i] = p.target[start + row] - col;
    }
    float own[8];                                // the target's logit, where a lane has its column: all asked for before the first is waited for
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = r0 + 2 * i + (threadIdx.x >> 7);
      own[i] = 0.f;
      if (row < live && col < ld && hit[i] >= 0 && hit[i] < 8) own[i] = p.at_target[row];
    }
    if constexpr (JOIN) {
      const int r = threadIdx.x & 15, wave = threadIdx.x >> 6, row = r0 + r, blocks = (p.V + kCeBlock - 1) / kCeBlock;
      const bool tells = c0 == 0 && threadIdx.x < 16 && row < live;        // the rows' losses
      int token = 0;
      float at_target = 0.f;
      if (tells) { token = p.rows[start + row]; at_target = p.at_target[row]; }
      float top = -INFINITY, sum = 0.f, total = 0.f;
#pragma unroll 4
      for (int b = threadIdx.x >> 4; b < blocks; b += 16) {
        const float2 x = stats[(int64_t)b * p.capacity + row];
        join_sums(top, sum, x.x, x.y);
        if (totals) total += totals[(int64_t)b * p.capacity + row];
      }
#pragma unroll
      for (int o = 16; o < 64; o <<= 1) {
        const float m = __shfl_xor(top, o, 64), s = __shfl_xor(sum, o, 64);
        join_sums(top, sum, m, s);
        total += __shfl_xor(total, o, 64);
      }
      if ((threadIdx.x & 63) < 16) { top_of[wave][r] = top; sum_of[wave][r] = sum; total_of[wave][r] = total; }
      __syncthreads();
      if (threadIdx.x < 16) {
#pragma unroll
        for (int w = 1; w < 4; ++w) { join_sums(top, sum, top_of[w][r], sum_of[w][r]); total += total_of[w][r]; }
        row_top[r] = top;
        row_inverse[r] = 1.f / sum;
        if (tells) p.losses[token] = token_loss(top, sum, at_target, total, p.smoothing, p.V);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) { top_of_row[i] = row_top[2 * i + (threadIdx.x >> 7)]; inverse[i] = row_inverse[2 * i + (threadIdx.x >> 7)]; }
      __syncthreads();                           // read before the next strip's rows are joined
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = r0 + 2 * i + (threadIdx.x >> 7);
      if (row >= live || col >= ld) continue;
      const float f = exp_of(scale[i] - top_of_row[i]) * inverse[i];
      Vec16<bf16> o, rest;
      auto set = [&](int e, float x) {
        o.set(e, x);
        if constexpr (LO) rest.set(e, x - o.get(e));
      };
#pragma unroll
      for (int e = 0; e < 8; ++e) set(e, col + e < p.V ? (float)v[i][e] * f - even : 0.f);
      if (hit[i] >= 0 && hit[i] < 8) {
        // the target's probability from its own logit: 1 - p keeps its digits where p is near 1
        const float d = (exp_of(own[i] - top_of_row[i]) * inverse[i] - 1.f) + (p.smoothing - even);
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e == hit[i]) set(e, d);
      }
      if constexpr (LO) rest.store<PAST>(E + lo + (int64_t)row * ld + col);
      o.store<PAST>(E + (int64_t)row * ld + col);
    }
  }
}
constexpr int kJoinBlocks = 64;                    // 16 rows' statistics are then no more than a quarter of what a strip reads

__device__ __forceinline__ float block_reduce(float x, bool max, float* lds) {
  x = max ? wave_max(x) : wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return max ? fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3])) : (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// fp32 logits, a workgroup (NT 256) or a wave (64) to a row of up to 4 NT PER of them, which it holds: loss and (grad) dz in place.  8969 rows of 2667: 46 us (4.1 TB/s);
// by single words, in registers for 8192, 105.
template <int NT, int PER>
__global__ __launch_bounds__(NT) void rows_f32_kernel(CePiece p, const CeHead* __restrict__ head, float* __restrict__ Z, int64_t ld, int grad) {
  __shared__ float lds[4];
  const int live = p.span->live, start = p.span->start;
  const float g = head->per_token, even = p.smoothing / (float)p.V;
  auto reduce = [&](float x, bool max) { return NT == 64 ? (max ? wave_max(x) : wave_sum(x)) : block_reduce(x, max, lds); };
  for (int row = blockIdx.x; row < live; row += gridDim.x) {
    float* const z = Z + row * ld + 4 * threadIdx.x;           // rows of whole 16-byte pieces, with room up to ld
    const int target = p.target[start + row], last = p.V - 4 * threadIdx.x;
    f32x4 v[PER];
    float top = -INFINITY, total = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (4 * NT * i < last) v[i] = *reinterpret_cast<const f32x4*>(z + 4 * NT * i);
    }
    const float at_target = Z[row * ld + target];
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = 4 * NT * i + e < last;
        if (!in) v[i][e] = -INFINITY;
        top = fmaxf(top, v[i][e]);
        total += in ? v[i][e] : 0.f;
      }
    top = reduce(top, true);
    if (p.smoothing > 0.f) total = reduce(total, false);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[i][e] = expf(v[i][e] - ref);
        sum += v[i][e];
      }
    sum = reduce(sum, false);
    __syncthreads();                             // the target's logit has been read by all
    if (threadIdx.x == 0) p.losses[p.rows[start + row]] = token_loss(ref, sum, at_target, total, p.smoothing, p.V);
    if (!grad) continue;
    const float inverse = 1.f / sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (4 * NT * i >= last) continue;
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float q = v[i][e] * inverse;
        o[e] = 4 * NT * i + e >= last ? 0.f : g * (4 * (NT * i + (int)threadIdx.x) + e == target ? (q - 1.f) + (p.smoothing - even) : q - even);      // the products read whole pieces
      }
      *reinterpret_cast<f32x4*>(z + 4 * NT * i) = o;
    }
  }
}
// Longer rows: (m, sum) of blocks of kWideBlock columns, joined by lse_kernel, and dz in place, a workgroup to a block
constexpr int kWideRow = 8192, kWideBlock = 4096;
template <bool GRAD>
__global__ __launch_bounds__(256) void wide_f32_kernel(CePiece p, const CeHead* __restrict__ head, float* __restrict__ Z, int64_t ld, float2* __restrict__ stats,
                                                       float* __restrict__ totals, float* __restrict__ at_target) {
  __shared__ float lds[4];
  constexpr int PER = kWideBlock / 1024;
  const int live = p.span->live, start = p.span->start, blocks = (p.V + kWideBlock - 1) / kWideBlock;
  const float g = GRAD ? head->per_token : 0.f, even = p.smoothing / (float)p.V;
  for (int64_t item = blockIdx.x; item < (int64_t)live * blocks; item += gridDim.x) {
    const int row = (int)(item / blocks), block = (int)(item - (int64_t)row * blocks), c0 = block * kWideBlock + 4 * threadIdx.x;
    float* const z = Z + row * ld + c0;          // rows of whole 16-byte pieces
    const int target = p.target[start + row] - c0;
    f32x4 v[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (c0 + 1024 * i < p.V) v[i] = *reinterpret_cast<const f32x4*>(z + 1024 * i);
    }
    const float base = GRAD ? p.top[row] : 0.f, inverse = GRAD ? p.inverse[row] : 0.f;
    float top = -INFINITY, total = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 1024 * i + e;
        if (GRAD) {
          const float q = exp_of(v[i][e] - base) * inverse;
          v[i][e] = c0 + c >= p.V ? 0.f : g * (c == target ? (q - 1.f) + (p.smoothing - even) : q - even);      // the products read whole 16-byte pieces
        } else {
          if (c0 + c >= p.V) v[i][e] = -INFINITY;
          else total += v[i][e];
          if (c == target) at_target[row] = v[i][e];
          top = fmaxf(top, v[i][e]);
        }
      }
      if (GRAD && c0 + 1024 * i < p.V) *reinterpret_cast<f32x4*>(z + 1024 * i) = v[i];       // past the row's end there is room up to ld
    }
    if constexpr (!GRAD) {
      top = block_reduce(top, true, lds);
      const float ref = reference(top);
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += exp_of(v[i][e] - ref);
      sum = block_reduce(sum, false, lds);
      if (totals) total = block_reduce(total, false, lds);
      if (threadIdx.x == 0) {
        stats[(int64_t)block * p.capacity + row] = make_float2(top, sum);
        if (totals) totals[(int64_t)block * p.capacity + row] = total;
      }
    }
  }
}

// ------------------------------------------------------------- the products by few_tile
// What the four-wave kernel makes of the same arguments (W4_SOFTMAX; dX to the tokens' rows; dtable), for few tokens, short rows or small tables.
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppMirror8 = 0x141;      // the last one gives the other four lanes' where all four have the same
template <int CTRL> __device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true)); }
template <typename F> __device__ __forceinline__ float across_eight(float x, F f) {
  x = f(x, dpp<kDppXor1>(x));
  x = f(x, dpp<kDppXor2>(x));
  return f(x, dpp<kDppMirror8>(x));
}
template <int RB>
__global__ __launch_bounds__(kFewNT, few_waves(RB)) void few_logits_kernel(W4Args p) {
  extern __shared__ __align__(16) unsigned char smem[];
  auto add = [](float a, float b) { return a + b; };
  auto high = [](float a, float b) { return fmaxf(a, b); };
  const int live = p.offsets[1], start = p.piece[0], tiles_m = (live + 16 * RB - 1) / (16 * RB);
  const int64_t items = (int64_t)tiles_m * ((p.N + 63) / 64);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int n0 = (int)(item / tiles_m) * 64, m0 = (int)(item % tiles_m) * 16 * RB;
    few_tile<true, true, RB>(p.A + (int64_t)start * p.lda, p.lda, m0, live, p.B, p.ldb, n0, p.N, p.K, smem, [&](int row, int col, float (&v)[8]) {
      const bool in = row < live, first = in && (threadIdx.x & 7) == 0;
      const int hit = (in ? p.rows[start + row] : -1) - col;
      const int64_t slot = (int64_t)(col / kCeBlock) * p.M + row;
      float total = 0.f, m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e == hit) p.at_target[row] = v[e];
        total += v[e];                           // rows of the table past its end count as zeros
        v[e] = col + e < p.N ? v[e] : -INFINITY;
        m = fmaxf(m, v[e]);
      }
      if (p.totals) {
        total = across_eight(total, add);
        if (first) p.totals[slot] = total;
      }
      m = across_eight(m, high);
      const float ref = reference(m);
      f16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = exp_of(v[e] - ref);
        sum += x;
        o[e] = (_Float16)x;
      }
      sum = across_eight(sum, add);
      if (first) p.stats[slot] = make_float2(m, sum);
      if (p.C && in && col < p.ldc) *reinterpret_cast<f16x8*>(p.C + (int64_t)row * p.ldc + col) = o;
    });
  }
}
// loss = sum of the tokens' / D, by one workgroup of NT threads: every thread its tokens in ascending order, in 64 bits
struct CeLoss { const float* losses; int T; const CeHead* head; float* loss; };
template <int NT>
__device__ __forceinline__ void add_losses(const CeLoss& l, double* part) {
  double sum = 0.0;
  for (int64_t t0 = threadIdx.x; t0 < l.T; t0 += 8 * NT) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = t0 + u * NT < l.T ? l.losses[t0 + u * NT] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += (double)v[u];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) sum += part[w];
    *l.loss = (float)(sum * (double)l.head->per_token);
  }
  __syncthreads();
}
// dX, and (TABLE) dtable in the same launch: 375 x 33 of 72: two launches 11.7 us, one 7.6.  The last workgroup also adds the losses, where there are no more
// pieces (loss not null).
template <bool LO>
__device__ __forceinline__ void few_dtable(const W4Args& p, int64_t item, unsigned char* smem, int64_t lo) {
  const int live = p.offsets[1], start = p.piece[0], cols = (p.N + 63) / 64, m0 = (int)(item / cols) * 64, n0 = (int)(item % cols) * 64;
  const float scale = *p.scale;
  few_tile<false, false, 4, LO>(p.A, p.lda, m0, p.M, p.B + (int64_t)start * p.ldb, p.ldb, n0, p.N, live, smem, [&](int row, int col, const float (&v)[8]) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16)(v[e] * scale);
    if (row < p.M && col < p.N) *reinterpret_cast<bf16x8*>(p.C + (int64_t)row * p.ldc + col) = o;
  }, lo);
}
constexpr int kBothItems = 512;
__device__ __host__ __forceinline__ int64_t few_dtable_items(int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 63) / 64); }
template <int RB, bool TABLE, bool LO>
__global__ __launch_bounds__(kFewNT, TABLE || LO ? 2 : few_waves(RB)) void few_dx_kernel(W4Args p, CeLoss l, W4Args w, int64_t lo) {
  extern __shared__ __align__(16) unsigned char smem[];
  if (l.loss && blockIdx.x == gridDim.x - 1) add_losses<kFewNT>(l, reinterpret_cast<double*>(smem));
  const int live = p.offsets[1], start = p.piece[0], tiles_m = (live + 16 * RB - 1) / (16 * RB);
  const float scale = *p.scale;
  const int64_t first = TABLE ? few_dtable_items(w.M, w.N) : 0, items = first + (int64_t)tiles_m * ((p.N + 63) / 64);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    if (TABLE && item < first) {                 // their contraction is the longer one as a rule
      few_dtable<LO>(w, item, smem, lo);
      continue;
    }
    const int n0 = (int)((item - first) / tiles_m) * 64, m0 = (int)((item - first) % tiles_m) * 16 * RB;
    few_tile<true, false, RB, LO>(p.A, p.lda, m0, live, p.B, p.ldb, n0, p.N, p.K, smem, [&](int row, int col, const float (&v)[8]) {
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (bf16)(v[e] * scale);
      if (row < live && col < p.N) *reinterpret_cast<bf16x8*>(p.C + (int64_t)p.rows[start + row] * p.ldc + col) = o;
    }, lo);
  }
}
template <bool LO>
__global__ __launch_bounds__(kFewNT) void few_dtable_kernel(W4Args p, int64_t lo) {
  extern __shared__ __align__(16) unsigned char smem[];
  for (int64_t item = blockIdx.x; item < few_dtable_items(p.M, p.N); item += gridDim.x) few_dtable<LO>(p, item, smem, lo);
}
// Up to 16 tokens: a piece of the vocabulary to a workgroup, sums [pieces][16][N] for join_kernel.  5 x 424, V 117715 (100 MB): 33 us
__global__ __launch_bounds__(kFewNT) void few_dx_pieces_kernel(W4Args p, int64_t lo, int per) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int live = p.offsets[1], cols = (p.N + 63) / 64, pieces = (p.K + per - 1) / per;
  if (live == 0) return;
  for (int item = blockIdx.x; item < pieces * cols; item += gridDim.x) {
    const int piece = item / cols, n0 = (item - piece * cols) * 64, k0 = piece * per;
    float* const out = p.sums + (int64_t)piece * kFewRows * p.N;
    few_tile<true, false, 1, true>(p.A + k0, p.lda, 0, live, p.B + (int64_t)k0 * p.ldb, p.ldb, n0, p.N, min(per, p.K - k0), smem, [&](int row, int col, const float (&v)[8]) {
      if (col >= p.N) return;
      *reinterpret_cast<f32x4*>(out + (int64_t)row * p.N + col) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(out + (int64_t)row * p.N + col + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }, lo);
  }
}
// dtable of up to 16 tokens: dz and what its rounding left are the 32 k-values of one matrix instruction for 16 x 16 results, so the stores are the time.  The tokens'
// rows of X for 1024 columns lie in LDS, [column][token]; a wave takes 16 rows of the table at a time.  16 tokens, 32000 x 4096: 74 us (3.5 TB/s).
constexpr int kOuterColumns = 1024;
constexpr int outer_at(int c) { return c * 32 + (c >> 4) * 128; }          // byte of a column in LDS: 16 columns apart means 32 banks apart
__global__ __launch_bounds__(256) void few_outer_kernel(W4Args p, int64_t lo) {
  __shared__ __align__(16) unsigned char lds[outer_at(kOuterColumns)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, g = lane >> 4, live = p.offsets[1];
  const int chunks = (p.N + kOuterColumns - 1) / kOuterColumns, tiles = (p.M + 15) / 16, grid = (int)gridDim.x;
  const float scale = *p.scale;
  for (int chunk = (int)blockIdx.x % chunks; chunk < chunks; chunk += grid) {
    const int c0 = chunk * kOuterColumns, columns = min(kOuterColumns, p.N - c0);
    const int first = (int)blockIdx.x / chunks, step = max(1, (grid - chunk + chunks - 1) / chunks);
    __syncthreads();                               // the chunk before has been read
    for (int i = threadIdx.x; i < kFewRows * (kOuterColumns / 8); i += 256) {
      const int t = i / (kOuterColumns / 8), c = i % (kOuterColumns / 8) * 8;
      bf16x8 v = {};
      if (t < live && c < columns) v = *reinterpret_cast<const bf16x8*>(p.B + (int64_t)t * p.ldb + c0 + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) *reinterpret_cast<bf16*>(lds + outer_at(c + e) + 2 * t) = v[e];
    }
    __syncthreads();
    for (int tile = first * 4 + wave; tile < tiles; tile += step * 4) {
      const int row = 16 * tile + lr;
      bf16x8 x;                                    // k-values 8 g ..: tokens 8 (g % 2) .. of dz (g < 2) or of the rest
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = 8 * (g & 1) + e;
        x[e] = (bf16)0.f;
        if (t < live && row < p.M) x[e] = p.A[(g >> 1) * lo + (int64_t)t * p.lda + row];
      }
      for (int c = 0; c < columns; c += 64) {
        f32x4 acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {              // columns 16 i / 4 + 4 j + i % 4, i = 0 .. 15: a lane's results are sixteen columns side by side
          const bf16x8 y = *reinterpret_cast<const bf16x8*>(lds + outer_at(c + 16 * (lr >> 2) + 4 * j + (lr & 3)) + 16 * (g & 1));
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int col = c + 16 * g + 8 * half;
          bf16x8 o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = (bf16)(acc[2 * half + (e >> 2)][e & 3] * scale);
          if (row < p.M && col < columns) *reinterpret_cast<bf16x8*>(p.C + (int64_t)row * p.ldc + c0 + col) = o;
        }
      }
    }
  }
}
template <int RB>
mosaic_status launch_few_logits(hipStream_t s, int quota, int most, const W4Args& p) {
  static std::once_flag once;
  static hipError_t rc = hipSuccess;
  constexpr int kLds = few_lds<true, true, RB>();
  MOSAIC_TRY(few_allow_lds(few_logits_kernel<RB>, kLds, &once, &rc));
  few_logits_kernel<RB><<<grid_for(quota, RB == 1 ? 2 : 1, ceil_div(most, 16 * RB) * ceil_div(p.N, 64)), kFewNT, kLds, s>>>(p);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}
template <int RB, bool TABLE, bool LO>
mosaic_status launch_few_dx(hipStream_t s, int quota, int most, const W4Args& p, const CeLoss& l, const W4Args& w, int64_t lo) {
  static std::once_flag once;
  static hipError_t rc = hipSuccess;
  constexpr int kLds = std::max(few_lds<true, false, RB>(), TABLE ? few_lds<false, false, 4>() : 0);
  MOSAIC_TRY(few_allow_lds(few_dx_kernel<RB, TABLE, LO>, kLds, &once, &rc));
  const int64_t items = ceil_div(most, 16 * RB) * ceil_div(p.N, 64) + (TABLE ? few_dtable_items(w.M, w.N) : 0);
  few_dx_kernel<RB, TABLE, LO><<<grid_for(quota, RB == 1 && !TABLE && !LO ? 2 : 1, items), kFewNT, kLds, s>>>(p, l, w, lo);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}
template <bool LO>
mosaic_status launch_few_dtable(hipStream_t s, int quota, const W4Args& w, int64_t lo) {
  static std::once_flag once;
  static hipError_t rc = hipSuccess;
  constexpr int kLds = few_lds<false, false, 4>();
  MOSAIC_TRY(few_allow_lds(few_dtable_kernel<LO>, kLds, &once, &rc));
  few_dtable_kernel<LO><<<grid_for(quota, 1, few_dtable_items(w.M, w.N)), kFewNT, kLds, s>>>(w, lo);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}
// row blocks of 16 that a product of `most` rows is computed in, or 0 where it costs `other` at most
inline int few_rows(int64_t most, int64_t N, int64_t K, double other) {
  int best = 0;
  for (int blocks = 1; blocks <= 4; blocks *= 2) {
    const double us = few_price((double)(ceil_div(most, 16 * blocks) * ceil_div(N, 64)), (double)K, blocks, blocks == 1);
    if (us < other) { other = us; best = blocks; }
  }
  return best;
}

// ------------------------------------------------------------------------- a few tokens
// The loss alone of up to 16 tokens (a scored continuation, the single token of a serving step): the table is read once, and that is the time.  Every
// wave takes 16 of its rows at a time straight into registers, 64 k-values of each (whole 128-byte lines, 32 bytes to a lane) in two matrix instructions
// whose second operand are the tokens, which lie in LDS; what leaves is (m, sum) of the 16 rows for every token.  Eight steps are requested ahead,
// eight waves to a CU: 32 MB in flight.  One token, h 4096, V 32000 (262 MB): 52.5 us (5.0 TB/s), by the four-wave kernel in tiles of 128 rows 94.
constexpr int kFew = 16, kFewThreads = 512, kFewAhead = 8;
constexpr int kFewLds = 150 << 10;
inline int few_pitch(int64_t h) { return (int)(align_up((size_t)h, 64) * 2 + 16); }      // bytes of a token in LDS: 16 past whole steps, so that 16 rows touch every bank
struct CeFew {
  const int32_t* targets;
  const bf16 *X, *table;
  int T, h, V, pitch;
  float smoothing, denom;
  float2* stats;           // [kFew][ceil(V / 16)]
  float *totals, *at_target;
  float *losses, *loss;
};
// lane t's target, its place among the tokens that count (-1: none); *live: their number.  T <= kFew
__device__ __forceinline__ int few_place(const CeFew& p, int lane, int* y, int* live) {
  *y = lane < p.T ? p.targets[lane] : -1;
  const bool counts = *y >= 0 && *y < p.V;
  const unsigned long long m = __ballot(counts);
  *live = __popcll(m);
  return counts ? __popcll(m & ((1ull << lane) - 1ull)) : -1;
}
__global__ __launch_bounds__(kFewThreads) void few_kernel(CeFew p) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int token_of[kFew], target_of[kFew];
  typedef std::integral_constant<int, 0> B0;
  typedef std::integral_constant<int, 1> B1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, g = lane >> 4;
  const int tiles = (p.V + 15) / 16, stride = (int)gridDim.x * (kFewThreads / 64), steps = (p.h + 63) / 64, chunks = steps * 8;
  int tile = (int)blockIdx.x + (int)gridDim.x * wave;
  const bf16* row = nullptr;
  auto point = [&] { row = p.table + (int64_t)min(16 * tile + lr, p.V - 1) * p.h + 16 * g; };
  bf16x8 w[2][kFewAhead][2];
  auto request = [&](auto buf, int step) {
    constexpr int B = decltype(buf)::value;
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k = 64 * (step + u) + 8 * half;
        w[B][u][half] = bf16x8{};
        if (k + 16 * g < p.h) w[B][u][half] = *reinterpret_cast<const bf16x8*>(row + k);
      }
  };
  if (tile < tiles) { point(); request(B0{}, 0); }          // under way while the tokens come
  int y, live;
  const int at = few_place(p, lane, &y, &live);
  if (wave == 0 && at >= 0) { token_of[at] = lane; target_of[at] = y; }
  if (live == 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < live * chunks; i += kFewThreads) {
    const int t = i / chunks, c = i - t * chunks;
    bf16x8 v = {};
    if (8 * c < p.h) v = *reinterpret_cast<const bf16x8*>(p.X + (int64_t)token_of[t] * p.h + 8 * c);
    *reinterpret_cast<bf16x8*>(smem + t * p.pitch + 16 * c) = v;
  }
  __syncthreads();
  const unsigned char* const mine = smem + min(lr, live - 1) * p.pitch + 32 * g;       // lanes past the tokens repeat the last one
  const int target = target_of[min(lr, live - 1)];
  for (; tile < tiles; tile += stride) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](auto buf, int step) {
      constexpr int B = decltype(buf)::value;
#pragma unroll
      for (int u = 0; u < kFewAhead; ++u) {
        if (step + u >= steps) break;
#pragma unroll
        for (int half = 0; half < 2; ++half)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[B][u][half], *reinterpret_cast<const bf16x8*>(mine + 128 * (step + u) + 16 * half), acc, 0, 0, 0);
      }
    };
    const int here = tile;
    for (int step = 0; step < steps; step += 2 * kFewAhead) {
      request(B1{}, step + kFewAhead);
      multiply(B0{}, step);
      if (step + 2 * kFewAhead < steps) request(B0{}, step + 2 * kFewAhead);
      multiply(B1{}, step + kFewAhead);
    }
    if (tile + stride < tiles) {                             // the next rows come while these are worked on
      tile += stride;
      point();
      request(B0{}, 0);
      tile = here;
    }
    // acc[e] is row 16 tile + 4g + e of the table, token lr
    const int r0 = 16 * tile + 4 * g;
    const bool in = lr < live;
    float m = -INFINITY, total = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (in && r0 + e == target) p.at_target[lr] = acc[e];
      total += r0 + e < p.V ? acc[e] : 0.f;
      acc[e] = r0 + e < p.V ? acc[e] : -INFINITY;
      m = fmaxf(m, acc[e]);
    }
    m = across_rows(m, [](float a, float b) { return fmaxf(a, b); });
    const float ref = reference(m);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += exp_of(acc[e] - ref);
    sum = across_rows(sum, [](float a, float b) { return a + b; });
    if (p.totals) total = across_rows(total, [](float a, float b) { return a + b; });
    if (in && g == 0) {
      p.stats[(int64_t)lr * tiles + tile] = make_float2(m, sum);
      if (p.totals) p.totals[(int64_t)lr * tiles + tile] = total;
    }
  }
}

// The tokens' losses and their sum, by one workgroup: a wave to a token
__global__ __launch_bounds__(1024) void few_join_kernel(CeFew p) {
  __shared__ float loss_of[kFew];
  const int lane = threadIdx.x & 63, row = threadIdx.x >> 6, tiles = (p.V + 15) / 16;
  int y, live;
  const int at = few_place(p, lane, &y, &live);
  if (row < live) {
    float top = -INFINITY, sum = 0.f, total = 0.f;
    const float2* const stats = p.stats + (int64_t)row * tiles;
    for (int b0 = lane; b0 < tiles; b0 += 64 * 8) {
      float2 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = b0 + 64 * u < tiles ? stats[b0 + 64 * u] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int u = 0; u < 8; ++u) if (b0 + 64 * u < tiles) join_sums(top, sum, v[u].x, v[u].y);
      if (p.totals) {
#pragma unroll
        for (int u = 0; u < 8; ++u) if (b0 + 64 * u < tiles) total += p.totals[(int64_t)row * tiles + b0 + 64 * u];
      }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const float m = __shfl_xor(top, o, 64), s = __shfl_xor(sum, o, 64);
      join_sums(top, sum, m, s);                 // a lane of its own and its partner differ in the order, and in a last bit: lane 0's is taken
      total += __shfl_xor(total, o, 64);
    }
    if (lane == 0) loss_of[row] = token_loss(top, sum, p.at_target[row], total, p.smoothing, p.V);
  }
  __syncthreads();
  if (row == 0 && lane < p.T) p.losses[lane] = at >= 0 ? loss_of[at] : 0.f;
  if (threadIdx.x == 0) {
    double all = 0.0;
    for (int i = 0; i < live; ++i) all += (double)loss_of[i];
    const float per_token = p.denom > 0.f ? 1.f / p.denom : live ? 1.f / (float)live : 0.f;
    *p.loss = (float)(all * (double)per_token);
  }
}

// ------------------------------------------------------------------------------- joins
// out[r] = sum over the pieces in ascending order, rows of N elements; TO_ROWS: those of the span, to the tokens' rows, and the last workgroup adds
// the losses (loss not null)
template <typename T, bool TO_ROWS, int V = 4>
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ P, int splits, int64_t M, int64_t N, const float* __restrict__ scale, int height, int K, const CeSpan* __restrict__ span,
                                                   const int32_t* __restrict__ to, T* __restrict__ out, CeLoss l) {
  __shared__ double part[4];
  if (TO_ROWS && l.loss && blockIdx.x == gridDim.x - 1) add_losses<256>(l, part);
  const int64_t rows = TO_ROWS ? span->live : M, pieces = N / V, items = rows * pieces, start = TO_ROWS ? span->start : 0;
  if (TO_ROWS && height) {                       // as the product cut itself: in tiles of `height` rows
    const int tiles_m = (int)(rows + height - 1) / height;
    splits = w4_cut(tiles_m * (int)((N + 255) / 256), K).pieces;
    M = (int64_t)tiles_m * height;
    if (splits == 1) return;                     // the rows are where they belong
  }
  typedef typename Pack<float, V>::type vec;
  const float factor = scale ? *scale : 1.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / pieces, c = (i - row * pieces) * V;
    vec sum = *reinterpret_cast<const vec*>(P + row * N + c);
    for (int s = 1; s < splits; s += 8) {        // eight on their way together
      vec part[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) part[u] = s + u < splits ? *reinterpret_cast<const vec*>(P + ((s + u) * M + row) * N + c) : vec{};
#pragma unroll
      for (int u = 0; u < 8; ++u) if (s + u < splits) sum += part[u];
    }
    typename Pack<T, V>::type o;
#pragma unroll
    for (int e = 0; e < V; ++e) pack_set<T, V>(o, e, pack_get<float, V>(sum, e) * factor);
    *reinterpret_cast<typename Pack<T, V>::type*>(out + (TO_ROWS ? (int64_t)to[start + row] : row) * N + c) = o;
  }
}

constexpr int kLossThreads = 1024;
__global__ __launch_bounds__(kLossThreads) void loss_kernel(CeLoss l) {
  __shared__ double part[kLossThreads / 64];
  add_losses<kLossThreads>(l, part);
}

// -------------------------------------------------------------------------------- sizes
// Tokens of a piece: as many as keep what is left of the logits to this many elements (2 GiB in bf16), and their rows to 2 GiB.  Several pieces
// cost the fp32 sums of dtable, read and written once a piece, and their place: where one piece of all tokens needs no more room than they and a
// piece of this size do, there is one (12288 tokens that count, h 4096, V 128000, two pieces 30100 us, one 29900).
constexpr int64_t kPieceElems = (int64_t)1 << 30;
struct CeLayout {
  bool few;                                    // bf16 gradients of up to 16 tokens and more of a table than one launch takes
  int few_k;
  int64_t piece, ld, blocks, lo;               // lo: elements from a dz to what its rounding left, 0 where that is not kept
  int pieces, dw_splits, dx_splits, dx_k;      // dx: fp32 (bf16: w4_cut)
  size_t head, spans, rows, target, slot, losses, at_target, top, inverse, stats, totals, x, e, sums, bytes;
  CeLayout(int dtype, int64_t T, int64_t h, int64_t V, bool grad) {
    const bool half = dtype == MOSAIC_BF16;
    const size_t es = dtype_size(dtype);
    ld = (V + 63) / 64 * 64;
    blocks = ceil_div(V, half ? kCeBlock : kWideBlock);
    int64_t most = std::min(kPieceElems / (half ? 1 : 2) / ld, ((int64_t)1 << 30) / h) / 256 * 256;
    most = std::max<int64_t>(most, 256);
    if (half && T * ld <= kPieceElems + 2 * V * h && T * h <= (int64_t)1 << 30) most = std::max<int64_t>(most, ceil_div(T, 256) * 256);
    pieces = (int)std::max<int64_t>(1, ceil_div(T, most));
    piece = std::max<int64_t>(256, ceil_div(ceil_div(T, pieces), 256) * 256);
    size_t at = 0;
    auto take = [&](int64_t n) { const size_t here = at; at = align_up(at + (size_t)n, 256); return here; };
    const int64_t padded = piece * pieces;
    head = take(sizeof(CeHead));
    spans = take((int64_t)sizeof(CeSpan) * pieces);
    rows = take(4 * padded); target = take(4 * padded); slot = take(4 * padded); losses = take(4 * T);
    at_target = take(4 * piece); top = take(4 * piece); inverse = take(4 * piece);
    stats = take(8 * blocks * piece); totals = take(4 * blocks * piece);
    x = take(padded * h * (int64_t)es);
    lo = !half || !grad ? 0 : T <= kFewRows ? kFewRows * ld : T <= kLowTokens && V <= kLowColumns ? piece * ld : 0;
    e = take(grad || !half ? (lo == piece * ld ? 2 : 1) * piece * ld * (int64_t)es : 0);
    // the input gradient of up to 16 tokens: a workgroup to a CU, no less than two steps to a wave
    few_k = (int)std::max<int64_t>(2 * kFewStep * kFewWaves, ceil_div(ceil_div(V, std::max<int64_t>(1, 256 / ceil_div(h, 64))), kFewStep) * kFewStep);
    few = lo && T <= kFewRows && V > kLowColumns;
    // Few tiles over a long contraction leave most CUs idle: it is cut until the tiles are about one to a CU, into no less than 1024 k-values.
    const int64_t tiles = ceil_div(V, 256) * ceil_div(h, 256);
    dw_splits = half && grad ? (int)std::max<int64_t>(1, std::min(256 / tiles, std::min(piece, T) / 1024)) : 1;
    int64_t n = 0;
    if (half && grad) {
      n = std::min<int64_t>(std::min<int64_t>(kMostPieces, ceil_div(V, kLeastPiece)) * ceil_div(std::min(piece, std::max<int64_t>(T, 1)), 128) * ceil_div(h, 256), kMostPieceTiles) * 65536;       // w4_cut
      if (dw_splits > 1) n = std::max(n, dw_splits * V * h);
      if (pieces > 1) n += V * h;
      if (few) n = std::max(n, ceil_div(V, few_k) * kFewRows * h);
    }
    dx_splits = 1;
    if (!half && grad) {                         // the pieces that price least, joined at 5 TB/s; up to 1 GiB of them
      auto cut = [&](bool a_kc, int64_t M, int64_t N, int64_t K, double join) {
        int best = 1;
        double least = grouped_f32_us(a_kc, M, N, K, 1);
        for (int s = 2; s <= 64 && K / s >= 128 && s * M * N <= (int64_t)1 << 28; ++s) {
          const double us = grouped_f32_us(a_kc, M, N, K, s) + join + (double)(8 * s) * (double)(M * N) / 5e6;
          if (us < least) { least = us; best = s; }
        }
        return best;
      };
      const int64_t some = std::min(piece, std::max<int64_t>(T, 1));
      const int pieces_of = cut(true, some, h, V, 0.0);        // which pass through a join even if there is one: its rows go to the tokens'
      dx_k = (int)(ceil_div(ceil_div(V, pieces_of), 64) * 64);
      dx_splits = (int)ceil_div(V, dx_k);
      n = dx_splits * piece * h;
      if (pieces == 1) dw_splits = cut(false, V, h, some, 4.0);
      if (dw_splits > 1) n = std::max(n, dw_splits * V * h);
    }
    sums = take(4 * n);
    bytes = at;
  }
};

template <bool A_KC, bool B_KC, int EPI>
mosaic_status launch_rows(hipStream_t s, int quota, W4Args p, bool low) {
  auto go = [&](auto mi) -> mosaic_status {
    constexpr int MI = decltype(mi)::value;
    p.tiles_m = (int)ceil_div(p.M, 32 * MI);
    const int most = p.tiles_m * p.tiles_n;
    p.tile_count = EPI == W4_PIECES && most <= kMostPieceTiles ? std::min((int)std::min<int64_t>(kMostPieces, ceil_div(p.K, kLeastPiece)) * most, kMostPieceTiles) : most;
    p.row_block = row_block_for(p.K, p.M, 32 * MI);
    return launch_w4_epi<A_KC, B_KC, EPI, MI, W4_GROUPED>(s, quota, p);
  };
  return low ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 8>{});
}

}  // namespace

size_t linear_ce_scratch_bytes(int dtype, int64_t T, int64_t h, int64_t V, bool grad) { return CeLayout(dtype, T, h, V, grad).bytes; }

mosaic_status launch_linear_ce(hipStream_t s, int quota, int dtype, int64_t T, int64_t h, int64_t V, float smoothing, float denom, const int32_t* targets,
                               const void* X, const void* table, float* loss, float* losses, bool grad, void* dX, void* dtable, void* scratch) {
  const bool half = dtype == MOSAIC_BF16;
  const CeLayout L(dtype, T, h, V, grad);
  char* const base = (char*)scratch;
  if (half && !grad && T > 0 && T <= kFew && T * few_pitch(h) <= kFewLds) {
    static std::once_flag attr_once;
    static hipError_t attr_rc = hipSuccess;
    std::call_once(attr_once, [] { attr_rc = hipFuncSetAttribute(reinterpret_cast<const void*>(few_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds); });
    MOSAIC_HIP(attr_rc);
    CeFew f = {targets, (const bf16*)X, (const bf16*)table, (int)T, (int)h, (int)V, few_pitch(h), smoothing, denom, (float2*)(base + L.stats),
               smoothing > 0.f ? (float*)(base + L.totals) : nullptr, (float*)(base + L.at_target), losses ? losses : (float*)(base + L.losses), loss};
    few_kernel<<<grid_for(quota, 1, ceil_div(V, 16)), kFewThreads, (size_t)T * f.pitch, s>>>(f);
    MOSAIC_LAUNCH_CHECK();
    few_join_kernel<<<1, 1024, 0, s>>>(f);
    MOSAIC_LAUNCH_CHECK();
    return MOSAIC_OK;
  }
  CeHead* const head = (CeHead*)(base + L.head);
  CeSpan* const spans = (CeSpan*)(base + L.spans);
  int32_t *rows = (int32_t*)(base + L.rows), *target = (int32_t*)(base + L.target), *slot = (int32_t*)(base + L.slot);
  if (!losses) losses = (float*)(base + L.losses);
  const CeList list = {targets, (int)T, (int)V, (int)L.piece, L.pieces, denom, half, head, spans, rows, target, slot};
  const bool wide = half || (h % 4 == 0 && (((uintptr_t)X | (uintptr_t)dX) & 15) == 0);       // bf16 rows are whole 16-byte pieces
  auto place = [&](auto t, auto v) -> mosaic_status {
    typedef decltype(t) E;
    constexpr int N = decltype(v)::value;
    if (T <= kListMax) {
      list_place_kernel<E, N><<<grid_for(quota, 1, ceil_div(T, 16)), kListThreads, 0, s>>>(list, (const E*)X, h, (E*)(base + L.x), (E*)dX, losses);
    } else {
      list_kernel<<<1, kListThreads, 0, s>>>(list);
      MOSAIC_LAUNCH_CHECK();
      place_kernel<E, N><<<grid_for(quota, 8, ceil_div(T, 4)), 256, 0, s>>>(slot, (int)T, (const E*)X, h, (E*)(base + L.x), (E*)dX, losses);
    }
    MOSAIC_LAUNCH_CHECK();
    return MOSAIC_OK;
  };
  if (half) MOSAIC_TRY(place(bf16(), std::integral_constant<int, 8>()));
  else MOSAIC_TRY(wide ? place(float(), std::integral_constant<int, 4>()) : place(float(), std::integral_constant<int, 1>()));
  float* const sums = (float*)(base + L.sums);
  // added by a launch that has the time, or by one of its own: up to this many tokens that takes 3 us of the workgroup that does
  constexpr int kAddMax = 16384;
  const CeLoss add = {losses, (int)T, head, loss};
  bool added = false;
  for (int i = 0; i < L.pieces; ++i) {
    const int64_t r0 = i * L.piece;
    const int capacity = (int)L.piece, some = (int)std::min(L.piece, std::max<int64_t>(T - (half ? 0 : r0), 1));      // at most that many rows
    const char* Xc = base + L.x;                 // of all tokens
    const int32_t* live = &spans[i].zero;        // 0 and how many
    const CeLoss now = {losses, (int)T, head, i + 1 == L.pieces && T <= kAddMax ? loss : nullptr};
    CePiece p = {};
    p.span = spans + i; p.rows = rows; p.target = target; p.at_target = (float*)(base + L.at_target);
    p.capacity = capacity; p.V = (int)V; p.smoothing = smoothing; p.top = (float*)(base + L.top); p.inverse = (float*)(base + L.inverse); p.losses = losses;
    if (!half) {
      float* Z = (float*)(base + L.e);
      MOSAIC_TRY(launch_grouped_f32(s, quota, dtype, true, true, some, (int)V, (int)h, Xc + r0 * h * 4, h, table, h, Z, L.ld, nullptr, live, 1, capacity, 0));
      if (V <= kWideRow) {
        const int grid = grid_for(quota, 8, some);
        if (V <= 256) rows_f32_kernel<64, 1><<<grid_for(quota, 32, some), 64, 0, s>>>(p, head, Z, L.ld, grad);
        else if (V <= 1024) rows_f32_kernel<256, 1><<<grid, 256, 0, s>>>(p, head, Z, L.ld, grad);
        else if (V <= 4096) rows_f32_kernel<256, 4><<<grid, 256, 0, s>>>(p, head, Z, L.ld, grad);
        else rows_f32_kernel<256, 8><<<grid, 256, 0, s>>>(p, head, Z, L.ld, grad);
      } else {
        float2* const stats = (float2*)(base + L.stats);
        float* const totals = smoothing > 0.f ? (float*)(base + L.totals) : nullptr;
        const int grid = grid_for(quota, 8, some * L.blocks);
        wide_f32_kernel<false><<<grid, 256, 0, s>>>(p, head, Z, L.ld, stats, totals, (float*)(base + L.at_target));
        MOSAIC_LAUNCH_CHECK();
        lse_kernel<<<grid_for(quota, 2, ceil_div(some, 16)), 1024, 0, s>>>(p, stats, totals, (int)L.blocks);
        MOSAIC_LAUNCH_CHECK();
        if (grad) wide_f32_kernel<true><<<grid, 256, 0, s>>>(p, head, Z, L.ld, stats, totals, nullptr);
      }
      MOSAIC_LAUNCH_CHECK();
      if (dX) {
        MOSAIC_TRY(launch_grouped_f32(s, quota, dtype, true, false, some, (int)h, (int)V, Z, L.ld, table, h, sums, h, nullptr, live, 1, capacity, 0, L.dx_k, L.dx_splits));
        const int64_t words = some * h;
        if (wide) join_kernel<float, true, 4><<<grid_for(quota, 8, ceil_div(words, 1024)), 256, 0, s>>>(sums, L.dx_splits, some, h, nullptr, 0, 0, p.span, rows, (float*)dX, now);
        else join_kernel<float, true, 1><<<grid_for(quota, 8, ceil_div(words, 256)), 256, 0, s>>>(sums, L.dx_splits, some, h, nullptr, 0, 0, p.span, rows, (float*)dX, now);
        added = now.loss != nullptr;
        MOSAIC_LAUNCH_CHECK();
      }
      if (dtable) {
        const bool cut = L.dw_splits > 1;
        MOSAIC_TRY(launch_grouped_f32(s, quota, dtype, false, false, (int)V, (int)h, some, Z, L.ld, Xc + r0 * h * 4, h, cut ? sums : (float*)dtable, h, i ? dtable : nullptr, live, 1,
                                      capacity, 0, 0, L.dw_splits));
        if (cut) {
          if (((uintptr_t)dtable & 15) == 0 && h % 4 == 0)
            join_kernel<float, false, 4><<<grid_for(quota, 8, ceil_div(V * h, 1024)), 256, 0, s>>>(sums, L.dw_splits, V, h, nullptr, 0, 0, nullptr, nullptr, (float*)dtable, {});
          else
            join_kernel<float, false, 1><<<grid_for(quota, 8, ceil_div(V * h, 256)), 256, 0, s>>>(sums, L.dw_splits, V, h, nullptr, 0, 0, nullptr, nullptr, (float*)dtable, {});
          MOSAIC_LAUNCH_CHECK();
        }
      }
      continue;
    }
    bf16* E = grad ? (bf16*)(base + L.e) : nullptr;
    W4Args z = {};
    z.A = (const bf16*)Xc; z.B = (const bf16*)table; z.C = E;
    z.M = capacity; z.N = (int)V; z.K = (int)h; z.lda = h; z.ldb = h; z.ldc = L.ld;
    z.offsets = live; z.piece = &spans[i].start; z.groups = 1; z.bound = capacity;
    z.b_bytes = (uint32_t)(V * h * 2);
    z.tiles_n = (int)ceil_div(V, 256);
    z.rows = target; z.at_target = (float*)(base + L.at_target); z.stats = (float2*)(base + L.stats);
    z.totals = smoothing > 0.f ? (float*)(base + L.totals) : nullptr;
    const bool low = some <= 128;
    auto w4_tiles = [&](int64_t N) { return (double)(ceil_div(some, low ? 128 : 256) * ceil_div(N, 256)); };
    // 8 us for the epilogue of a round: 375 x 33 of 72, four-wave kernel 20.7 us, few_tile 5.3
    switch (few_rows(some, V, h, w4_price(w4_tiles(V), (double)h, low) + 8.0 * std::ceil(w4_tiles(V) / 256.0))) {
      case 1: MOSAIC_TRY(launch_few_logits<1>(s, quota, some, z)); break;
      case 2: MOSAIC_TRY(launch_few_logits<2>(s, quota, some, z)); break;
      case 4: MOSAIC_TRY(launch_few_logits<4>(s, quota, some, z)); break;
      default: MOSAIC_TRY((launch_rows<true, true, W4_SOFTMAX>(s, quota, z, low)));
    }
    const bool join = grad && L.blocks <= kJoinBlocks;
    if (!join) {
      lse_kernel<<<grid_for(quota, 2, ceil_div(some, 16)), 1024, 0, s>>>(p, z.stats, z.totals, (int)L.blocks);
      MOSAIC_LAUNCH_CHECK();
    }
    if (!grad) continue;
    const int64_t left = 2 * some * L.ld;
    const Sweep sweep = sweep_grid(s, quota, ceil_div(some, 16) * ceil_div(L.ld, kStrip), 2 * left);
    if (L.lo && !join) grad_kernel<false, false, true><<<sweep.grid, 256, 0, s>>>(p, z.stats, nullptr, E, L.ld, L.lo);
    else if (L.lo) grad_kernel<false, true, true><<<sweep.grid, 256, 0, s>>>(p, z.stats, z.totals, E, L.ld, L.lo);
    else if (join) grad_kernel<false, true, false><<<sweep.grid, 256, 0, s>>>(p, z.stats, z.totals, E, L.ld, 0);
    else if (sweep.in_order && left > kPastCacheBytes) grad_kernel<true, false, false><<<sweep.grid, 256, 0, s>>>(p, z.stats, nullptr, E, L.ld, 0);
    else grad_kernel<false, false, false><<<sweep.grid, 256, 0, s>>>(p, z.stats, nullptr, E, L.ld, 0);
    MOSAIC_LAUNCH_CHECK();
    W4Args w = {};
    bool few_table = false;
    if (dtable) {
      w.A = E; w.B = (const bf16*)Xc; w.C = (bf16*)dtable;
      w.M = (int)V; w.N = (int)h; w.K = capacity; w.lda = L.ld; w.ldb = h; w.ldc = h;
      w.offsets = live; w.piece = &spans[i].start; w.groups = 1; w.bound = capacity;
      w.tiles_m = (int)ceil_div(V, 256); w.tiles_n = (int)ceil_div(h, 256);
      w.tile_count = w.tiles_m * w.tiles_n;
      w.row_block = row_block_for(w.K, V, 256);
      w.sums = sums; w.first = i == 0; w.scale = &head->per_token;
      w.splits = L.dw_splits;
      const double w4_us = w4_price((double)w.tile_count * L.dw_splits, (double)some / L.dw_splits, false) + (L.dw_splits > 1 ? 5.0 + (double)(V * h) * (4 * L.dw_splits + 2) / 5e6 : 0.0);
      few_table = L.lo || (L.pieces == 1 && few_price((double)few_dtable_items(V, h), (double)some, 4, false) < w4_us);
    }
    if (dX) {
      W4Args d = {};
      d.A = E; d.B = (const bf16*)table; d.C = (bf16*)dX;
      d.M = capacity; d.N = (int)h; d.K = (int)L.ld; d.lda = L.ld; d.ldb = h; d.ldc = h;
      d.offsets = live; d.piece = &spans[i].start; d.groups = 1; d.bound = capacity;
      d.b_bytes = z.b_bytes;
      d.tiles_n = (int)ceil_div(h, 256);
      d.rows = rows;
      d.scale = &head->per_token;
      d.sums = sums + (L.pieces > 1 ? V * h : 0);
      if (L.few) {
        d.K = (int)V;
        static std::once_flag once;
        static hipError_t rc = hipSuccess;
        constexpr int kLds = few_lds<true, false, 1>();
        MOSAIC_TRY(few_allow_lds(few_dx_pieces_kernel, kLds, &once, &rc));
        const int64_t pieces = ceil_div(V, L.few_k);
        few_dx_pieces_kernel<<<grid_for(quota, 1, pieces * ceil_div(h, 64)), kFewNT, kLds, s>>>(d, L.lo, L.few_k);
        MOSAIC_LAUNCH_CHECK();
        join_kernel<bf16, true><<<grid_for(quota, 8, ceil_div((int64_t)some * (h / 4), 256)), 256, 0, s>>>(d.sums, (int)pieces, kFewRows, h, d.scale, 0, 0, p.span, rows, (bf16*)dX, now);
        MOSAIC_LAUNCH_CHECK();
        added = now.loss != nullptr;
        if (!dtable) continue;
      }
      const int blocks = L.few ? 0 : few_rows(some, h, V, L.lo ? HUGE_VAL : 8.0 + w4_cut_us((int)w4_tiles(h), d.K));
      if (blocks) {
        d.K = (int)V;                            // the rows of E are readable up to ld
        const bool both = few_table && ceil_div(some, 16 * blocks) * ceil_div(h, 64) + few_dtable_items(V, h) <= kBothItems;
        auto go = [&](auto rb) -> mosaic_status {
          constexpr int RB = decltype(rb)::value;
          if (L.lo) return both ? launch_few_dx<RB, true, true>(s, quota, some, d, now, w, L.lo) : launch_few_dx<RB, false, true>(s, quota, some, d, now, w, L.lo);
          return both ? launch_few_dx<RB, true, false>(s, quota, some, d, now, w, 0) : launch_few_dx<RB, false, false>(s, quota, some, d, now, w, 0);
        };
        MOSAIC_TRY(blocks == 1 ? go(std::integral_constant<int, 1>{}) : blocks == 2 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{}));
        added = now.loss != nullptr;
        if (both) continue;
      } else if (!L.few) {
        MOSAIC_TRY((launch_rows<true, false, W4_PIECES>(s, quota, d, low)));
        if (d.K > kLeastPiece) {                 // or there is one piece, which went where it belongs
          join_kernel<bf16, true><<<grid_for(quota, 8, ceil_div((int64_t)some * (h / 4), 256)), 256, 0, s>>>(d.sums, 0, 0, h, d.scale, low ? 128 : 256, d.K, p.span, rows, (bf16*)dX, now);
          MOSAIC_LAUNCH_CHECK();
          added = now.loss != nullptr;
        }
      }
    }
    if (!dtable) continue;
    if (L.few) {
      few_outer_kernel<<<grid_for(quota, 3, ceil_div(V, 64) * ceil_div(h, kOuterColumns)), 256, 0, s>>>(w, L.lo);
      MOSAIC_LAUNCH_CHECK();
    } else if (few_table) {
      MOSAIC_TRY(L.lo ? launch_few_dtable<true>(s, quota, w, L.lo) : launch_few_dtable<false>(s, quota, w, 0));
    } else if (L.pieces > 1) MOSAIC_TRY((launch_w4_epi<false, false, W4_ADD, 8, W4_GROUPED>(s, quota, w)));
    else if (L.dw_splits > 1) {
      w.tile_count *= w.splits;
      MOSAIC_TRY((launch_w4_epi<false, false, W4_PIECES, 8, W4_GROUPED>(s, quota, w)));
      join_kernel<bf16, false><<<grid_for(quota, 8, ceil_div(V * (h / 4), 256)), 256, 0, s>>>(sums, w.splits, V, h, w.scale, 0, 0, nullptr, nullptr, (bf16*)dtable, {});
      MOSAIC_LAUNCH_CHECK();
    } else MOSAIC_TRY((launch_w4_epi<false, false, W4_PLAIN, 8, W4_GROUPED>(s, quota, w)));
  }
  if (!added) {
    loss_kernel<<<1, kLossThreads, 0, s>>>(add);
    MOSAIC_LAUNCH_CHECK();
  }
  return MOSAIC_OK;
}
