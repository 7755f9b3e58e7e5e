// Softmax cross entropy behind a linear layer, without the logits: z_t = x_t table^T over the V rows of a table [V, h], and for every
// token whose target lies in the table
//   l_t = log sum_v exp(z_tv) - (1 - s) z_t,target - s mean_v z_tv          (s: label smoothing)
//   loss = sum l_t / D;  dz_tv = (softmax(z_t)_v - (1 - s) [v = target] - s / V) / D;  dX = dz table;  dtable = dz^T X
// with D given, or the number of such tokens.  The others take no part: their rows of X are not multiplied (they may hold anything).
//
//   1. The tokens that count are listed in order, and their rows copied side by side (rows_kernel, gather_kernel): how many there are
//      stays on the device, where the products' workgroups read it.
//   2. In pieces of tokens (kPieceElems): the product with the table, whose epilogue leaves exp(z - m) in bf16 and, for each row and 64 columns, the
//      largest logit m and the sum (w4_softmax in gemm_w4.h); or only these, when the loss alone is asked for.
//   3. lse_kernel joins a row's blocks to the logarithm of the sum and the loss; grad_kernel turns what lies there into dz, in place.
//   4. dX = dz table, into the rows of X that the tokens came from; dtable = dz^T X, summed in fp32 over the pieces.
// So the gradients take three products of 2 T h V operations, where pieces of the vocabulary would want the logits twice: their softmax needs the whole
// row.  fp32: the same on fp32 logits, whose rows one workgroup normalises (rows_f32_kernel).
//
// All sums have an order that the sizes and the targets fix.
#include "gemm_plan.h"
#include "gemm_w4.h"
#include "kernels.h"

mosaic_status launch_grouped_f32(hipStream_t s, int quota, int dtype, bool a_kc, bool b_kc, int M, int N, int K, const void* A, int64_t lda, const void* B,
                                 int64_t ldb, void* C, int64_t ldc, const void* R, const int32_t* offsets, int groups, int bound, int64_t stride);

namespace {

constexpr float kLn2 = 0.69314718055994530942f, kLog2e = 1.44269504088896340736f;

// ------------------------------------------------------------------------- the tokens that count
struct CeHead { int count; float per_token; };      // their number, and 1 / D

// In order: rows[i] = token, target[i] = its target; slot[t] = i, or -1; piece_rows[2p], [2p + 1] = 0 and how many of them piece p of `piece` tokens has.
// One workgroup: 16 waves in order, lanes in order.
constexpr int kRowsThreads = 1024;
__global__ __launch_bounds__(kRowsThreads) void rows_kernel(const int32_t* __restrict__ targets, int T, int V, float denom, int piece, int pieces,
                                                            CeHead* __restrict__ head, int32_t* __restrict__ piece_rows, int32_t* __restrict__ rows,
                                                            int32_t* __restrict__ target, int32_t* __restrict__ slot) {
  constexpr int kWaves = kRowsThreads / 64;
  __shared__ int wave_count[2][kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int run = 0;
  for (int t0 = 0, turn = 0; t0 < T; t0 += kRowsThreads, turn ^= 1) {
    const int t = t0 + threadIdx.x;
    const int y = t < T ? targets[t] : -1;
    const bool counts = y >= 0 && y < V;
    const unsigned long long m = __ballot(counts);
    if (lane == 0) wave_count[turn][wave] = __popcll(m);
    __syncthreads();                             // the other half of wave_count was read before the barrier of the turn before
    int before = run;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int n = wave_count[turn][w];
      if (w < wave) before += n;
      run += n;
    }
    const int at = before + __popcll(m & ((1ull << lane) - 1ull));
    if (counts) { rows[at] = t; target[at] = y; }
    if (t < T) slot[t] = counts ? at : -1;
  }
  for (int p = threadIdx.x; p < pieces; p += kRowsThreads) {
    piece_rows[2 * p] = 0;
    piece_rows[2 * p + 1] = (int)min((int64_t)piece, max((int64_t)run - (int64_t)p * piece, (int64_t)0));
  }
  if (threadIdx.x == 0) *head = {run, denom > 0.f ? 1.f / denom : run ? 1.f / (float)run : 0.f};
}

// A wave per token: its row of X to where it counts, or zeros to its gradient and loss.
template <typename T, int V>
__global__ __launch_bounds__(256) void gather_kernel(const T* __restrict__ X, const int32_t* __restrict__ slot, int tokens, int64_t h, T* __restrict__ Xc,
                                                     T* __restrict__ dX, float* __restrict__ losses) {
  typedef typename Pack<T, V>::type vec;
  const int lane = threadIdx.x & 63;
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < tokens; t += (int64_t)gridDim.x * 4) {
    const int at = slot[t];
    if (at >= 0) {
      for (int64_t c = lane * V; c < h; c += 64 * V) *reinterpret_cast<vec*>(Xc + at * h + c) = *reinterpret_cast<const vec*>(X + t * h + c);
    } else {
      if (dX) for (int64_t c = lane * V; c < h; c += 64 * V) *reinterpret_cast<vec*>(dX + t * h + c) = vec{};
      if (lane == 0) losses[t] = 0.f;
    }
  }
}

// -------------------------------------------------------------------------- rows of the softmax
struct CePiece {
  const int32_t* live;         // [1]: how many tokens it has
  const int32_t *rows, *target;
  const float* at_target;
  int capacity, V;
  float smoothing;
  float* lse;                  // of each row, to the base of 2
  float* losses;
};

// 64 rows to a workgroup, a lane each; sixteen waves share their blocks, whose statistics lie row by row.
__global__ __launch_bounds__(1024) void lse_kernel(CePiece p, const float2* __restrict__ stats, const float* __restrict__ totals, int blocks) {
  __shared__ float top_of[16][64], sum_of[16][64], total_of[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, live = p.live[1];
  for (int r0 = blockIdx.x * 64; r0 < live; r0 += gridDim.x * 64) {
    const int row = r0 + lane;                   // below capacity, a multiple of 64
    float top = -INFINITY, sum = 0.f, total = 0.f;
    for (int b0 = wave; b0 < blocks; b0 += 16 * 8) {
      float2 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = b0 + 16 * u < blocks ? stats[(int64_t)(b0 + 16 * u) * p.capacity + row] : make_float2(-INFINITY, 0.f);
      float high = top;
#pragma unroll
      for (int u = 0; u < 8; ++u) high = fmaxf(high, v[u].x);
      // where nothing has come yet there is nothing to scale; infinities and NaN go into the sum as they are
      if (high != top) { sum *= __builtin_amdgcn_exp2f(top - high); top = high; }
#pragma unroll
      for (int u = 0; u < 8; ++u) if (b0 + 16 * u < blocks) sum = fmaf(v[u].y, __builtin_amdgcn_exp2f(v[u].x - top), sum);
      if (totals) {
#pragma unroll
        for (int u = 0; u < 8; ++u) if (b0 + 16 * u < blocks) total += totals[(int64_t)(b0 + 16 * u) * p.capacity + row];
      }
    }
    top_of[wave][lane] = top; sum_of[wave][lane] = sum; total_of[wave][lane] = total;
    __syncthreads();
    if (wave == 0 && row < live) {
      float high = -INFINITY;
#pragma unroll
      for (int w = 0; w < 16; ++w) high = fmaxf(high, top_of[w][lane]);
      float all = 0.f, z = 0.f;
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        if (top_of[w][lane] != -INFINITY) all = fmaf(sum_of[w][lane], __builtin_amdgcn_exp2f(top_of[w][lane] - high), all);
        z += total_of[w][lane];
      }
      const float lse = high + __builtin_amdgcn_logf(all);      // to the base of 2
      p.lse[row] = lse;
      float loss = lse * kLn2 - (1.f - p.smoothing) * p.at_target[row];
      if (totals) loss -= p.smoothing * (z / (float)p.V);
      p.losses[p.rows[row]] = loss;
    }
    __syncthreads();
  }
}

// exp(z - m) -> dz, in place: a strip of 16 rows and 1024 columns at a time, 16 bytes to a lane.
constexpr int kStrip = 1024;
__global__ __launch_bounds__(256) void grad_kernel(CePiece p, const CeHead* __restrict__ head, const float2* __restrict__ stats, bf16* __restrict__ E, int64_t ld) {
  const int live = p.live[1], strips = (int)((ld + kStrip - 1) / kStrip);
  const float g = head->per_token, even = p.smoothing / (float)p.V;
  const int64_t items = (int64_t)((live + 15) / 16) * strips;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int r0 = (int)(item / strips) * 16, c0 = (int)(item % strips) * kStrip;
    Vec16<bf16> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = r0 + 2 * i + (threadIdx.x >> 7), col = c0 + 8 * (threadIdx.x & 127);
      if (row < live && col < ld) v[i].load(E + (int64_t)row * ld + col);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = r0 + 2 * i + (threadIdx.x >> 7), col = c0 + 8 * (threadIdx.x & 127);
      if (row >= live || col >= ld) continue;
      const float lse = p.lse[row];
      const float scale = __builtin_amdgcn_exp2f(stats[(int64_t)(col / kCeBlock) * p.capacity + row].x - lse);
      const int hit = p.target[row] - col;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float d = v[i].get(e) * scale - even;
        // the target's probability from its own logit: 1 - p keeps its digits where p is near 1
        if (e == hit) d = (__builtin_amdgcn_exp2f(fmaf(p.at_target[row], kLog2e, -lse)) - 1.f) + (p.smoothing - even);
        v[i].set(e, col + e < p.V ? d * g : 0.f);
      }
      v[i].store(E + (int64_t)row * ld + col);
    }
  }
}

__device__ __forceinline__ float block_reduce(float x, bool max, float* lds) {
  x = max ? wave_max(x) : wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return max ? fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3])) : (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// fp32 logits, a workgroup per row: loss and (Z written) dz in place
__global__ __launch_bounds__(256) void rows_f32_kernel(CePiece p, const CeHead* __restrict__ head, float* __restrict__ Z, int64_t ld, int grad) {
  __shared__ float lds[4];
  const int live = p.live[1];
  const float g = head->per_token, even = p.smoothing / (float)p.V;
  for (int row = blockIdx.x; row < live; row += gridDim.x) {
    float* z = Z + row * ld;
    const int target = p.target[row];
    float top = -INFINITY, total = 0.f;
    for (int c = threadIdx.x; c < p.V; c += 256) { top = fmaxf(top, z[c]); total += z[c]; }
    top = block_reduce(top, true, lds);
    total = block_reduce(total, false, lds);
    float sum = 0.f;
    for (int c = threadIdx.x; c < p.V; c += 256) sum += expf(z[c] - top);
    sum = block_reduce(sum, false, lds);
    const float lse = top + logf(sum);
    if (threadIdx.x == 0) {
      float loss = lse - (1.f - p.smoothing) * z[target];
      if (p.smoothing > 0.f) loss -= p.smoothing * (total / (float)p.V);
      p.losses[p.rows[row]] = loss;
    }
    if (!grad) continue;
    __syncthreads();                             // the target's logit has been read
    for (int c = threadIdx.x; c < p.V; c += 256) {
      const float q = expf(z[c] - lse);
      z[c] = g * (c == target ? (q - 1.f) + (p.smoothing - even) : q - even);
    }
  }
}

// ------------------------------------------------------------------------------- joins
// out[r] = sum over the pieces in ascending order (+ what is there), rows of N elements; TO_ROWS: row r to row to[r], r < live
template <typename T, bool TO_ROWS>
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ P, int splits, int64_t M, int64_t N, const int32_t* __restrict__ live,
                                                   const int32_t* __restrict__ to, T* __restrict__ out) {
  const int64_t rows = TO_ROWS ? live[1] : M, n4 = N / 4, items = rows * n4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / n4, c = (i - row * n4) * 4;
    f32x4 sum = *reinterpret_cast<const f32x4*>(P + row * N + c);
    for (int s = 1; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(P + (s * M + row) * N + c);
    typename Pack<T, 4>::type o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (T)sum[e];
    *reinterpret_cast<typename Pack<T, 4>::type*>(out + (TO_ROWS ? (int64_t)to[row] : row) * N + c) = o;
  }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void scatter_kernel(const T* __restrict__ from, const int32_t* __restrict__ live, const int32_t* __restrict__ to, int64_t h,
                                                      T* __restrict__ out) {
  typedef typename Pack<T, V>::type vec;
  const int lane = threadIdx.x & 63, rows = live[1];
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.x * 4)
    for (int64_t c = lane * V; c < h; c += 64 * V) *reinterpret_cast<vec*>(out + to[r] * h + c) = *reinterpret_cast<const vec*>(from + r * h + c);
}

// loss = sum of the tokens' / D: one workgroup, every thread its tokens in ascending order, in 64 bits
__global__ __launch_bounds__(1024) void loss_kernel(const float* __restrict__ losses, int T, const CeHead* __restrict__ head, float* __restrict__ loss) {
  __shared__ double part[16];
  double sum = 0.0;
  for (int t = threadIdx.x; t < T; t += 1024) sum += (double)losses[t];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += part[w];
    *loss = (float)(sum * (double)head->per_token);
  }
}

// -------------------------------------------------------------------------------- sizes
// Tokens of a piece: as many as keep what is left of the logits to this many elements (1 GiB in bf16), and their rows to 2 GiB.  Several pieces
// cost the fp32 sums of dtable, read and written once a piece.
constexpr int64_t kPieceElems = (int64_t)1 << 29;
struct CeLayout {
  int64_t piece, ld, blocks;
  int pieces, dx_splits, dx_k, dw_splits, dw_k;
  size_t head, piece_rows, rows, target, slot, losses, at_target, lse, stats, totals, x, e, sums, bytes;
  CeLayout(int dtype, int64_t T, int64_t h, int64_t V, bool grad) {
    const bool half = dtype == MOSAIC_BF16;
    const size_t es = dtype_size(dtype);
    ld = (V + 63) / 64 * 64;
    blocks = ceil_div(V, kCeBlock);
    int64_t most = std::min(kPieceElems / (half ? 1 : 2) / ld, ((int64_t)1 << 29) / h) / 256 * 256;
    most = std::max<int64_t>(most, 256);
    pieces = (int)std::max<int64_t>(1, ceil_div(T, most));
    piece = std::max<int64_t>(256, ceil_div(ceil_div(T, pieces), 256) * 256);
    size_t at = 0;
    auto take = [&](int64_t n) { const size_t here = at; at = align_up(at + (size_t)n, 256); return here; };
    const int64_t padded = piece * pieces;
    head = take(sizeof(CeHead));
    piece_rows = take(8 * (int64_t)pieces);
    rows = take(4 * padded); target = take(4 * padded); slot = take(4 * padded); losses = take(4 * T);
    at_target = take(4 * piece); lse = take(4 * piece);
    stats = take(half ? 8 * blocks * piece : 0); totals = take(half ? 4 * blocks * piece : 0);
    x = take(padded * h * (int64_t)es);
    e = take(grad || !half ? piece * ld * (int64_t)es : 0);
    // Few tiles over a long contraction leave most CUs idle: it is cut until the tiles are about one to a CU, into no less than 1024 k-values.
    auto cut = [&](int64_t M, int64_t K, int* k) {
      const int64_t tiles = ceil_div(M, 256) * ceil_div(h, 256);
      int64_t n = std::max<int64_t>(1, std::min(256 / tiles, K / 1024));
      *k = (int)(ceil_div(ceil_div(K, n), 64) * 64);
      return (int)std::max<int64_t>(1, ceil_div(K, *k));
    };
    dx_splits = half && grad ? cut(std::min(piece, std::max<int64_t>(T, 1)), ld, &dx_k) : 1;
    dw_splits = half && grad ? cut(V, piece, &dw_k) : 1;
    int64_t n = 0;
    if (half && grad) {
      if (dx_splits > 1) n = std::max(n, dx_splits * piece * h);
      if (dw_splits > 1) n = std::max(n, dw_splits * V * h);
      if (pieces > 1) n = std::max(n, V * h + (dx_splits > 1 ? dx_splits * piece * h : 0));
    }
    if (!half && grad) n = piece * h;            // dX of the piece
    sums = take(4 * n);
    bytes = at;
  }
};

template <bool A_KC, bool B_KC, int EPI>
mosaic_status launch_rows(hipStream_t s, int quota, W4Args p, bool low) {
  auto go = [&](auto mi) -> mosaic_status {
    constexpr int MI = decltype(mi)::value;
    p.tiles_m = (int)ceil_div(p.M, 32 * MI);
    p.tile_count = p.tiles_m * p.tiles_n * (EPI == W4_PIECES ? p.splits : 1);
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
  CeHead* head = (CeHead*)(base + L.head);
  int32_t *piece_rows = (int32_t*)(base + L.piece_rows), *rows = (int32_t*)(base + L.rows), *target = (int32_t*)(base + L.target), *slot = (int32_t*)(base + L.slot);
  if (!losses) losses = (float*)(base + L.losses);
  rows_kernel<<<1, kRowsThreads, 0, s>>>(targets, (int)T, (int)V, denom, (int)L.piece, L.pieces, head, piece_rows, rows, target, slot);
  MOSAIC_LAUNCH_CHECK();
  const bool wide = h % (half ? 8 : 4) == 0 && (((uintptr_t)X | (uintptr_t)dX) & 15) == 0;
  auto gather = [&](auto t) {
    typedef decltype(t) E;
    const int grid = grid_for(quota, 8, ceil_div(T, 4));
    if (wide) gather_kernel<E, Vec16<E>::N><<<grid, 256, 0, s>>>((const E*)X, slot, (int)T, h, (E*)(base + L.x), (E*)dX, losses);
    else gather_kernel<E, 1><<<grid, 256, 0, s>>>((const E*)X, slot, (int)T, h, (E*)(base + L.x), (E*)dX, losses);
  };
  if (T > 0) {
    if (half) gather(bf16()); else gather(float());
    MOSAIC_LAUNCH_CHECK();
  }
  float* const sums = (float*)(base + L.sums);
  for (int i = 0; i < L.pieces; ++i) {
    const int64_t r0 = i * L.piece;
    const int capacity = (int)L.piece, some = (int)std::min(L.piece, std::max<int64_t>(T - r0, 1));      // at most that many rows
    const char* Xc = base + L.x + r0 * h * dtype_size(dtype);
    CePiece p = {};
    p.live = piece_rows + 2 * i; p.rows = rows + r0; p.target = target + r0; p.at_target = (float*)(base + L.at_target);
    p.capacity = capacity; p.V = (int)V; p.smoothing = smoothing; p.lse = (float*)(base + L.lse); p.losses = losses;
    if (!half) {
      float* Z = (float*)(base + L.e);
      MOSAIC_TRY(launch_grouped_f32(s, quota, dtype, true, true, some, (int)V, (int)h, Xc, h, table, h, Z, L.ld, nullptr, p.live, 1, capacity, 0));
      rows_f32_kernel<<<grid_for(quota, 8, some), 256, 0, s>>>(p, head, Z, L.ld, grad);
      MOSAIC_LAUNCH_CHECK();
      if (dX) {
        MOSAIC_TRY(launch_grouped_f32(s, quota, dtype, true, false, some, (int)h, (int)V, Z, L.ld, table, h, sums, h, nullptr, p.live, 1, capacity, 0));
        const int grid = grid_for(quota, 8, ceil_div(some, 4));
        if (wide) scatter_kernel<float, 4><<<grid, 256, 0, s>>>(sums, p.live, p.rows, h, (float*)dX);
        else scatter_kernel<float, 1><<<grid, 256, 0, s>>>(sums, p.live, p.rows, h, (float*)dX);
        MOSAIC_LAUNCH_CHECK();
      }
      if (dtable) MOSAIC_TRY(launch_grouped_f32(s, quota, dtype, false, false, (int)V, (int)h, some, Z, L.ld, Xc, h, dtable, h, i ? dtable : nullptr, p.live, 1, capacity, 0));
      continue;
    }
    bf16* E = grad ? (bf16*)(base + L.e) : nullptr;
    W4Args z = {};
    z.A = (const bf16*)Xc; z.B = (const bf16*)table; z.C = E;
    z.M = capacity; z.N = (int)V; z.K = (int)h; z.lda = h; z.ldb = h; z.ldc = L.ld;
    z.offsets = p.live; z.groups = 1; z.bound = capacity;
    z.b_bytes = (uint32_t)(V * h * 2);
    z.tiles_n = (int)ceil_div(V, 256);
    z.rows = p.target; z.at_target = (float*)(base + L.at_target); z.stats = (float2*)(base + L.stats);
    z.totals = smoothing > 0.f ? (float*)(base + L.totals) : nullptr;
    MOSAIC_TRY((launch_rows<true, true, W4_SOFTMAX>(s, quota, z, some <= 128)));
    lse_kernel<<<grid_for(quota, 2, ceil_div(some, 64)), 1024, 0, s>>>(p, z.stats, z.totals, (int)L.blocks);
    MOSAIC_LAUNCH_CHECK();
    if (!grad) continue;
    grad_kernel<<<grid_for(quota, 8, ceil_div(some, 16) * ceil_div(L.ld, kStrip)), 256, 0, s>>>(p, head, z.stats, E, L.ld);
    MOSAIC_LAUNCH_CHECK();
    float* const dx_sums = sums + (L.pieces > 1 ? V * h : 0);
    if (dX) {
      W4Args d = {};
      d.A = E; d.B = (const bf16*)table; d.C = (bf16*)dX;
      d.M = capacity; d.N = (int)h; d.K = (int)L.ld; d.lda = L.ld; d.ldb = h; d.ldc = h;
      d.offsets = p.live; d.groups = 1; d.bound = capacity;
      d.b_bytes = z.b_bytes;
      d.tiles_n = (int)ceil_div(h, 256);
      d.rows = p.rows;
      d.splits = L.dx_splits; d.split_k = L.dx_k; d.sums = dx_sums;
      if (L.dx_splits > 1) {
        MOSAIC_TRY((launch_rows<true, false, W4_PIECES>(s, quota, d, some <= 128)));
        join_kernel<bf16, true><<<grid_for(quota, 8, ceil_div((int64_t)some * (h / 4), 256)), 256, 0, s>>>(dx_sums, L.dx_splits, capacity, h, p.live, p.rows, (bf16*)dX);
        MOSAIC_LAUNCH_CHECK();
      } else {
        MOSAIC_TRY((launch_rows<true, false, W4_SCATTER>(s, quota, d, some <= 128)));
      }
    }
    if (dtable) {
      W4Args w = {};
      w.A = E; w.B = (const bf16*)Xc; w.C = (bf16*)dtable;
      w.M = (int)V; w.N = (int)h; w.K = capacity; w.lda = L.ld; w.ldb = h; w.ldc = h;
      w.offsets = p.live; w.groups = 1; w.bound = capacity;
      w.tiles_m = (int)ceil_div(V, 256); w.tiles_n = (int)ceil_div(h, 256);
      w.tile_count = w.tiles_m * w.tiles_n;
      w.row_block = row_block_for(w.K, V, 256);
      w.sums = sums; w.first = i == 0; w.last = i == L.pieces - 1;
      w.splits = L.dw_splits; w.split_k = L.dw_k;
      if (L.pieces > 1) MOSAIC_TRY((launch_w4_epi<false, false, W4_ADD, 8, W4_GROUPED>(s, quota, w)));
      else if (L.dw_splits > 1) {
        w.tile_count *= w.splits;
        MOSAIC_TRY((launch_w4_epi<false, false, W4_PIECES, 8, W4_GROUPED>(s, quota, w)));
        join_kernel<bf16, false><<<grid_for(quota, 8, ceil_div(V * (h / 4), 256)), 256, 0, s>>>(sums, w.splits, V, h, nullptr, nullptr, (bf16*)dtable);
        MOSAIC_LAUNCH_CHECK();
      } else MOSAIC_TRY((launch_w4_epi<false, false, W4_PLAIN, 8, W4_GROUPED>(s, quota, w)));
    }
  }
  loss_kernel<<<1, 1024, 0, s>>>(losses, (int)T, head, loss);
  MOSAIC_LAUNCH_CHECK();
  return MOSAIC_OK;
}
