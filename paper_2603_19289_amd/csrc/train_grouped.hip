// Products of rows grouped by expert with the experts' matrices:
//   y_r = W_e x_r, or W_e^T x_r,  for the rows r of expert e        (grouped_kernel: tiles of rows of one expert each)
//   dW_e = sum_{r of e} dy_r x_r^T                                  (weight_grad_kernel: tiles of one expert's matrix each)
// Which expert a workgroup works for it finds in `ends` itself, a wavefront's scan over at most 256 words, so that nothing has to be known on
// the host and a captured call follows other groups.
#include "f32_tiles.h"

namespace moe_spec {
namespace {

// ---- groups -------------------------------------------------------------------------------------------------
// Group e is the rows [max of ends before e, max of ends up to e), both within [0, rows]: whatever ends holds, groups do not overlap and
// lie inside the matrix.
__device__ __forceinline__ int wave_max(int v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = max(v, __shfl_xor(v, d));
  return v;
}

struct RowTile {
  int expert;                  // n_experts: rows behind the last group; -1: none
  int row0, rows;              // of all rows
  int tile_n;
};

// Tile number `at` of rows x cols of them, in strips of `high` rows, down each column of a strip: tiles that are worked on at the same time then lie in
// a block, and share rows and columns through the L2.
struct TilePlace { int row, col; };
__device__ __forceinline__ TilePlace tile_place(int at, int rows, int cols, int high) {
  const int strip = at / (high * cols), in = at - strip * high * cols, rest = min(high, rows - strip * high);
  return {strip * high + in % rest, in / rest};
}

// Which tile of at most BM rows of one expert, and of which columns, this workgroup takes.  Consecutive workgroups go to the eight
// dies in turn; each die gets a run of tiles: large ones in strips of 6 rows of the 32 that a die's compute units work on (32 experts of 5760 x 2880,
// 1024 rows each, transposed: 1147 -> 1114 us then, 1105 now), others columns first.
template <int BM>
__device__ __forceinline__ RowTile row_tile(const int32_t *ends, int n_experts, int rows, int tiles_n) {
  const int lane = threadIdx.x & 63;
  int end[4], count[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * lane + i;
    end[i] = e < n_experts ? min(max(ends[e], 0), rows) : 0;
    if (i) end[i] = max(end[i], end[i - 1]);
  }
  int before = end[3];                                   // inclusive running maximum over the lanes, then exclusive
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int v = __shfl_up(before, d);
    if (lane >= d) before = max(before, v);
  }
  const int last = __builtin_amdgcn_readlane(before, 63);
  before = __shfl_up(before, 1);
  if (lane == 0) before = 0;
  int sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    end[i] = max(end[i], before);
    const int n = end[i] - (i ? end[i - 1] : before);
    count[i] = n / BM + (n % BM != 0);
    sum += count[i];
  }
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  const int tiles = __builtin_amdgcn_readlane(upto, 63), all = tiles + (rows - last) / BM + ((rows - last) % BM != 0);
  const int64_t total = int64_t(all) * tiles_n, share = (total + 7) / 8, slot = blockIdx.x / 8, logical = blockIdx.x % 8 * share + slot;
  RowTile t{-1, 0, 0, 0};
  if (slot >= share || logical >= total) return t;
  const int at = int(logical / tiles_n);
  if (at >= tiles) {
    t.tile_n = int(logical % tiles_n);
    t.expert = n_experts;
    t.row0 = last + (at - tiles) * BM;
    t.rows = min(BM, rows - t.row0);
    return t;
  }
  const int who = __builtin_amdgcn_readfirstlane(__popcll(__ballot(upto <= at)));        // the lane whose experts have it
  int from = upto - sum, which = 0, first = 0, begin = 0, stop = 0, many = 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (at >= from && at < from + count[i]) {
      which = i;
      first = from;
      begin = i ? end[i - 1] : before;
      stop = end[i];
      many = count[i];
    }
    from += count[i];
  }
  t.expert = 4 * who + __builtin_amdgcn_readlane(which, who);
  begin = __builtin_amdgcn_readlane(begin, who);
  stop = __builtin_amdgcn_readlane(stop, who);
  first = __builtin_amdgcn_readlane(first, who);
  const TilePlace p = BM == 256 ? tile_place(int(logical - int64_t(first) * tiles_n), __builtin_amdgcn_readlane(many, who), tiles_n, 6)
                                : TilePlace{at - first, int(logical % tiles_n)};
  t.tile_n = p.col;
  t.row0 = begin + p.row * BM;
  t.rows = min(BM, stop - t.row0);
  return t;
}

// ---- y = x W^T, y = x W ----------------------------------------------------------------------------------------
struct GroupedArgs {
  const void *x, *w;
  void *y;
  const int32_t *ends;
  int64_t x_stride, w_stride, w_expert, y_stride, k;
  int rows, n_experts, n, tiles_n, out_bf16;
};

// A wavefront's part of a tile into a row-major matrix, of which the tile's first `rows` rows and `cols` columns exist, from (row, col) on; bfloat16
// by way of its part of LDS.  PAST: past the caches.
template <bool PAST, int FM, int FN>
__device__ __forceinline__ void store_tile(void *out, int64_t at, int64_t stride, bool bf16, const f32x4_t (&acc)[FM][FN], char *lds, int row, int col,
                                           int rows, int cols) {
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  if (bf16) {
    using R = ResultTile<16 * FM, 16 * FN>;
    char *mine = lds + (threadIdx.x >> 6) * R::kBytes;
    __syncthreads();                             // the operands have been read by all
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int h = 0; h < FN; ++h) R::put(mine, f, h, uint2{pack_bf16(acc[f][h][0], acc[f][h][1]), pack_bf16(acc[f][h][2], acc[f][h][3])}, lane);
#pragma unroll
    for (int q = 0; q < R::kEach; ++q) {
      const int r = (q * 64 + lane) / R::kAcross, c = (q * 64 + lane) % R::kAcross;
      uint16_t *to = static_cast<uint16_t *>(out) + at + int64_t(row + r) * stride + col + 8 * c;
      const int n = cols - col - 8 * c;
      if (row + r >= rows) continue;
      if (PAST && n >= 8) store_past(to, R::chunk(mine, r, c));
      else store8(to, R::chunk(mine, r, c), n);
    }
    return;
  }
#pragma unroll
  for (int f = 0; f < FM; ++f) {
    const int r = row + 16 * f + i;
    if (r >= rows) continue;
    float *q = static_cast<float *>(out) + at + int64_t(r) * stride;
#pragma unroll
    for (int h = 0; h < FN; ++h) {
      const int c = col + 16 * h + 4 * g;
      if (PAST && cols - c >= 4) store_past(q + c, __builtin_bit_cast(uint4, acc[f][h]));
      else store4(q + c, acc[f][h], cols - c);
    }
  }
}

template <typename P, int BM, int BN, int WM, int WN, typename Elem>
__device__ __forceinline__ void grouped_tile(const GroupedArgs &a, const RowTile &t, char *lds, bool w_imajor) {
  const int col0 = t.tile_n * BN, cols = min(BN, a.n - col0), wave = threadIdx.x >> 6;
  P p;
  const bool behind = t.expert == a.n_experts;
  const Elem *w = static_cast<const Elem *>(a.w) + (behind ? 0 : t.expert * a.w_expert) + (w_imajor ? int64_t(col0) : col0 * a.w_stride);
  p.run(lds, static_cast<const Elem *>(a.x) + t.row0 * a.x_stride, a.x_stride, t.rows, w, a.w_stride, cols, behind ? 0 : a.k);
  store_tile<false>(a.y, t.row0 * a.y_stride + col0, a.y_stride, a.out_bf16, p.acc, lds, wave / WN * (BM / WM), wave % WN * (BN / WN), t.rows, cols);
}

// Tiles of 256 rows whose expert has no more than 128 left are half the work as one of 128.
template <typename Type, int BM, int BN, int WM, int WN, int STEPS, bool W_IMAJOR, bool WHOLE16>
__global__ __launch_bounds__(WM *WN * 64, Type::kWaves) void grouped_kernel(const GroupedArgs a) {
  using P = TileProduct<Type, BM, BN, WM, WN, false, W_IMAJOR, WHOLE16, STEPS>;
  __shared__ __attribute__((aligned(16))) char lds[P::kLds];
  const RowTile t = row_tile<BM>(a.ends, a.n_experts, a.rows, a.tiles_n);
  if (t.expert < 0) return;
  if constexpr (BM == 256) {
    if (t.rows <= BM / 2) {
      grouped_tile<TileProduct<Type, BM / 2, BN, WM, WN, false, W_IMAJOR, WHOLE16>, BM / 2, BN, WM, WN, typename Type::Elem>(a, t, lds, W_IMAJOR);
      return;
    }
  }
  grouped_tile<P, BM, BN, WM, WN, typename Type::Elem>(a, t, lds, W_IMAJOR);
}

// A few rows, as one decoded token's choices: sixteen weight rows a workgroup, whose four wavefronts take every fourth run of columns (32 of
// bfloat16, 16 of float) and ask for all they need of 2048 (1024) at once, straight into registers; the sums meet in LDS.  Up to 16 rows
// of an expert share the weights.  Any stride and alignment.  8 rows of 8 of 128 matrices 1536 x 2048: 10.9 us, 4.6 TB/s; tiles of 64 x 128: 14.
constexpr int kFewBlock = 256, kFewWaves = kFewBlock / 64, kFewDeep = 16;

template <typename Elem>
__global__ __launch_bounds__(kFewBlock) void grouped_few_kernel(const GroupedArgs a) {
  constexpr int V = 16 / sizeof(Elem);
  __shared__ f32x4_t part[kFewWaves][64];
  const RowTile t = row_tile<16>(a.ends, a.n_experts, a.rows, a.tiles_n);
  if (t.expert < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int col0 = t.tile_n * 16, K = t.expert == a.n_experts ? 0 : int(a.k);
  const Elem *w = static_cast<const Elem *>(a.w) + (t.expert == a.n_experts ? 0 : t.expert * a.w_expert) + min(col0 + i, a.n - 1) * a.w_stride;
  const Elem *x = static_cast<const Elem *>(a.x) + (t.row0 + int64_t(min(i, t.rows - 1))) * a.x_stride;
  // V values of a row from column k on, zeros behind its end
  const auto ask = [=](const Elem *row, int n) {
    uint4 v = {0, 0, 0, 0};
    if (n >= V) {
      v = load_raw<uint4>(row);
    } else if (n > 0) {
      Elem e[V] = {};
#pragma unroll
      for (int j = 0; j < V - 1; ++j) if (j < n) e[j] = row[j];
      __builtin_memcpy(&v, e, 16);
    }
    return v;
  };
  f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};        // of each round's, so that a long sum's roundings stay small, as the tiles' do
  for (int first = (wave * 4 + g) * V; first - g * V < K; first += kFewWaves * kFewDeep * 4 * V) {
    f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    uint4 vw[kFewDeep], vx[kFewDeep];
#pragma unroll
    for (int d = 0; d < kFewDeep; ++d) {
      const int k = first + d * kFewWaves * 4 * V;
      vw[d] = ask(w + k, K - k);
      vx[d] = ask(x + k, i < t.rows ? K - k : 0);
    }
#pragma unroll
    for (int d = 0; d < kFewDeep; ++d) {
      if constexpr (V == 8) {
        acc = Bf16::mfma(__builtin_bit_cast(s16x8_t, vw[d]), __builtin_bit_cast(s16x8_t, vx[d]), acc);
      } else {                                   // which four columns an instruction takes together does not matter
        const f32x4_t fw = __builtin_bit_cast(f32x4_t, vw[d]), fx = __builtin_bit_cast(f32x4_t, vx[d]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[j], fx[j], acc, 0, 0, 0);
      }
    }
    sum += acc;
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int v = 1; v < kFewWaves; ++v) sum += part[v][lane];
  if (i >= t.rows) return;
  const int64_t at = (t.row0 + int64_t(i)) * a.y_stride + col0 + 4 * g;
  const int n = a.n - col0 - 4 * g;
  if (a.out_bf16) store8(static_cast<uint16_t *>(a.y) + at, uint4{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]), 0, 0}, n < 4 ? n : 4);
  else store4(static_cast<float *>(a.y) + at, sum, n);
}

template <int BM, int BN, int WM, int WN, bool W_IMAJOR>
__global__ __launch_bounds__(WM *WN * 64) void grouped_f32_kernel(const GroupedArgs a) {
  using P = TileProductF32<BM, BN, WM, WN, false, W_IMAJOR>;
  __shared__ __attribute__((aligned(16))) char lds[P::kLds];
  const RowTile t = row_tile<BM>(a.ends, a.n_experts, a.rows, a.tiles_n);
  if (t.expert >= 0) grouped_tile<P, BM, BN, WM, WN, float>(a, t, lds, W_IMAJOR);
}

// The same for transposed float weights, whose rows lie along the result: a lane reads four columns of one of four rows of a step, a wavefront 64 columns of
// the result, and each of four instructions takes one column of every lane.  Eight wavefronts take every eighth four rows, sixteen of them at
// once.  One row each for 8 of 128 matrices 1536 x 2048: 19 us, with tiles 38; 32 rows 69 and 116.  (The same with bfloat16 widened
// on the way was slower than its tiles: 23 and 14 for 8 of them.)
constexpr int kFewTBlock = 512, kFewTWaves = kFewTBlock / 64, kFewTCols = 64;

__global__ __launch_bounds__(kFewTBlock) void grouped_few_transposed_kernel(const GroupedArgs a) {
  __shared__ f32x4_t part[kFewTWaves][4][64];
  const RowTile t = row_tile<16>(a.ends, a.n_experts, a.rows, a.tiles_n);
  if (t.expert < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int col0 = t.tile_n * kFewTCols, K = t.expert == a.n_experts ? 0 : int(a.k), mine = col0 + 4 * i, n = a.n - mine;
  const float *w = static_cast<const float *>(a.w) + (t.expert == a.n_experts ? 0 : t.expert * a.w_expert) + mine;
  const float *x = static_cast<const float *>(a.x) + (t.row0 + int64_t(min(i, t.rows - 1))) * a.x_stride;
  f32x4_t sums[4];                               // of each round's, as above
#pragma unroll
  for (int j = 0; j < 4; ++j) sums[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  // rows of weights behind the last are the first one's, and count for nothing
  const auto walk = [&](auto whole) {
    for (int first = 4 * wave; first < K; first += kFewTWaves * kFewDeep * 4) {
      f32x4_t acc[4];
      Run<float, 4> vw[kFewDeep];
      float vx[kFewDeep];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int d = 0; d < kFewDeep; ++d) {
        const int at = first + d * kFewTWaves * 4 + g, k = at < K ? at : 0;
        vw[d].load(w + int64_t(k) * a.w_stride, decltype(whole)::value ? 4 : n);
        vx[d] = x[k];
      }
#pragma unroll
      for (int d = 0; d < kFewDeep; ++d) {
        const bool in = first + d * kFewTWaves * 4 + g < K;
        float f[4];
        vw[d].get(f);
        const float v = in && i < t.rows ? vx[d] : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? f[j] : 0.0f, v, acc[j], 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sums[j] += acc[j];
    }
  };
  if (a.n - col0 >= kFewTCols) walk(std::true_type());
  else walk(std::false_type());
#pragma unroll
  for (int j = 0; j < 4; ++j) part[wave][j][lane] = sums[j];
  __syncthreads();
  // lane (token i, g), value q of column set j: column col0 + 4 (4 g + q) + j
  for (int q = threadIdx.x; q < t.rows * kFewTCols; q += kFewTBlock) {
    const int row = q / kFewTCols, c = q % kFewTCols, from = c / 4;
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < kFewTWaves; ++v) sum += part[v][c % 4][from / 4 * 16 + row][from % 4];
    if (col0 + c >= a.n) continue;
    const int64_t to = (t.row0 + int64_t(row)) * a.y_stride + col0 + c;
    if (a.out_bf16) static_cast<uint16_t *>(a.y)[to] = to_bf16(sum);
    else static_cast<float *>(a.y)[to] = sum;
  }
}

// ---- dW = dy^T x -------------------------------------------------------------------------------------------------
struct WeightGradArgs {
  const void *dy, *x;
  void *dw;
  const int32_t *ends;
  int64_t dy_stride, x_stride, dw_stride, dw_expert;
  int rows, n_experts, n, k, tiles_n, tiles_k, out_bf16;
  int parts;                   // of each expert's rows; more than one: sums of each go to `partial`
  float *partial;              // [parts, n_experts, n, k]
  int past;                    // gradients that no cache would keep for who reads them go past the caches: 805 MB in 555 instead of 576 us
};

constexpr int kPartRows = 64;            // a part of an expert's rows is a multiple of these

// Each die gets an eighth of every expert's tiles (another one for each expert, where eighths differ), since experts differ in their rows: where dies
// had experts of their own, the last one to finish kept the others waiting (65536 rows over 128 experts: 634 -> 570 us).
template <typename P, int BM, int BN, int WM, int WN, typename Elem>
__device__ __forceinline__ void weight_grad_tile(const WeightGradArgs &a, char *lds) {
  const int per = a.tiles_n * a.tiles_k;
  const unsigned most = (per + 7) / 8, slot = blockIdx.x / 8, group = slot / most, die = (blockIdx.x + group) % 8;
  const int tile = int(int64_t(die) * per / 8 + slot % most), expert = group / a.parts, part = group % a.parts;
  if (tile >= (int64_t(die) + 1) * per / 8) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;
  for (int e = lane; e < expert; e += 64) before = max(before, a.ends[e]);
  int begin = __builtin_amdgcn_readfirstlane(min(wave_max(before), a.rows));
  int end = __builtin_amdgcn_readfirstlane(min(max(a.ends[expert], begin), a.rows));
  if (a.parts > 1) {
    const int64_t length = ((int64_t(end - begin) + kPartRows - 1) / kPartRows + a.parts - 1) / a.parts * kPartRows;
    const int64_t from = begin + part * length, to = from + length;
    begin = int(from < end ? from : end);
    end = int(to < end ? to : end);
  }
  // A die's run of an expert's tiles as a block, about as high as wide.  Heights 1, 2, 3 and 6: 65536 rows, 128 of 1536 x 2048 (6 tiles a die) 545, 542,
  // 550 and 560 us; 16384 rows, 8 of 2048 x 4096 (16) 271, 262, 263 and 263; 32768 rows, 32 of 5760 x 2880 (35) 1210, 1200, 1188 and 1186.
  const TilePlace place = tile_place(tile, a.tiles_n, a.tiles_k, most < 4 ? 1 : most < 9 ? 2 : most < 20 ? 3 : 6);
  const int row0 = place.row * BM, col0 = place.col * BN, rows = min(BM, a.n - row0), cols = min(BN, a.k - col0);
  P p;
  p.run(lds, static_cast<const Elem *>(a.dy) + begin * a.dy_stride + row0, a.dy_stride, rows,
        static_cast<const Elem *>(a.x) + begin * a.x_stride + col0, a.x_stride, cols, end - begin);
  const int row = wave / WN * (BM / WM), col = wave % WN * (BN / WN);
  if (a.parts > 1) {
    store_tile<false>(a.partial, ((int64_t(part) * a.n_experts + expert) * a.n + row0) * a.k + col0, a.k, false, p.acc, lds, row, col, rows, cols);
  } else if (a.past) {
    store_tile<true>(a.dw, expert * a.dw_expert + row0 * a.dw_stride + col0, a.dw_stride, a.out_bf16, p.acc, lds, row, col, rows, cols);
  } else {
    store_tile<false>(a.dw, expert * a.dw_expert + row0 * a.dw_stride + col0, a.dw_stride, a.out_bf16, p.acc, lds, row, col, rows, cols);
  }
}

// The parts' sums, in their order.
__global__ __launch_bounds__(256) void weight_grad_join_kernel(const WeightGradArgs a) {
  const int64_t across = (a.k + 3) / 4, at = int64_t(blockIdx.x) * 256 + threadIdx.x, row = at / across, matrix = int64_t(a.n_experts) * a.n * a.k;
  if (row >= int64_t(a.n_experts) * a.n) return;
  const int c = int(at % across) * 4, n = min(4, a.k - c);
  f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = 0; p < a.parts; ++p) {
    const float *from = a.partial + p * matrix + row * a.k + c;
    if (n == 4) {
      sum += load_raw<f32x4_t>(from);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j) if (j < n) sum[j] += from[j];
    }
  }
  const int64_t to = row / a.n * a.dw_expert + row % a.n * a.dw_stride + c;
  if (a.out_bf16) store8(static_cast<uint16_t *>(a.dw) + to, uint4{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]), 0, 0}, n);
  else store4(static_cast<float *>(a.dw) + to, sum, n);
}

template <typename Type, int BM, int BN, int WM, int WN, int STEPS, bool WHOLE16, int KS = Type::kStep>
__global__ __launch_bounds__(WM *WN * 64, Type::kWaves) void weight_grad_kernel(const WeightGradArgs a) {
  using P = TileProduct<Type, BM, BN, WM, WN, true, true, WHOLE16, STEPS, KS>;
  __shared__ __attribute__((aligned(16))) char lds[P::kLds];
  weight_grad_tile<P, BM, BN, WM, WN, typename Type::Elem>(a, lds);
}

template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64) void weight_grad_f32_kernel(const WeightGradArgs a) {
  using P = TileProductF32<BM, BN, WM, WN, true, true>;
  __shared__ __attribute__((aligned(16))) char lds[P::kLds];
  weight_grad_tile<P, BM, BN, WM, WN, float>(a, lds);
}

// ---- host ----------------------------------------------------------------------------------------------------------
constexpr int kComputeUnits = 256;
constexpr int64_t kCacheBytes = int64_t(256) << 20;     // memory-side
constexpr int64_t kMostExpertStride = int64_t(1) << 40;
inline int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }
// Whether rows of `width` values can travel straight to LDS.
inline bool whole16(const void *p, int64_t stride, int width, int elem) {
  const int of = 16 / elem;
  return !misaligned(p, 16) && stride % of == 0 && width % of == 0 && stride >= width && stride <= kMostTileStride;
}

// Workgroups of a launch of `threads` each, or 0 where a launch cannot have so many.
inline unsigned grid_of(int64_t tiles, int threads) {
  const int64_t grid = (tiles + 7) / 8 * 8;
  return grid * threads < (int64_t(1) << 32) ? unsigned(grid) : 0;
}

// Most tiles of BM rows that any groups of these rows come to: one begun per group and the rows behind them.
inline int64_t row_tiles(int64_t rows, int n_experts, int tile) {
  const int64_t most = rows / tile + n_experts + 1;
  return most < rows ? most : rows;
}

const char *sizes_fault(int64_t rows, int n_experts, int n, int k) {
  if (rows < 0 || rows > MOE_SPEC_TRAIN_MAX_ROWS) return "rows must be between 0 and 2^31 - 1";
  if (n_experts < 1 || n_experts > MOE_SPEC_MAX_EXPERTS) return "n_experts must be between 1 and 256";
  if (n < 1 || n > MOE_SPEC_TRAIN_MAX_FEATURES || k < 1 || k > MOE_SPEC_TRAIN_MAX_FEATURES) return "n and k must be between 1 and 65536";
  return nullptr;
}

// A kernel and the tile that it takes.
template <typename Args>
struct Choice {
  void (*kernel)(Args);
  int bm, bn, threads;
};
template <typename Type, int BM, int BN, int WM, int WN, int STEPS, bool W_IMAJOR, bool WHOLE16>
Choice<GroupedArgs> grouped_choice() { return {grouped_kernel<Type, BM, BN, WM, WN, STEPS, W_IMAJOR, WHOLE16>, BM, BN, WM * WN * 64}; }
// Float: 64 x 64, of which three workgroups fit a compute unit; its instructions take eight times as long as those of 16 bits, so that fewer reads
// gain little (32768 rows, 8 of 2048 x 2048: 2165 us, 127 TFLOP/s; 128 x 128 2097; but 4096 rows, 8 of 1024 x 2048 171 and 249).  Three steps under
// way: 2227.  Through registers 2500.
template <bool W_IMAJOR>
Choice<GroupedArgs> grouped_f32_choice(bool whole) {
  if (whole) return grouped_choice<F32, 64, 64, 2, 4, 2, W_IMAJOR, true>();
  return {grouped_f32_kernel<64, 64, 2, 4, W_IMAJOR>, 64, 64, 512};
}

// Large tiles need few reads for their products, small ones leave fewer places empty and are more.  By rows an expert has on average,
// where there are as many tiles as compute units: 256 x 256 from 128 rows on (128 matrices of 1536 x 2048, 256 rows each: 286 us, 128 x 128 333),
// 128 x 128 from 48 (32 of 5760 x 2880, 64 rows each: 243 us; 64 x 128 284), otherwise 64 x 128 with three steps under way (12 rows each: 149 and
// 186 us, 5.5 and 5.9 TB/s; 128 x 128 149 and 187; 8 matrices of 512 x 2048: 14 us, 128 x 128 24).
// Through registers the same two smaller tiles (8 experts of 1001 x 1501, 500 rows each: 42 and 47 us; 16 of 333 x 777, 31 rows each: 18 and 15).
template <bool W_IMAJOR, bool WHOLE16>
Choice<GroupedArgs> choose_grouped(int64_t rows, int n_experts, int n) {
  const int64_t mean = rows / n_experts;
  const auto tiles = [&](int tile) { return n_experts * tiles_of(mean, tile) * tiles_of(n, tile); };
  if constexpr (WHOLE16) {
    if (mean >= 128 && tiles(256) >= kComputeUnits) return grouped_choice<Bf16, 256, 256, 2, 4, 2, W_IMAJOR, WHOLE16>();
  }
  if (mean >= 48 && tiles(128) >= kComputeUnits) return grouped_choice<Bf16, 128, 128, 2, 4, 2, W_IMAJOR, WHOLE16>();
  return grouped_choice<Bf16, 64, 128, 2, 4, WHOLE16 ? 3 : 2, W_IMAJOR, WHOLE16>();
}
// Whether a kernel for few rows takes a product.
//   bfloat16, not transposed: up to 16 rows an expert, and up to 48 Mi weights to read.  Beyond that (16 rows of 1536 x 2048: 20.3 us, with tiles
//   20.8; 4 of 5760 x 2880: 31.8 and 28.3) its reads of 64 bytes a row are slower than those of the tiles.  Transposed: never.
//   float, not transposed: the same, and up to 4 rows an expert of any size (32 rows over 128 of 1536 x 2048: 80 us, with tiles 109; 512 rows 349
//   and 386; but 200 over 32 of 2880 x 2880 294 and 288).
//   float, transposed: sums of at least 128 products, and up to 16 rows an expert with up to 48 Mi weights (100 rows of 16 experts, 333 x 777: 9.4 us, with
//   tiles 13.9; but 20 rows of 16, 64 x 64: 7.1 and 4.6), or up to 8 (200 over 32 of 2880 x 2880: 221 and 288; but 400 over 32 of 2880 x 5760 609 and 562).
bool few_rows(int dtype, bool transpose, int64_t rows, int n_experts, int n, int k) {
  if (transpose && (dtype != MOE_SPEC_F32 || n < 128)) return false;
  if (dtype == MOE_SPEC_F32 && rows <= (transpose ? 8 : 4) * int64_t(n_experts)) return true;
  return rows <= 16 * int64_t(n_experts) && (rows < n_experts ? rows : n_experts) * int64_t(n) * k <= int64_t(48) << 20;
}

// How a weight gradient is split: tiles of the matrices, and parts of each expert's rows where those alone leave half of the compute units
// without work and the rows are many (192 of them for a part, three steps).  3 experts of 224 x 544, 11000 rows each: 149 -> 30 us; one of
// 1024 x 1024, 8192 rows: 89 -> 34; but 8 of 1024 x 512, 2048 rows each, 256 tiles in two parts: 38 -> 41, so not there.
struct WeightGradSplit { int tile, parts; };
WeightGradSplit split_weight_grad(int dtype, bool whole, int64_t rows, int n_experts, int n, int k) {
  const auto tiles = [&](int b) { return n_experts * tiles_of(n, b) * tiles_of(k, b); };
  const bool narrow = dtype == MOE_SPEC_F32 || (whole && n <= 64 && k <= 64);
  if (!narrow && whole && tiles(256) >= kComputeUnits) return {256, 1};
  const int tile = narrow ? 64 : 128;
  int64_t parts = tiles(tile) > kComputeUnits / 2 ? 1 : 2 * kComputeUnits / tiles(tile);
  const int64_t most = rows / n_experts / (3 * kPartRows);
  if (parts > most) parts = most;
  return {tile, int(parts < 1 ? 1 : parts > 64 ? 64 : parts)};
}

// Through registers: 99 experts of 72 x 218 9.6 us with 64 x 128, 12.7 with 128 x 128; 8 of 1001 x 1501, 4000 rows, 42 and 39.
Choice<WeightGradArgs> staged_weight_grad(int n_experts, int n, int k) {
  if (n_experts * tiles_of(n, 128) * tiles_of(k, 128) >= kComputeUnits) return {weight_grad_kernel<Bf16, 128, 128, 2, 4, 2, false>, 128, 128, 512};
  return {weight_grad_kernel<Bf16, 64, 128, 2, 4, 2, false>, 64, 128, 512};
}

}  // namespace
}  // namespace moe_spec

using namespace moe_spec;

extern "C" int moe_spec_grouped_product(void *stream, int dtype, const void *x, int64_t x_stride, int64_t rows, const void *w, int64_t w_stride,
                                        int64_t w_expert_stride, int n_experts, int n, int k, const int32_t *ends, int transpose,
                                        int out_dtype, void *y, int64_t y_stride) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: unknown dtype %d", dtype);
  if (!known_type(out_dtype)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: unknown out_dtype %d", out_dtype);
  if (const char *why = sizes_fault(rows, n_experts, n, k)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: %s", why);
  const int in = transpose ? n : k, out = transpose ? k : n, elem = size_of(dtype);
  if (rows == 0) return MOE_SPEC_OK;
  if (const char *why = matrix_fault(x, x_stride, rows, in, elem, false)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: x %s", why);
  if (const char *why = matrix_fault(w, w_stride, n, k, elem, false)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: w %s", why);
  if (const char *why = matrix_fault(y, y_stride, rows, out, size_of(out_dtype), true)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: y %s", why);
  if (n_experts > 1 && (w_expert_stride < 0 || w_expert_stride > kMostExpertStride))
    return train_fail(MOE_SPEC_EINVAL, "grouped_product: w_expert_stride must be between 0 and 2^40");
  if (!ends || misaligned(ends, 4)) return train_fail(MOE_SPEC_EINVAL, "grouped_product: ends is null or not aligned to its elements");
  if (y == x || y == w) return train_fail(MOE_SPEC_EINVAL, "grouped_product: y must not be x or w");
  if (rows == 1) x_stride = in, y_stride = out;         // strides that are never taken are not looked at
  if (n == 1) w_stride = k;
  if (n_experts == 1) w_expert_stride = 0;
  GroupedArgs a{x, w, y, ends, x_stride, w_stride, w_expert_stride, y_stride, in, int(rows), n_experts, out, 0, out_dtype == MOE_SPEC_BF16};
  const bool whole = whole16(x, x_stride, in, elem) && whole16(w, w_stride, k, elem) && w_expert_stride % (16 / elem) == 0;
  const bool few = few_rows(dtype, transpose, rows, n_experts, n, k), wide = dtype == MOE_SPEC_F32;
  const Choice<GroupedArgs> c = few && transpose ? Choice<GroupedArgs>{grouped_few_transposed_kernel, 16, kFewTCols, kFewTBlock}
                                : few ? Choice<GroupedArgs>{wide ? grouped_few_kernel<float> : grouped_few_kernel<uint16_t>, 16, 16, kFewBlock}
                                : wide ? (transpose ? grouped_f32_choice<true>(whole) : grouped_f32_choice<false>(whole))
                                : transpose           ? (whole ? choose_grouped<true, true>(rows, n_experts, out) : choose_grouped<true, false>(rows, n_experts, out))
                                                      : (whole ? choose_grouped<false, true>(rows, n_experts, out) : choose_grouped<false, false>(rows, n_experts, out));
  a.tiles_n = int(tiles_of(out, c.bn));
  const unsigned grid = grid_of(row_tiles(rows, n_experts, c.bm) * a.tiles_n, c.threads);
  if (!grid) return train_fail(MOE_SPEC_EINVAL, "grouped_product: more rows and columns than one launch can take");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  const hipError_t e = on.error() == hipSuccess ? launch(c.kernel, grid, c.threads, s, a) : on.error();
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "grouped_product: %s", hipGetErrorString(e));
}

extern "C" size_t moe_spec_grouped_weight_grad_workspace_bytes(int dtype, int64_t rows, int n_experts, int n, int k) {
  if (!known_type(dtype) || sizes_fault(rows, n_experts, n, k)) return 0;
  const int parts = split_weight_grad(dtype, true, rows, n_experts, n, k).parts;
  return parts > 1 ? size_t(parts) * n_experts * n * k * 4 : 0;
}

extern "C" int moe_spec_grouped_weight_grad(void *stream, int dtype, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                                            int64_t rows, int n_experts, int n, int k, const int32_t *ends, int out_dtype, void *dw,
                                            int64_t dw_stride, int64_t dw_expert_stride, void *workspace, size_t workspace_bytes) {
  if (!known_type(dtype)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: unknown dtype %d", dtype);
  if (!known_type(out_dtype)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: unknown out_dtype %d", out_dtype);
  if (const char *why = sizes_fault(rows, n_experts, n, k)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: %s", why);
  const int elem = size_of(dtype);
  if (const char *why = matrix_fault(dy, dy_stride, rows, n, elem, false)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: dy %s", why);
  if (const char *why = matrix_fault(x, x_stride, rows, k, elem, false)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: x %s", why);
  if (const char *why = matrix_fault(dw, dw_stride, n, k, size_of(out_dtype), true)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: dw %s", why);
  if (n == 1) dw_stride = k;
  if (n_experts > 1 && (dw_expert_stride < (n - 1) * dw_stride + k || dw_expert_stride > kMostExpertStride))
    return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: dw_expert_stride is below a matrix or above 2^40");
  if (!ends || misaligned(ends, 4)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: ends is null or not aligned to its elements");
  if (rows && (dw == dy || dw == x)) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: dw must not be dy or x");
  if (rows <= 1) dy_stride = n, x_stride = k;
  if (n_experts == 1) dw_expert_stride = 0;
  const bool whole = whole16(dy, dy_stride, n, elem) && whole16(x, x_stride, k, elem);
  // the workspace is that of sixteen-byte rows, whatever these are, so that its size goes by sizes alone
  const WeightGradSplit split = split_weight_grad(dtype, true, rows, n_experts, n, k);
  const size_t need = moe_spec_grouped_weight_grad_workspace_bytes(dtype, rows, n_experts, n, k);
  if (need && (!workspace || misaligned(workspace, 16) || workspace_bytes < need))
    return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: the workspace is null, not aligned to 16 bytes or smaller than %zu bytes", need);
  WeightGradArgs a{dy, x, dw, ends, dy_stride, x_stride, dw_stride, dw_expert_stride, int(rows), n_experts, n, k, 0, 0, out_dtype == MOE_SPEC_BF16, split.parts,
                   static_cast<float *>(workspace), int64_t(n_experts) * n * k * size_of(out_dtype) > kCacheBytes};
  // Large tiles take four steps of 32 rows: an expert's rows are few steps, and the first arrives sooner (512 rows an expert, 128 of
  // 1536 x 2048: 562 -> 521 us).
  const Choice<WeightGradArgs> c = dtype == MOE_SPEC_F32 ? Choice<WeightGradArgs>{whole ? weight_grad_kernel<F32, 64, 64, 2, 4, 2, true> : weight_grad_f32_kernel<64, 64, 2, 4>, 64, 64, 512}
                                   : !whole              ? staged_weight_grad(n_experts, n, k)
                                   : split.tile == 256   ? Choice<WeightGradArgs>{weight_grad_kernel<Bf16, 256, 256, 2, 4, 4, true, 32>, 256, 256, 512}
                                   : split.tile == 128   ? Choice<WeightGradArgs>{weight_grad_kernel<Bf16, 128, 128, 2, 4, 2, true>, 128, 128, 512}
                                                         : Choice<WeightGradArgs>{weight_grad_kernel<Bf16, 64, 64, 2, 2, 4, true>, 64, 64, 256};
  a.tiles_n = int(tiles_of(n, c.bm));
  a.tiles_k = int(tiles_of(k, c.bn));
  const unsigned grid = grid_of(int64_t(n_experts) * a.parts * tiles_of(int64_t(a.tiles_n) * a.tiles_k, 8) * 8, c.threads);
  if (!grid) return train_fail(MOE_SPEC_EINVAL, "grouped_weight_grad: more experts' values than one launch can take");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const OnDeviceOf on(s);
  hipError_t e = on.error() == hipSuccess ? launch(c.kernel, grid, c.threads, s, a) : on.error();
  if (e == hipSuccess && a.parts > 1) e = launch(weight_grad_join_kernel, unsigned((int64_t(n_experts) * n * tiles_of(k, 4) + 255) / 256), 256, s, a);
  return e == hipSuccess ? MOE_SPEC_OK : train_fail(MOE_SPEC_EHIP, "grouped_weight_grad: %s", hipGetErrorString(e));
}
