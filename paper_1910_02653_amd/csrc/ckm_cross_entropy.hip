// Softmax cross entropy of hidden states against a vocabulary's table, without the
// logits, and its gradient.
//
//   forward   l = x W', lse = log sum over v of exp l, loss = lse - l_target
//   gradient  d = (exp(l - lse) - 1[v = target]) dloss, dx = d W, dW = d' x
//
// Forward: a tile of the logits stays in registers; of each of its rows remain the
// largest logit and the sum of exponentials, which a second launch joins over the
// tiles in their order. 64 columns have one base and one sum, two of them are joined, and two
// of these: the same sums in every shape of tile. Gradient: the vocabulary in pieces; a piece's logits are
// computed again, d is written for that piece alone, in the tensors' type, and the two
// products after it read it from the caches; dx is summed over pieces in binary32.
//
// In 16 bits d is held relative to s, the largest |dloss|, and the products' results are
// multiplied by s: of a mean, where every row has the same dloss, a target's d is then
// near -1, whose rounding is small; that of dloss itself would be off by as much in
// every row, up to 2^-9 in bfloat16 and the same way. binary16, whose exponents are
// too few (exp(l - lse) is about 1 / vocab), holds d 2^15 / s, of at most 32768.
//
// Bound by the products: f16 2048x2048x32768 234 us (1180 TFLOP/s), its gradient 739 (the
// least of a trace: the copy 6, logits 262, dx 221 and 19 for its shares, dW 239); bf16
// 4096x4096x131072 10.0 ms (1320 TFLOP/s) in eight pieces; f32 2048x1024x32768 986 us and 2980,
// 139 of 154 TFLOP/s. A tile's exponentials are a difference, a product and one 2^x each. Few
// rows are bound by reading the table: bf16 16x4096x50021 85 us, 410 MB at 4.8 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "ckm_matrix.h"

namespace ckm {
namespace {

constexpr float kLog2e = 1.44269504f;
template <typename T>
constexpr float kGain = std::is_same<T, _Float16>::value ? 32768.0f : 1.0f;
template <typename T>
constexpr bool kRelative = sizeof(T) == 2;       // d relative to the largest |dloss|

struct LossArgs {
  ProductArgs p;            // n: of the vocabulary, or of a piece of it
  int32_t tiles_m, tiles_n;
  const int64_t* targets;
  float2* parts;            // [rows][tiles_all]: base and sum of exponentials (join_parts)
  float* hit;               // [rows]: the target's logit
  float* loss;
  float* lse;               // written, or the gradient's input
  const float* dloss;
  const float* most;        // 16 bits: the largest |dloss|
  void* d;                  // [rows][ld_d]
  int64_t ld_d, first;      // first: the piece's first column
  int32_t tile0, tiles_all; // its first tile, of all
  bool pairs;               // tiles of 128 columns
  int64_t vocab;
};

// e^(v - base) for v <= base or so. The difference first: its rounding is relative to
// itself, so that logits of any size keep their distances (v log2 e less a rounded base
// log2 e, one operation instead of two, is off by 2^7 and more past logits of 2^31, and was
// no faster: f16 2048x2048x32768 255 to 259 us both).
template <typename T>
__device__ __forceinline__ float power_of(float v, float base) {
  if constexpr (std::is_same<T, float>::value) return expf(v - base);
  else return __builtin_amdgcn_exp2f((v - base) * kLog2e);
}

// (base, sum): sum e^base of exponentials, whose largest is e^base; sum 0: none.
__device__ __forceinline__ float2 join_parts(float2 p, float2 q) {
  if (q.y == 0.0f) return p;
  if (p.y == 0.0f) return q;
  const float base = fmaxf(p.x, q.x);   // a NaN is in the sums too
  return make_float2(base, p.y * power_of<_Float16>(p.x, base) + q.y * power_of<_Float16>(q.x, base));
}

template <class P>
__global__ void __launch_bounds__(P::kThreads, P::kWaveSlots) ckm_loss_kernel(LossArgs a) {
  using T = typename P::T;
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
  const P p;
  int tm, tn;
  tile_of(blockIdx.x, a.tiles_m, a.tiles_n, tm, tn);
  F4 acc[P::kFN][P::kFM];
  p.run(acc, a.p, tm * P::kM, tn * P::kN, 0, (a.p.k + P::kStep - 1) / P::kStep, (LdsChar*)lds);
  // a group: 64 columns, which one wave has, or two
  constexpr bool kWhole = P::kFN == 4;
  static_assert(kWhole || (P::kFN == 2 && P::kFM == 1 && P::kWavesN == 4), "");
  float2* joined = (float2*)lds;   // [groups of the tile][its rows]
  if (a.p.n - tn * P::kN < P::kN) {   // columns past the vocabulary count for nothing
#pragma unroll
    for (int j = 0; j < P::kFN; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (tn * P::kN + p.col(j) + k >= a.p.n)
#pragma unroll
          for (int i = 0; i < P::kFM; ++i) acc[j][i][k] = -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < P::kFM; ++i) {
    const int m = tm * P::kM + p.row(i);
    const int64_t target = m < a.p.m ? a.targets[m] - a.first - (int64_t)tn * P::kN : -1;   // within the tile
    if (target >= 0 && target < P::kN && target < a.p.n - tn * P::kN) {
#pragma unroll
      for (int j = 0; j < P::kFN; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (p.col(j) + k == (int)target) a.hit[m] = acc[j][i][k];
    }
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < P::kFN; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) most = fmaxf(most, acc[j][i][k]);
    // the four lanes that hold a row
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    if constexpr (!kWhole) {
      float* mosts = (float*)(lds + 4096);   // [waves][rows]
      if (p.lane < 16) mosts[p.wn * 16 + p.lane] = most;
      __syncthreads();
      most = fmaxf(most, mosts[(p.wn ^ 1) * 16 + (p.lane & 15)]);
    }
    const float base = most == -INFINITY ? 0.0f : most;
    float sum[4] = {};
    if constexpr (!kWhole) {   // the second wave of a group adds to the first one's sums
      F4* sums = (F4*)(lds + 8192);   // [groups][lanes]
      F4 first = {power_of<T>(acc[0][i][0], base), power_of<T>(acc[0][i][1], base), power_of<T>(acc[0][i][2], base),
                  power_of<T>(acc[0][i][3], base)};
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] = power_of<T>(acc[1][i][k], base);
      if (p.wn % 2 == 0) sums[p.wn / 2 * 64 + p.lane] = F4{first[0] + sum[0], first[1] + sum[1], first[2] + sum[2], first[3] + sum[3]};
      __syncthreads();
      first += sums[p.wn / 2 * 64 + p.lane];
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] += first[k];
    } else {
#pragma unroll
      for (int j = 0; j < P::kFN; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += power_of<T>(acc[j][i][k], base);
    }
    float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    all += __shfl_xor(all, 16);
    all += __shfl_xor(all, 32);
    if (p.lane < 16 && (kWhole || p.wn % 2 == 1)) joined[(kWhole ? p.wn : p.wn / 2) * P::kM + p.row(i)] = make_float2(base, all);
  }
  __syncthreads();
  for (int r = threadIdx.x; r < P::kM; r += P::kThreads) {
    const int m = tm * P::kM + r;
    if (m >= a.p.m) continue;
    float2 v = join_parts(joined[r], joined[P::kM + r]);
    if constexpr (P::kN == 256) v = join_parts(v, join_parts(joined[2 * P::kM + r], joined[3 * P::kM + r]));
    a.parts[(int64_t)m * a.tiles_all + a.tile0 + tn] = v;
  }
}

// Part k of a row's `all`, of 256 columns (two of 128 where tiles have so many).
__device__ __forceinline__ float2 part_of(const LossArgs& a, const float2* parts, int k) {
  if (!a.pairs) return parts[k];
  return 2 * k + 1 < a.tiles_all ? join_parts(parts[2 * k], parts[2 * k + 1]) : parts[2 * k];
}
// A wave a row: the parts in their order (each lane every 64th, then the lanes).
__global__ void __launch_bounds__(256) ckm_loss_join_kernel(LossArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.p.m) return;
  const float2* parts = a.parts + row * a.tiles_all;
  const int all = a.pairs ? (a.tiles_all + 1) / 2 : a.tiles_all;
  float base = -INFINITY, sum = 0.0f;
  for (int k = lane; k < all; k += 64) {
    const float2 v = part_of(a, parts, k);
    base = fmaxf(base, v.y == 0.0f ? -INFINITY : v.x);
  }
  base = reduce64<OpMax>(base);
  if (base == -INFINITY) base = 0.0f;
  for (int k = lane; k < all; k += 64) {
    const float2 v = part_of(a, parts, k);
    if (v.y != 0.0f) sum += v.y * power_of<_Float16>(v.x, base);
  }
  sum = reduce64<OpSum>(sum);
  if (lane == 0) {
    const float lse = base + logf(sum);
    const int64_t target = a.targets[row];
    if (a.lse) a.lse[row] = lse;
    if (a.loss) a.loss[row] = target >= 0 && target < a.vocab ? lse - a.hit[row] : 0.0f;
  }
}

template <class P>
__global__ void __launch_bounds__(P::kThreads, P::kWaveSlots) ckm_loss_back_kernel(LossArgs a) {
  using T = typename P::T;
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
  const P p;
  int tm, tn;
  tile_of(blockIdx.x, a.tiles_m, a.tiles_n, tm, tn);
  F4 acc[P::kFN][P::kFM];
  p.run(acc, a.p, tm * P::kM, tn * P::kN, 0, (a.p.k + P::kStep - 1) / P::kStep, (LdsChar*)lds);
  const int width = (int)whole(a.p.n, 16 / sizeof(T));   // zeros to the end of a group
#pragma unroll
  for (int i = 0; i < P::kFM; ++i) {
    const int m = tm * P::kM + p.row(i);
    const bool live = m < a.p.m;
    int64_t target = live ? a.targets[m] : -1;
    const bool some = target >= 0 && target < a.vocab;
    target -= a.first + (int64_t)tn * P::kN;   // within the tile
    const float base = live ? a.lse[m] : 0.0f;
    float by = some ? a.dloss[m] : 0.0f;
    if constexpr (kRelative<T>) by = by / *a.most * kGain<T>;
#pragma unroll
    for (int j = 0; j < P::kFN; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[j][i][k] = some ? power_of<T>(acc[j][i][k], base) * by : 0.0f;
    if (some && target >= 0 && target < P::kN) {
#pragma unroll
      for (int j = 0; j < P::kFN; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (p.col(j) + k == (int)target) acc[j][i][k] -= by;
    }
  }
  if (a.p.n - tn * P::kN < P::kN) {
#pragma unroll
    for (int j = 0; j < P::kFN; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (tn * P::kN + p.col(j) + k >= a.p.n)
#pragma unroll
          for (int i = 0; i < P::kFM; ++i) acc[j][i][k] = 0.0f;
  }
  p.template each8<1>(acc, (LdsChar*)lds, [&](int row, int col, float (&v)[1][8]) {
    const int m = tm * P::kM + row, n = tn * P::kN + col;
    if (m < a.p.m && n < width) store_part<false>((T*)a.d + m * a.ld_d, rounded8<T>(v[0]), n, width);
  });
}

template <typename T, bool kBack>
void launch_logits(LossArgs a, const Cut& cut, hipStream_t s) {
  a.tiles_m = cut.tiles_m;
  a.tiles_n = (a.p.n + cut.cols - 1) / cut.cols;   // fewer in the last piece
  with_shape<T, true, true, 1>(cut, [&](auto p) {
    using P = typename decltype(p)::Shape;
    const uint32_t blocks = (uint32_t)(a.tiles_m * a.tiles_n);
    if constexpr (kBack) ckm_loss_back_kernel<P><<<blocks, P::kThreads, 0, s>>>(a);
    else ckm_loss_kernel<P><<<blocks, P::kThreads, 0, s>>>(a);
  });
}

// A piece of the vocabulary: in the gradient d of at most 128 MB, which stays in the caches
// between its writer and its readers, but never fewer than 8192 columns: dx, summed over
// pieces in memory, is read and written for each. Past 8192 rows (4096 of binary32) d grows
// with them, out of the caches: 1 GB at 65536 rows of 16 bits, as much as dx's sums at width 4096. Pieces of the gradient go by the sizes, as
// the sums' order does. Where the table has to be copied: forward 96 MB pieces of it; in the
// gradient a piece; of a piece of more than 4 GB (vast tables, few rows) as many shares of dx
// as take that, so that the copy's room has a bound (their launches fill fewer CUs: bf16
// 16x4097x300000, 2.5 GB, 2.9 ms whole and 4.2 in three parts).
constexpr int64_t kPieceBytes = (int64_t)128 << 20, kTableBytes = (int64_t)96 << 20, kLeastPiece = 8192;
constexpr int64_t kCopyBytes = (int64_t)4 << 30;

struct LossPlan {
  bool pack_x, pack_w;
  int64_t ld_x, ld_w;
  int64_t piece;             // columns
  int64_t copied;            // columns of the table in the work buffer at a time: of a piece, or of some of dx's shares
  Cut logits, dx, dw;
  bool together;             // dx and dW in a launch
  size_t x, w, parts, hit, most, d, slab, dw_slab, total;
  double time;               // the model's, us
};

// packed: operands that cannot be loaded as they are are copied, or else staged.
LossPlan plan_as(int type, const ckm_vocab& c, bool back, bool ragged_x, bool ragged_w, bool packed) {
  const size_t elt = dtype_bytes(type);
  const int64_t group = 16 / elt, step = kStepBytes / elt;
  LossPlan p = {};
  // the gradient takes a copy whose rows without a target are zeros: in d' x they are
  // multiplied by d's zeros, and may hold anything
  p.pack_x = back || (ragged_x && packed);
  p.pack_w = ragged_w && packed;
  p.ld_x = p.pack_x || c.rows == 1 ? whole(c.hidden, group) : c.ld_x;
  p.ld_w = p.pack_w || c.vocab == 1 ? whole(c.hidden, group) : c.ld_weight;
  const bool staged_x = ragged_x && !p.pack_x, staged_w = ragged_w && !packed;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at = whole(at + bytes, 256);
    return here;
  };
  if (p.pack_x) p.x = take(c.rows * p.ld_x * elt);
  // pieces of at most so many columns, as many in each
  const auto piece_of = [&](int64_t most) {
    const int64_t pieces = (c.vocab + std::max(most, kLeastPiece) - 1) / std::max(most, kLeastPiece);
    return std::min(c.vocab, whole((c.vocab + pieces - 1) / pieces, 256));
  };
  int64_t most = ((int64_t)1 << 30) / ((c.rows + 255) / 256);   // 2^22 tiles in a launch
  if (back) most = std::min(most, kPieceBytes / (int64_t)(c.rows * elt));
  const int64_t all = piece_of(most);   // were the table not copied
  p.piece = p.pack_w && !back ? std::min(all, piece_of(std::min(most, kTableBytes / (int64_t)(c.hidden * elt)))) : all;
  p.copied = p.piece;
  const int64_t steps = (c.hidden + step - 1) / step, x_bytes = c.rows * c.hidden * elt, w_bytes = p.piece * c.hidden * elt;
  p.logits = cut_product(type, c.rows, p.piece, 1, 1, steps, x_bytes + w_bytes, false, true);
  if (staged_x || staged_w)
    p.logits = cut_like(type, c.rows, p.piece, 1, 1, steps, x_bytes + w_bytes, true, kStagedAlong, p.logits);
  p.time = p.logits.time + (p.pack_w ? copy_time(w_bytes) : 0.0);
  if (!back) {   // pieces are of whole tiles, and of whole pairs
    p.parts = take((size_t)c.rows * ((c.vocab + p.logits.cols - 1) / p.logits.cols) * sizeof(float2));
    p.hit = take(c.rows * sizeof(float));
  } else {
    const int64_t d_bytes = p.piece * c.rows * elt;
    const int64_t steps_v = (p.piece + step - 1) / step, steps_m = (c.rows + step - 1) / step;
    p.dx = cut_product(type, c.rows, c.hidden, 1, 1, steps_v, d_bytes + w_bytes, true, true);
    p.dw = cut_product(type, p.piece, c.hidden, 1, 1, steps_m, d_bytes + x_bytes + w_bytes, true, false);
    p.together = cut_together(type, p.dx, c.rows, c.hidden, steps_v, p.dw, p.piece, c.hidden, steps_m,
                              d_bytes + x_bytes + 2 * w_bytes);
    if (staged_w) {
      p.together = false;
      p.dx = cut_like(type, c.rows, c.hidden, 1, 1, steps_v, d_bytes + w_bytes, true, kStagedAcross, p.dx);
      p.dw = cut_like(type, p.piece, c.hidden, 1, 1, steps_m, d_bytes + x_bytes + w_bytes, false, kStraight, p.dw);
    }
    p.time += p.dx.time + p.dw.time;
    const int64_t share = p.dx.steps * step, most_shares = kCopyBytes / (int64_t)(share * p.ld_w * elt);
    if (p.pack_w && p.dx.splits > 1) p.copied = std::min(p.piece, std::max<int64_t>(1, most_shares) * share);
    p.most = take(sizeof(float));
    p.d = take((size_t)c.rows * row_of(p.piece, elt) * elt);
    if (p.dx.splits > 1 || p.piece < c.vocab) p.slab = take((size_t)p.dx.splits * c.rows * whole(c.hidden, 8) * 4);
    if (p.dw.splits > 1) p.dw_slab = take((size_t)p.dw.splits * p.piece * whole(c.hidden, 8) * 4);
  }
  if (p.pack_w) p.w = take(p.copied * p.ld_w * elt);
  p.time *= (double)c.vocab / p.piece;
  if (!back && p.pack_x) p.time += copy_time(x_bytes);
  p.total = at;
  return p;
}

LossPlan plan_of(int type, const ckm_vocab& c, bool back) {
  const size_t elt = dtype_bytes(type);
  const bool x = !loadable(c.d_x, c.rows, c.hidden, c.ld_x, elt, true);
  const bool w = !loadable(c.d_weight, c.vocab, c.hidden, c.ld_weight, elt, true);
  const LossPlan p = plan_as(type, c, back, x, w, true);
  if ((!x && !w) || !stageable(c.rows, c.ld_x, elt) || !stageable(c.vocab, c.ld_weight, elt)) return p;
  const LossPlan q = plan_as(type, c, back, x, w, false);
  return q.time < p.time ? q : p;
}

template <typename T>
void launch_loss(int type, const ckm_vocab& c, const LossPlan& plan, bool back, const float* dloss, float* loss,
                 float* lse, void* dx, int64_t ld_dx, void* dw, int64_t ld_dw, char* work, hipStream_t s) {
  const T *x = (const T*)c.d_x, *w = (const T*)c.d_weight;
  if (plan.pack_x) {
    PackArgs one = {};
    if (back) {
      one.targets = c.d_targets;
      one.vocab = c.vocab;
      one.dloss = dloss;
      one.rows = c.rows;
      if (kRelative<T>) one.most = (float*)(work + plan.most);
    }
    one.add(x, c.rows, c.hidden, c.ld_x, work + plan.x, plan.ld_x);
    launch_pack(type, one, s);
    x = (const T*)(work + plan.x);
  }
  // the rows of the table from v on, as they are multiplied
  const auto rows_from = [&](int64_t v, int32_t width) {
    if (!plan.pack_w) return w + v * plan.ld_w;
    PackArgs one = {};
    one.add(w + v * c.ld_weight, width, c.hidden, c.ld_weight, work + plan.w, plan.ld_w);
    launch_pack(type, one, s);
    return (const T*)(work + plan.w);
  };
  LossArgs a = {};
  a.p = {{x, x, plan.ld_x}, {w, w, plan.ld_w}, (int32_t)c.rows, (int32_t)c.vocab, (int32_t)c.hidden, 1};
  a.targets = c.d_targets;
  a.vocab = c.vocab;
  a.lse = lse;
  if (!back) {
    a.parts = (float2*)(work + plan.parts);
    a.hit = (float*)(work + plan.hit);
    a.loss = loss;
    a.tiles_all = (int32_t)((c.vocab + plan.logits.cols - 1) / plan.logits.cols);
    a.pairs = plan.logits.cols == 128;
    for (int64_t v = 0; v < c.vocab; v += plan.piece) {
      a.first = v;
      a.tile0 = (int32_t)(v / plan.logits.cols);
      a.p.n = (int32_t)std::min(plan.piece, c.vocab - v);
      a.p.b.p = rows_from(v, a.p.n);
      launch_logits<T, false>(a, plan.logits, s);
    }
    ckm_loss_join_kernel<<<(uint32_t)((c.rows + 3) / 4), 256, 0, s>>>(a);
    return;
  }
  a.dloss = dloss;
  if (kRelative<T>) a.most = (const float*)(work + plan.most);
  a.ld_d = row_of(plan.piece, sizeof(T));
  ResultArgs rx = {}, rw = {};
  rx.alpha = rw.alpha = a.most;
  rx.factor = rw.factor = 1.0f / kGain<T>;
  const bool slab = plan.dx.splits > 1 || plan.piece < c.vocab;
  if (slab) rx.slab = (float*)(work + plan.slab);
  rx.ld_slab = rw.ld_slab = whole(c.hidden, 8);
  rx.c[0] = dx;
  rx.ld_c[0] = ld_dx;
  rx.halves = rw.halves = 1;
  if (plan.dw.splits > 1) rw.slab = (float*)(work + plan.dw_slab);
  rw.ld_c[0] = ld_dw;
  T* const d = (T*)(work + plan.d);
  for (int64_t v = 0; v < c.vocab; v += plan.piece) {
    const int32_t width = (int32_t)std::min(plan.piece, c.vocab - v);
    const bool whole = width <= plan.copied, both = plan.together && dx && dw && whole;
    // d' x
    rw.p = {{d, d, a.ld_d}, {x, x, plan.ld_x}, width, (int32_t)c.hidden, (int32_t)c.rows, 1};
    rw.c[0] = (T*)dw + v * ld_dw;
    Cut cut = plan.dw;
    cut.tiles_m = (width + cut.rows - 1) / cut.rows;
    for (int64_t u = 0; u < width; u += plan.copied) {
      const int32_t now = (int32_t)std::min(plan.copied, width - u);
      const T* wv = rows_from(v + u, now);
      a.first = v + u;
      a.p.b.p = a.p.b.q = wv;
      a.p.n = now;
      a.d = d + u;
      launch_logits<T, true>(a, plan.logits, s);
      // d W, all shares or those of these columns; a short last piece leaves shares at the end of k with nothing to add
      rx.p = {{d + u, d + u, a.ld_d}, {wv, wv, plan.ld_w}, (int32_t)c.rows, (int32_t)c.hidden, now, 1};
      Cut shares = plan.dx;
      if (!whole) {
        const int64_t share = plan.dx.steps * (kStepBytes / (int64_t)sizeof(T));
        shares.splits = (int)((now + share - 1) / share);
        rx.slab = (float*)(work + plan.slab) + u / share * c.rows * rx.ld_slab;
      }
      if (both) launch_two<T, false>(rx, shares, rw, cut, s);
      else if (dx) launch_product<T, true, false>(rx, shares, s);
    }
    if (slab) rx.slab = (float*)(work + plan.slab);
    rx.add = true;
    if (dw && !both) {
      launch_product<T, false, false>(rw, cut, s);
      if (cut.splits > 1) launch_join(type, rw, cut.splits, s);
    }
  }
  if (dx && slab) launch_join(type, rx, plan.dx.splits, s);
}

ckm_status check_vocab(ckm_dtype type, const ckm_vocab* c) {
  if (!dtype_ok(type)) return set_error(CKM_E_INVALID_ARG, "unknown type %d", (int)type);
  if (!c) return set_error(CKM_E_INVALID_ARG, "vocab is NULL");
  if (c->rows < 0 || c->hidden < 1 || c->vocab < 1)
    return set_error(CKM_E_INVALID_ARG, "%lld rows, hidden width %lld, vocabulary of %lld", (long long)c->rows,
                     (long long)c->hidden, (long long)c->vocab);
  if (c->rows > CKM_MAX_MATRIX_ROWS || c->hidden > CKM_MAX_MATRIX_COLS || c->vocab > CKM_MAX_VOCAB)
    return set_error(CKM_E_UNSUPPORTED, "%lld rows, hidden width %lld, vocabulary of %lld", (long long)c->rows,
                     (long long)c->hidden, (long long)c->vocab);
  const size_t elt = dtype_bytes(type);
  ckm_status st;
  if ((st = check_matrix(c->d_weight, "weight", c->vocab, c->hidden, c->ld_weight, elt, false)) != CKM_OK) return st;
  if (!c->rows) return CKM_OK;
  if ((st = check_matrix(c->d_x, "x", c->rows, c->hidden, c->ld_x, elt, false)) != CKM_OK) return st;
  return check_matrix(c->d_targets, "targets", 1, c->rows, 0, 8, false);
}

ckm_status loss(ckm_dtype type, const ckm_vocab* c, bool back, const float* dloss, float* loss_out, float* lse,
                void* dx, int64_t ld_dx, void* dw, int64_t ld_dw, void* work, size_t work_bytes, void* stream) {
  ckm_status st = check_vocab(type, c);
  if (st != CKM_OK) return st;
  const size_t elt = dtype_bytes(type);
  const hipStream_t s = (hipStream_t)stream;
  if (dw && (st = check_matrix(dw, "dweight", c->vocab, c->hidden, ld_dw, elt, true)) != CKM_OK) return st;
  const Place x = {"x", c->d_x, c->rows, c->hidden, c->ld_x, elt}, w = {"weight", c->d_weight, c->vocab, c->hidden, c->ld_weight, elt};
  if (c->rows == 0) {
    if (!dw) return CKM_OK;
    if ((st = check_apart({{"dweight", dw, c->vocab, c->hidden, ld_dw, elt}}, {w})) != CKM_OK) return st;
    launch_zero(type, dw, c->vocab, c->hidden, ld_dw, s);
    return launched("cross entropy gradient launch");
  }
  if (back) {
    if ((st = check_matrix(dloss, "dloss", 1, c->rows, 0, 4, false)) != CKM_OK) return st;
    if ((st = check_matrix(lse, "lse", 1, c->rows, 0, 4, false)) != CKM_OK) return st;
    if (dx && (st = check_matrix(dx, "dx", c->rows, c->hidden, ld_dx, elt, true)) != CKM_OK) return st;
    if (!dx && !dw) return CKM_OK;
  } else {
    if ((uintptr_t)loss_out % 4 || (uintptr_t)lse % 4)
      return set_error(CKM_E_INVALID_ARG, "loss or lse is not aligned to 4 bytes");
    if (!loss_out && !lse) return CKM_OK;
  }
  const Place targets = {"targets", c->d_targets, 1, c->rows, 0, 8}, sums = {"lse", lse, 1, c->rows, 0, 4};
  st = back ? check_apart({{"dx", dx, c->rows, c->hidden, ld_dx, elt}, {"dweight", dw, c->vocab, c->hidden, ld_dw, elt}},
                          {x, w, targets, sums, {"dloss", dloss, 1, c->rows, 0, 4}})
            : check_apart({{"loss", loss_out, 1, c->rows, 0, 4}, sums}, {x, w, targets});
  if (st != CKM_OK) return st;
  const LossPlan plan = plan_of(type, *c, back);
  if ((st = check_blocks(plan.logits)) != CKM_OK) return st;
  if (back && ((st = check_blocks(plan.dx)) != CKM_OK || (st = check_blocks(plan.dw)) != CKM_OK)) return st;
  if (plan.total && (!work || work_bytes < plan.total))
    return set_error(CKM_E_INVALID_ARG, "work buffer of %zu bytes, %zu needed", work ? work_bytes : (size_t)0,
                     plan.total);
  if ((uintptr_t)work % 16) return set_error(CKM_E_INVALID_ARG, "work is not aligned to 16 bytes");
  const auto go = [&](auto t) {
    launch_loss<decltype(t)>(type, *c, plan, back, dloss, loss_out, lse, dx, ld_dx, dw, ld_dw, (char*)work, s);
  };
  switch (type) {
    case CKM_F32: go(0.0f); break;
    case CKM_F16: go((_Float16)0); break;
    default: go((__bf16)0.0f); break;
  }
  return launched(back ? "cross entropy gradient launch" : "cross entropy launch");
}

}  // namespace
}  // namespace ckm

extern "C" ckm_status ckm_cross_entropy_workspace_size(ckm_dtype type, const ckm_vocab* vocab, int32_t backward,
                                                       size_t* bytes) {
  using namespace ckm;
  if (!bytes) return set_error(CKM_E_INVALID_ARG, "bytes is NULL");
  const ckm_status st = check_vocab(type, vocab);
  if (st != CKM_OK) return st;
  *bytes = vocab->rows ? plan_of(type, *vocab, backward != 0).total : 0;
  return CKM_OK;
}

extern "C" ckm_status ckm_cross_entropy_async(ckm_dtype type, const ckm_vocab* vocab, float* d_loss, float* d_lse,
                                              void* d_work, size_t work_bytes, void* stream) {
  return ckm::loss(type, vocab, false, nullptr, d_loss, d_lse, nullptr, 0, nullptr, 0, d_work, work_bytes, stream);
}

extern "C" ckm_status ckm_cross_entropy_backward_async(ckm_dtype type, const ckm_vocab* vocab, const float* d_dloss,
                                                       const float* d_lse, void* d_dx, int64_t ld_dx, void* d_dweight,
                                                       int64_t ld_dweight, void* d_work, size_t work_bytes,
                                                       void* stream) {
  return ckm::loss(type, vocab, true, d_dloss, nullptr, const_cast<float*>(d_lse), d_dx, ld_dx, d_dweight, ld_dweight,
                   d_work, work_bytes, stream);
}
