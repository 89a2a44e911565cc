// Layer norm over rows, forward and gradient, with the dropout and the
// residual sum before it in the same pass.
//
//   forward   h = T(r + D(x)) (T: rounded to the tensors' type, since h is a
//             value of its own that other nodes read; h = x when nothing is
//             fused), mean = sum h / n, rstd = 1 / sqrt(sum (h - mean)^2 / n +
//             eps), y = (h - mean) rstd w + b
//   gradient  xh = (h - mean) rstd, g = dy w, dh = rstd (g - sum g / n - xh
//             sum(g xh) / n) + dres, dx = D(T(dh)), dw = sum over rows of dy xh,
//             db = sum over rows of dy
//
// Statistics and sums are in binary32; the variance is summed from the
// centred values, in registers, so that a large mean costs no digits. The
// gradient's products are rounded on their own: in rows of few columns, where dh is
// a small difference of them, opposite elements then stay opposite.
//
// The forward pass reads and writes each element once: a row lives in the
// registers of 16 to 1024 threads, which hold one to four groups of eight columns
// each. The gradient does too up to 16384 columns, with the weights' gradients as
// sums in registers beside the row, and reads its inputs twice beyond that.
//
// Bound by memory on large inputs: the fused forward pass of bf16 8192x8192 moves
// 537 MB in 100 us (5.4 TB/s, where a large copy moves 5.2), the fused gradient of
// bf16 16384x4096 671 MB in 133 us. Small ones are bound by the launch and one
// row's chain of load, two sums and store: f16 2048x2048 6.6 us forward, 14.5 us
// gradient (10.8 and 4 for joining the blocks' sums).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "ckm_ops.h"

namespace ckm {
namespace {

struct NormArgs {
  int32_t rows, cols;
  const void* x;
  int64_t ld_x;
  const void* res;
  int64_t ld_res;
  const void* w;
  const void* b;
  bool w32;           // weights (and their gradients) in binary32 rather than the tensors' type
  float eps;
  void* h;
  int64_t ld_h;
  void* y;
  int64_t ld_y;
  float* stats;       // [rows][2]: mean, rstd
  DropArgs drop;
};

// A group of the weights (or biases) in binary32; `absent` where there are none.
template <typename T>
__device__ __forceinline__ void weight_group(float (&v)[kVec], const void* p, bool w32, int col, int left, float absent) {
  if (!p || left <= 0) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = absent;
  } else if (w32) {
    const Raw8<float> r = load_left((const float*)p + col, left);
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = r.get(j);
  } else {
    const Raw8<T> r = load_left((const T*)p + col, left);
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = (float)r.get(j);
  }
}

constexpr int norm_block(int lanes) { return lanes < 256 ? 256 : lanes; }
// Up to two groups a thread, the weights stay in registers from row to row;
// with four they are read again for each row (from the caches).
constexpr bool keep_weights(int per) { return per <= 2; }

template <typename T, int kLanes, int kPer, bool kFused, bool kEven>
__global__ void __launch_bounds__(norm_block(kLanes)) ckm_norm_kernel(NormArgs a) {
  constexpr int kBlock = norm_block(kLanes), kRowsAt = kBlock / kLanes;   // rows of a block at a time
  __shared__ float lds[kLanes > 64 ? 2 * kBlock / 64 : 1];
  const int lane = threadIdx.x % kLanes;
  const DropSite site = drop_site(a.drop);
  constexpr int kKept = keep_weights(kPer) ? kPer : 1;
  float w[kKept][kVec], b[kKept][kVec];
  if constexpr (keep_weights(kPer)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec;
      weight_group<T>(w[i], a.w, a.w32, col, a.cols - col, 1.0f);
      weight_group<T>(b[i], a.b, a.w32, col, a.cols - col, 0.0f);
    }
  }
  // a residual that is not there adds -0, which leaves a kept zero its sign
  const uint32_t absent = a.res ? 0u : sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
  for (int64_t first = (int64_t)blockIdx.x * kRowsAt; first < a.rows; first += (int64_t)gridDim.x * kRowsAt) {
    const int64_t row = first + row_in_block<kLanes>();
    const bool live = row < a.rows;
    // every load of the row first, then the arithmetic
    Raw8<T> r[kPer], rr[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec, left = live ? a.cols - col : 0;
      r[i] = zero_group<T>();
      if (left > 0) r[i] = load_cols<kEven>((const T*)a.x + row * a.ld_x, col, a.cols);
      if constexpr (kFused) {
        rr[i] = group_of<T>(absent);
        if (a.res && left > 0) rr[i] = load_cols<kEven>((const T*)a.res + row * a.ld_res, col, a.cols);
      }
    }
    float v[kPer][kVec];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int group = lane + i * kLanes, col = group * kVec;
      fix_tail<kEven>(r[i], col, a.cols);
      if constexpr (kFused) {
        const int left = live ? a.cols - col : 0;
        if (a.drop.on) drop_choice(r[i], a.drop, site, group, (uint32_t)row);
        fix_tail<kEven>(rr[i], col, a.cols);
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[i][j] = (float)r[i].get(j) * a.drop.scale + (float)rr[i].get(j);
        const Raw8<T> h = rounded8<T>(v[i]);
        if (a.h && left > 0) store_part<kEven>((T*)a.h + row * a.ld_h, h, col, a.cols);
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[i][j] = (float)h.get(j);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[i][j] = (float)r[i].get(j);
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j) sum += v[i][j];
    }
    const float mean = reduce_row<OpSum, kLanes, kBlock>(sum, lds, 0) / (float)a.cols;
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int left = a.cols - (lane + i * kLanes) * kVec;
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const float d = (kEven ? left > 0 : j < left) ? v[i][j] - mean : 0.0f;
        sq = fmaf(d, d, sq);
      }
    }
    const float rstd = 1.0f / sqrtf(reduce_row<OpSum, kLanes, kBlock>(sq, lds, 1) / (float)a.cols + a.eps);
    if (live) {
      if (lane == 0 && a.stats) {
        a.stats[2 * row] = mean;
        a.stats[2 * row + 1] = rstd;
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int col = (lane + i * kLanes) * kVec, left = a.cols - col;
        if (left <= 0) continue;
        const int k = keep_weights(kPer) ? i : 0;
        if constexpr (!keep_weights(kPer)) {
          weight_group<T>(w[0], a.w, a.w32, col, left, 1.0f);
          weight_group<T>(b[0], a.b, a.w32, col, left, 0.0f);
        }
        float o[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = fmaf((v[i][j] - mean) * rstd, w[k][j], b[k][j]);
        store_part<kEven>((T*)a.y + row * a.ld_y, rounded8<T>(o), col, a.cols);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------

struct NormGradArgs {
  int32_t rows, cols;
  const void* dy;
  int64_t ld_dy;
  const void* h;
  int64_t ld_h;
  const float* stats;
  const void* w;
  bool w32;
  const void* dres;
  int64_t ld_dres;
  void* dh;
  int64_t ld_dh;
  void* dx;
  int64_t ld_dx;
  void* dw;
  void* db;
  float* part;     // [blocks][2][padded columns]: each block's sums over its rows
  DropArgs drop;
};

__host__ __device__ __forceinline__ int padded_cols(int cols) { return (cols + kVec - 1) / kVec * kVec; }

template <typename T>
__device__ __forceinline__ void store_weight(void* p, bool w32, int col, float v) {
  if (w32)
    ((float*)p)[col] = v;
  else
    ((T*)p)[col] = rounded<T>(v);
}

// The gradient of the norm's input, o: rounds and stores it as dh
// and, through the dropout, as dx (of the rounded dh, which other nodes see).
template <typename T, bool kEven>
__device__ __forceinline__ void finish_grad(const NormGradArgs& a, DropSite site, int64_t row, int group,
                                            float (&o)[kVec]) {
  const int col = group * kVec;
  const Raw8<T> r = rounded8<T>(o);
  if (a.dh) store_part<kEven>((T*)a.dh + row * a.ld_dh, r, col, a.cols);
  if (a.dx) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) o[j] = (float)r.get(j);
    store_part<kEven>((T*)a.dx + row * a.ld_dx, dropped8<T>(o, a.drop, site, group, (uint32_t)row), col, a.cols);
  }
}
// A block's sum over its rows for one column (which 0: dw, 1: db): the result
// itself when it is the only block, else one of the parts to be joined.
template <typename T>
__device__ __forceinline__ void put_sum(const NormGradArgs& a, bool only, float* part, int width, int which, int col,
                                        float v) {
  if (!only) {
    if (col < width) part[which * width + col] = v;
  } else if (col < a.cols) {
    void* out = which ? a.db : a.dw;
    if (out) store_weight<T>(out, a.w32, col, v);
  }
}

// The sum of kCount floats `step` apart, as a tree: a small term is not lost beside a
// large one, as in a chain of as many additions.
template <int kCount>
__device__ __forceinline__ float tree_sum(const float* at, int step) {
  if constexpr (kCount == 1)
    return *at;
  else
    return tree_sum<kCount / 2>(at, step) + tree_sum<kCount / 2>(at + kCount / 2 * step, step);
}

constexpr int kGradBlock = 1024;

// A row of the gradient's inputs as a thread holds it, in its own type: its
// products are made twice, since registers are what limits the waves here.
template <typename T, int kPer>
struct GradRow {
  Raw8<T> dy[kPer], h[kPer], past[kPer];
  float mean, rstd;
};
template <int kLanes, bool kEven, typename T, int kPer>
__device__ __forceinline__ void load_grad_row(GradRow<T, kPer>& r, const NormGradArgs& a, int64_t row, int lane) {
  const bool live = row < a.rows;
  r.mean = live ? a.stats[2 * row] : 0.0f;
  r.rstd = live ? a.stats[2 * row + 1] : 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int col = (lane + i * kLanes) * kVec, left = live ? a.cols - col : 0;
    r.dy[i] = r.h[i] = r.past[i] = zero_group<T>();
    if (left > 0) {
      r.dy[i] = load_cols<kEven>((const T*)a.dy + row * a.ld_dy, col, a.cols);
      r.h[i] = load_cols<kEven>((const T*)a.h + row * a.ld_h, col, a.cols);
      if (a.dres) r.past[i] = load_cols<kEven>((const T*)a.dres + row * a.ld_dres, col, a.cols);
    }
  }
}

// One pass over dy and h. A block takes every gridDim-th set of rows, one in each
// of its row places, and keeps its columns' sums of dy xh and dy in registers; at
// the end its places join through LDS in a fixed order, and
// ckm_norm_join_kernel adds the blocks' sums in a fixed order, so the weights'
// gradients do not depend on scheduling.
template <typename T, int kLanes, int kPer, bool kEven>
__global__ void __launch_bounds__(kGradBlock) ckm_norm_grad_kernel(NormGradArgs a) {
  constexpr int kPlaces = kGradBlock / kLanes;
  __shared__ float lds[kLanes > 64 ? 4 * kGradBlock / 64 : 1];
  __shared__ __align__(16) float join[kPlaces > 1 ? kPlaces * 2 * kLanes * kVec : 1];
  const int lane = threadIdx.x % kLanes;
  const DropSite site = drop_site(a.drop);
  int turn = 0;
  // two groups' weights are read again for each row: no registers for them
  constexpr bool kKeep = kPer == 1;
  float w[kVec], dw[kPer][kVec], db[kPer][kVec];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int col = (lane + i * kLanes) * kVec;
    if constexpr (kKeep) weight_group<T>(w, a.w, a.w32, col, a.cols - col, 1.0f);
#pragma unroll
    for (int j = 0; j < kVec; ++j) dw[i][j] = db[i][j] = 0.0f;
  }
  for (int64_t first = (int64_t)blockIdx.x * kPlaces; first < a.rows; first += (int64_t)gridDim.x * kPlaces) {
    const int64_t row = first + row_in_block<kLanes>();
    const bool live = row < a.rows;
    GradRow<T, kPer> r;
    load_grad_row<kLanes, kEven>(r, a, row, lane);
    float s[2] = {};   // sum g, sum g xh
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec, left = live ? a.cols - col : 0;
      fix_tail<kEven>(r.dy[i], col, a.cols);
      fix_tail<kEven>(r.h[i], col, a.cols);
      fix_tail<kEven>(r.past[i], col, a.cols);
      if constexpr (!kKeep) weight_group<T>(w, a.w, a.w32, col, left, 1.0f);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const float d = (float)r.dy[i].get(j);
        const float xh = (kEven ? left > 0 : j < left) ? ((float)r.h[i].get(j) - r.mean) * r.rstd : 0.0f;
        const float g = d * w[j];
        dw[i][j] = fmaf(d, xh, dw[i][j]);
        db[i][j] += d;
        s[0] += g;
        s[1] += g * xh;
      }
    }
    reduce_rows<OpSum, kLanes, kGradBlock>(s, lds, turn);
    turn ^= 1;
    if (!live) continue;
    const float s1 = s[0] / (float)a.cols, s2 = s[1] / (float)a.cols;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int group = lane + i * kLanes, col = group * kVec, left = a.cols - col;
      if (left <= 0) continue;
      if constexpr (!kKeep) weight_group<T>(w, a.w, a.w32, col, left, 1.0f);
      float o[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const float xh = ((float)r.h[i].get(j) - r.mean) * r.rstd;
        o[j] = r.rstd * ((float)r.dy[i].get(j) * w[j] - s1 - xh * s2) + (float)r.past[i].get(j);
      }
      finish_grad<T, kEven>(a, site, row, group, o);
    }
  }
  if (!a.dw && !a.db) return;
  const bool only = gridDim.x == 1;
  const int width = padded_cols(a.cols);
  float* part = a.part + (size_t)blockIdx.x * 2 * width;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if constexpr (kPlaces == 1) {
      const int col = (lane + i * kLanes) * kVec;
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        put_sum<T>(a, only, part, width, 0, col + j, dw[i][j]);
        put_sum<T>(a, only, part, width, 1, col + j, db[i][j]);
      }
    } else {
      constexpr int kSpan = kLanes * kVec;   // columns of the i-th groups
      float* at = join + (threadIdx.x / kLanes) * (2 * kSpan) + lane * kVec;
      if (i > 0) __syncthreads();
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        at[j] = dw[i][j];
        at[kSpan + j] = db[i][j];
      }
      __syncthreads();
      for (int k = threadIdx.x; k < 2 * kSpan; k += kGradBlock) {
        const float s = tree_sum<kPlaces>(join + k, 2 * kSpan);
        put_sum<T>(a, only, part, width, k / kSpan, i * kSpan + k % kSpan, s);
      }
    }
  }
}

// Adds `parts` blocks' sums of a column: 32 columns to a block, eight threads of
// four columns by 32 that share the parts.
template <typename T>
__global__ void __launch_bounds__(256) ckm_norm_join_kernel(const float* __restrict__ part, int parts, int cols,
                                                            bool w32, void* dw, void* db) {
  __shared__ float4 lds[32][8];
  const int width = padded_cols(cols);
  const int col = blockIdx.x * 32 + (threadIdx.x & 7) * 4, slot = threadIdx.x >> 3;
  float4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  void* out = blockIdx.y ? db : dw;
  if (!out) return;
  if (col < width)
    for (int p = slot; p < parts; p += 32) {
      const float4 v = *(const float4*)(part + ((size_t)p * 2 + blockIdx.y) * width + col);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  lds[slot][threadIdx.x & 7] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    const float* f = (const float*)&lds[0][0];
    const float t = tree_sum<32>(f + threadIdx.x, 32);
    const int c = blockIdx.x * 32 + threadIdx.x;
    if (c < cols) store_weight<T>(out, w32, c, t);
  }
}

// Rows wider than the registers hold beside the column sums (kWideCols): the row
// sums first, then a pass by columns, each block 2048 columns of a share of rows.
// It reads dy and h twice; rows that fit the registers are faster there (f16
// 4096x16384: 125 us in registers, 149 by columns).
constexpr int kWideCols = 16384;

template <typename T>
__global__ void __launch_bounds__(1024) ckm_norm_wide_sums_kernel(NormGradArgs a, float* sums) {
  __shared__ float lds[4 * 1024 / 64];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
    float s1 = 0.0f, s2 = 0.0f;
    for (int col = threadIdx.x * kVec; col < a.cols; col += 1024 * kVec) {
      const int left = a.cols - col;
      const Raw8<T> rd = load_left((const T*)a.dy + row * a.ld_dy + col, left);
      const Raw8<T> rh = load_left((const T*)a.h + row * a.ld_h + col, left);
      float w[kVec];
      weight_group<T>(w, a.w, a.w32, col, left, 1.0f);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const float g = (float)rd.get(j) * w[j];
        s1 += g;
        s2 += j < left ? g * (((float)rh.get(j) - mean) * rstd) : 0.0f;
      }
    }
    float s[2] = {s1, s2};
    reduce_rows<OpSum, 1024, 1024>(s, lds, turn);
    turn ^= 1;
    if (threadIdx.x == 0) {
      sums[2 * row] = s[0] / (float)a.cols;
      sums[2 * row + 1] = s[1] / (float)a.cols;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) ckm_norm_wide_grad_kernel(NormGradArgs a, const float* __restrict__ sums) {
  const int group = blockIdx.x * 256 + threadIdx.x, col = group * kVec, left = a.cols - col;
  if (left <= 0) return;
  const DropSite site = drop_site(a.drop);
  float w[kVec], dw[kVec] = {}, db[kVec] = {};
  weight_group<T>(w, a.w, a.w32, col, left, 1.0f);
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1], s1 = sums[2 * row], s2 = sums[2 * row + 1];
    const Raw8<T> rd = load_left((const T*)a.dy + row * a.ld_dy + col, left);
    const Raw8<T> rh = load_left((const T*)a.h + row * a.ld_h + col, left);
    Raw8<T> past = zero_group<T>();
    if (a.dres) past = load_left((const T*)a.dres + row * a.ld_dres + col, left);
    float o[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const float d = (float)rd.get(j), xh = ((float)rh.get(j) - mean) * rstd;
      dw[j] = fmaf(d, xh, dw[j]);
      db[j] += d;
      o[j] = rstd * (d * w[j] - s1 - xh * s2) + (float)past.get(j);
    }
    finish_grad<T, false>(a, site, row, group, o);
  }
  if (!a.dw && !a.db) return;
  const int width = padded_cols(a.cols);
  float* part = a.part + (size_t)blockIdx.y * 2 * width;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    put_sum<T>(a, gridDim.y == 1, part, width, 0, col + j, dw[j]);
    put_sum<T>(a, gridDim.y == 1, part, width, 1, col + j, db[j]);
  }
}

// ---------------------------------------------------------------------------
// launch rules
// ---------------------------------------------------------------------------

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename T, int kLanes, int kPer>
void launch_norm_as(const NormArgs& a, bool fused, hipStream_t s) {
  constexpr int kBlock = norm_block(kLanes), kRowsAt = kBlock / kLanes;
  const dim3 grid((uint32_t)std::min<int64_t>(ceil_div(a.rows, kRowsAt), 256 * (2048 / kBlock)));
  const bool even = a.cols % kVec == 0;
  if (fused && even) ckm_norm_kernel<T, kLanes, kPer, true, true><<<grid, kBlock, 0, s>>>(a);
  else if (fused) ckm_norm_kernel<T, kLanes, kPer, true, false><<<grid, kBlock, 0, s>>>(a);
  else if (even) ckm_norm_kernel<T, kLanes, kPer, false, true><<<grid, kBlock, 0, s>>>(a);
  else ckm_norm_kernel<T, kLanes, kPer, false, false><<<grid, kBlock, 0, s>>>(a);
}

// Threads and groups a thread: two groups where a row has that many beyond 64
// threads. Measured at bf16 8192x8192 fused: 512 threads of two 100 us, 1024 of one
// 101, 256 of four (whose weights do not stay in registers) 107; 8192x4096 fused: 256
// of two 54.1, 512 of one 54.5, 128 of four 55.6.
template <typename T>
void launch_norm(const NormArgs& a, bool fused, hipStream_t s) {
  const int groups = padded_cols(a.cols) / kVec;
  if (groups <= 16) launch_norm_as<T, 16, 1>(a, fused, s);
  else if (groups <= 32) launch_norm_as<T, 16, 2>(a, fused, s);
  else if (groups <= 64) launch_norm_as<T, 32, 2>(a, fused, s);
  else if (groups <= 128) launch_norm_as<T, 64, 2>(a, fused, s);
  else if (groups <= 256) launch_norm_as<T, 256, 1>(a, fused, s);
  else if (groups <= 512) launch_norm_as<T, 256, 2>(a, fused, s);
  else if (groups <= 1024) launch_norm_as<T, 512, 2>(a, fused, s);
  else if (groups <= 2048) launch_norm_as<T, 1024, 2>(a, fused, s);
  else launch_norm_as<T, 1024, 4>(a, fused, s);
}

// Blocks of the gradient for `rows` rows: their number fixes the order of the
// sums, so it depends on the sizes alone. 256 blocks of 1024 threads: blocks of 512,
// twice as many, write twice the sums (f16 2048x2048 17.4 us, 13.7 so; bf16 16384x4096
// 140 and 132). One group a thread up to 8192 columns, over as many threads as a row
// needs: two groups on half the threads leave no registers (f16 16384x1024 fused 48
// us, 43 so), and two rows at a time neither (bf16 16384x4096 159 us, 130 so). Rows that four
// blocks take in one turn (two, with two groups a thread) are one block's, in as many
// turns, which has no sums to join: a call on f16 256x128 10.6 us, 15.2 in four blocks;
// 64x512 10.7, 15.3; 16x2048 10.7, 15.3; 4x8192 12.4, 15.9 (f32 14.7, 15.3); 2x16384 17.9,
// 23.3 (f32 26.3, 24.9); 4x16384 25.9, 23.3 (f32 34.9, 24.9). That is the host's second
// launch: in a graph the joined blocks are faster from three turns on (16x2048 6.6 us,
// 9.9 in one block; of two turns, 8x2048 6.6, 6.3). f16 32x2048 as calls 17.3, 15.5 in
// eight blocks.
struct GradPlan {
  int lanes, per;       // 0, 0: by columns
  int64_t blocks;       // sets of column sums
};
GradPlan grad_plan(int64_t rows, int64_t cols) {
  const int groups = padded_cols((int)cols) / kVec;
  GradPlan p;
  if (cols > kWideCols) {
    p.lanes = p.per = 0;
    p.blocks = std::max<int64_t>(1, std::min<int64_t>(rows, 256));
    return p;
  }
  int lanes = 16;
  while (lanes < 1024 && lanes < groups) lanes *= 2;
  p.lanes = lanes;
  p.per = groups <= 1024 ? 1 : 2;
  p.blocks = std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, kGradBlock / lanes), 256));
  if (p.blocks <= (p.per == 1 ? 4 : 2)) p.blocks = 1;
  return p;
}

size_t grad_workspace(int64_t rows, int64_t cols) {
  const GradPlan p = grad_plan(rows, cols);
  size_t bytes = p.blocks > 1 ? (size_t)p.blocks * 2 * padded_cols((int)cols) * sizeof(float) : 0;
  if (p.lanes == 0) bytes += (size_t)rows * 2 * sizeof(float);
  return bytes;
}

template <typename T, int kLanes, int kPer>
void launch_grad_as(const NormGradArgs& a, int64_t blocks, hipStream_t s) {
  const dim3 grid((uint32_t)blocks);
  if (a.cols % kVec == 0)
    ckm_norm_grad_kernel<T, kLanes, kPer, true><<<grid, kGradBlock, 0, s>>>(a);
  else
    ckm_norm_grad_kernel<T, kLanes, kPer, false><<<grid, kGradBlock, 0, s>>>(a);
}

template <typename T>
void launch_grad(NormGradArgs a, void* work, hipStream_t s) {
  const GradPlan p = grad_plan(a.rows, a.cols);
  a.part = (float*)work;
  if (p.lanes == 0) {
    float* sums = (float*)work + (p.blocks > 1 ? (size_t)p.blocks * 2 * padded_cols(a.cols) : 0);
    if (a.rows > 0)
      ckm_norm_wide_sums_kernel<T><<<dim3((uint32_t)std::min<int64_t>(a.rows, 2048)), 1024, 0, s>>>(a, sums);
    ckm_norm_wide_grad_kernel<T><<<dim3((uint32_t)ceil_div(a.cols, 256 * kVec), (uint32_t)p.blocks), 256, 0, s>>>(a, sums);
  } else {
    switch (p.lanes) {
      case 16: launch_grad_as<T, 16, 1>(a, p.blocks, s); break;
      case 32: launch_grad_as<T, 32, 1>(a, p.blocks, s); break;
      case 64: launch_grad_as<T, 64, 1>(a, p.blocks, s); break;
      case 128: launch_grad_as<T, 128, 1>(a, p.blocks, s); break;
      case 256: launch_grad_as<T, 256, 1>(a, p.blocks, s); break;
      case 512: launch_grad_as<T, 512, 1>(a, p.blocks, s); break;
      default:
        if (p.per == 1)
          launch_grad_as<T, 1024, 1>(a, p.blocks, s);
        else
          launch_grad_as<T, 1024, 2>(a, p.blocks, s);
    }
  }
  if (p.blocks > 1 && (a.dw || a.db))
    ckm_norm_join_kernel<T><<<dim3((uint32_t)ceil_div(a.cols, 32), 2), 256, 0, s>>>(a.part, (int)p.blocks, a.cols, a.w32,
                                                                                   a.dw, a.db);
}

ckm_status check_norm(int type, int wtype, int64_t rows, int64_t cols) {
  if (!dtype_ok(type)) return set_error(CKM_E_INVALID_ARG, "unknown type %d", type);
  if (wtype != type && wtype != CKM_F32)
    return set_error(CKM_E_INVALID_ARG, "weight type %d: weights are of the tensors' type %d or CKM_F32", wtype, type);
  if (rows < 0 || cols < 1)
    return set_error(CKM_E_INVALID_ARG, "rows = %lld, cols = %lld", (long long)rows, (long long)cols);
  if (rows > CKM_MAX_ROWS || cols > CKM_MAX_NORM_COLS)
    return set_error(CKM_E_UNSUPPORTED, "rows = %lld, cols = %lld (at most %d columns)", (long long)rows,
                     (long long)cols, CKM_MAX_NORM_COLS);
  return CKM_OK;
}

ckm_status check_aligned(const void* p, const char* name, size_t elt) {
  if ((uintptr_t)p % elt) return set_error(CKM_E_INVALID_ARG, "%s is not aligned to its %zu-byte elements", name, elt);
  return CKM_OK;
}

}  // namespace
}  // namespace ckm

extern "C" ckm_status ckm_layer_norm_async(ckm_dtype type, ckm_dtype wtype, int64_t rows, int64_t cols,
                                           const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual,
                                           const ckm_drop* drop, const void* d_weight, const void* d_bias, float eps,
                                           void* d_h, int64_t ld_h, void* d_y, int64_t ld_y, float* d_stats,
                                           void* stream) {
  using namespace ckm;
  ckm_status st = check_norm(type, wtype, rows, cols);
  if (st != CKM_OK) return st;
  if (!(eps >= 0.0f) || eps > 3.4e38f) return set_error(CKM_E_INVALID_ARG, "eps = %g", (double)eps);
  NormArgs a;
  if ((st = drop_args(drop, &a.drop)) != CKM_OK) return st;
  const bool fused = drop || d_residual;
  if (d_h && !fused) return set_error(CKM_E_INVALID_ARG, "h given without a dropout or a residual: h is x");
  const size_t elt = dtype_bytes(type), welt = dtype_bytes(wtype);
  if ((st = check_aligned(d_weight, "weight", welt)) != CKM_OK) return st;
  if ((st = check_aligned(d_bias, "bias", welt)) != CKM_OK) return st;
  if ((st = check_aligned(d_stats, "stats", 4)) != CKM_OK) return st;
  if (rows == 0) return CKM_OK;
  if ((st = check_matrix(d_x, "x", rows, cols, ld_x, elt, false)) != CKM_OK) return st;
  if (d_residual && (st = check_matrix(d_residual, "residual", rows, cols, ld_residual, elt, false)) != CKM_OK) return st;
  if (d_h && (st = check_matrix(d_h, "h", rows, cols, ld_h, elt, true)) != CKM_OK) return st;
  if ((st = check_matrix(d_y, "y", rows, cols, ld_y, elt, true)) != CKM_OK) return st;
  a.rows = (int32_t)rows;
  a.cols = (int32_t)cols;
  a.x = d_x;
  a.ld_x = ld_x;
  a.res = d_residual;
  a.ld_res = ld_residual;
  a.w = d_weight;
  a.b = d_bias;
  a.w32 = wtype == CKM_F32;
  a.eps = eps;
  a.h = d_h;
  a.ld_h = ld_h;
  a.y = d_y;
  a.ld_y = ld_y;
  a.stats = d_stats;
  const hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case CKM_F32: launch_norm<float>(a, fused, s); break;
    case CKM_F16: launch_norm<_Float16>(a, fused, s); break;
    default: launch_norm<__bf16>(a, fused, s); break;
  }
  return launched("layer norm launch");
}

extern "C" ckm_status ckm_layer_norm_workspace_size(int64_t rows, int64_t cols, size_t* bytes) {
  using namespace ckm;
  if (!bytes) return set_error(CKM_E_INVALID_ARG, "bytes is NULL");
  const ckm_status st = check_norm(CKM_F32, CKM_F32, rows, cols);
  if (st != CKM_OK) return st;
  *bytes = grad_workspace(rows, cols);
  return CKM_OK;
}

extern "C" ckm_status ckm_layer_norm_backward_async(ckm_dtype type, ckm_dtype wtype, int64_t rows, int64_t cols,
                                                    const void* d_dy, int64_t ld_dy, const void* d_h, int64_t ld_h,
                                                    const float* d_stats, const void* d_weight, const void* d_dres,
                                                    int64_t ld_dres, const ckm_drop* drop, void* d_dh, int64_t ld_dh,
                                                    void* d_dx, int64_t ld_dx, void* d_dweight, void* d_dbias,
                                                    void* d_work, size_t work_bytes, void* stream) {
  using namespace ckm;
  ckm_status st = check_norm(type, wtype, rows, cols);
  if (st != CKM_OK) return st;
  NormGradArgs a;
  if ((st = drop_args(drop, &a.drop)) != CKM_OK) return st;
  if (d_dx && !drop) return set_error(CKM_E_INVALID_ARG, "dx given without a dropout: dx is dh");
  const size_t elt = dtype_bytes(type), welt = dtype_bytes(wtype);
  if ((st = check_aligned(d_weight, "weight", welt)) != CKM_OK) return st;
  if ((st = check_aligned(d_dweight, "dweight", welt)) != CKM_OK) return st;
  if ((st = check_aligned(d_dbias, "dbias", welt)) != CKM_OK) return st;
  if (rows > 0) {
    if (!d_stats) return set_error(CKM_E_INVALID_ARG, "stats is NULL");
    if ((st = check_aligned(d_stats, "stats", 4)) != CKM_OK) return st;
    if ((st = check_matrix(d_dy, "dy", rows, cols, ld_dy, elt, false)) != CKM_OK) return st;
    if ((st = check_matrix(d_h, "h", rows, cols, ld_h, elt, false)) != CKM_OK) return st;
    if (d_dres && (st = check_matrix(d_dres, "dres", rows, cols, ld_dres, elt, false)) != CKM_OK) return st;
    if (d_dh && (st = check_matrix(d_dh, "dh", rows, cols, ld_dh, elt, true)) != CKM_OK) return st;
    if (d_dx && (st = check_matrix(d_dx, "dx", rows, cols, ld_dx, elt, true)) != CKM_OK) return st;
  }
  const size_t need = grad_workspace(rows, cols);
  if (need > 0 && (!d_work || work_bytes < need))
    return set_error(CKM_E_INVALID_ARG, "work buffer of %zu bytes, %zu needed", d_work ? work_bytes : (size_t)0, need);
  if ((uintptr_t)d_work % 16) return set_error(CKM_E_INVALID_ARG, "work is not aligned to 16 bytes");
  a.rows = (int32_t)rows;
  a.cols = (int32_t)cols;
  a.dy = d_dy;
  a.ld_dy = ld_dy;
  a.h = d_h;
  a.ld_h = ld_h;
  a.stats = d_stats;
  a.w = d_weight;
  a.w32 = wtype == CKM_F32;
  a.dres = d_dres;
  a.ld_dres = ld_dres;
  a.dh = d_dh;
  a.ld_dh = ld_dh;
  a.dx = d_dx;
  a.ld_dx = ld_dx;
  a.dw = d_dweight;
  a.db = d_dbias;
  a.part = nullptr;
  const hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case CKM_F32: launch_grad<float>(a, d_work, s); break;
    case CKM_F16: launch_grad<_Float16>(a, d_work, s); break;
    default: launch_grad<__bf16>(a, d_work, s); break;
  }
  return launched("layer norm gradient launch");
}
