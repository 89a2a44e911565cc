// What the operators' products share: how they are cut into tiles and shares of k,
// copies of operands that cannot be loaded straight to LDS, and the sums of shares.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ckm_matrix.h"

namespace ckm {
namespace {

constexpr int kBlock = 256;

// A thread a group of eight columns of a copy; each copy has blocks of its own.
template <typename T>
__global__ void __launch_bounds__(kBlock) ckm_pack_kernel(PackArgs a) {
  uint32_t block = blockIdx.x;
  if (a.most && block == gridDim.x - 1) {
    __shared__ float lds[2 * kBlock / 64];
    float most = 0.0f;
    constexpr int kAtOnce = 8;   // rows of a thread whose loads are in flight together; the last row may be taken again
    for (int64_t first = threadIdx.x; first < a.rows; first += kAtOnce * kBlock) {
      float v[kAtOnce];
      int64_t target[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int64_t r = min(first + j * kBlock, a.rows - 1);
        v[j] = fabsf(a.dloss[r]);
        target[j] = a.targets[r];
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (target[j] >= 0 && target[j] < a.vocab && v[j] < INFINITY) most = fmaxf(most, v[j]);
    }
    most = reduce_row<OpMax, kBlock, kBlock>(most, lds, 0);
    if (threadIdx.x == 0) *a.most = most > 0.0f ? most : 1.0f;
    return;
  }
  PackArgs::One p = a.one[0];
  if (block >= p.blocks) {
    block -= p.blocks;
    p = a.one[1];
    if (block >= p.blocks) {
      block -= p.blocks;
      p = a.one[2];
    }
  }
  for (int64_t at = (int64_t)block * kBlock + threadIdx.x; at < p.total; at += (int64_t)p.blocks * kBlock) {
    const int64_t row = at / p.groups;
    const int col = (int)(at - row * p.groups) * kVec;
    Raw8<T> r = zero_group<T>();
    const bool live = !a.targets || (a.targets[row] >= 0 && a.targets[row] < a.vocab);
    if (live && col < p.cols) r = load_left((const T*)p.src + row * p.ld_src + col, p.cols - col);
    store_part<false>((T*)p.dst + row * p.ld, r, col, (int)p.ld);
  }
}

template <typename T>
__global__ void __launch_bounds__(kBlock) ckm_zero_kernel(int64_t total, int64_t cols, T* dst, int64_t ld) {
  for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock)
    dst[at / cols * ld + at % cols] = (T)0;
}

// A thread four columns of a row.
template <typename T>
__global__ void __launch_bounds__(kBlock) ckm_join_kernel(ResultArgs a, int splits, int64_t total, uint32_t fours) {
  const float factor = a.alpha ? a.factor * *a.alpha : a.factor;
  const int64_t one = (int64_t)a.p.m * a.ld_slab;
  for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock) {
    const int64_t line = at / fours;
    const int half = line >= a.p.m, col = (int)(at - line * fours) * 4;
    const int64_t row = line - (half ? a.p.m : 0);
    const float* p = a.slab + half * one + row * a.ld_slab + col;
    F4 sum = *(const F4*)p;
#pragma unroll 8
    for (int k = 1; k < splits; ++k) sum += *(const F4*)(p + k * a.halves * one);
    store4((T*)(half ? a.c[1] : a.c[0]) + row * (half ? a.ld_c[1] : a.ld_c[0]), col, a.p.n, sum * factor);
  }
}

template <typename T>
void join(const ResultArgs& a, int splits, hipStream_t s) {
  const uint32_t fours = (uint32_t)((a.p.n + 3) / 4);
  const int64_t total = (int64_t)a.p.m * a.halves * fours;
  ckm_join_kernel<T><<<(uint32_t)std::min<int64_t>((total + kBlock - 1) / kBlock, 1 << 16), kBlock, 0, s>>>(a, splits,
                                                                                                         total, fours);
}

}  // namespace

// What the model of a product's time goes by (cut_product), in us.
struct Time {
  double one, more;   // a step where a CU has one tile, or several
};
struct Shape {
  int rows, cols;
  Time half, full;    // 16-bit types, binary32
  double fixed;
  const Time& step(int type) const { return type == CKM_F32 ? full : half; }
};
// Largest first.
constexpr Shape kShapes[] = {{256, 256, {1.5, 1.5}, {8.1, 8.1}, 7.0},
                             {128, 128, {0.68, 0.51}, {2.05, 1.95}, 4.0},
                             {64, 128, {0.38, 0.33}, {1.15, 1.03}, 2.5},
                             {16, 128, {0.30, 0.225}, {0.50, 0.38}, 2.5}};
constexpr double kCUs = 256.0, kBytesAUs = 5.0e6, kJoin = 4.0, kLaunch = 4.0;
constexpr double kSharesAUs = 6.5e6;   // bytes of shares, which the caches hold in part

// The first values of a cut: its tiles and shares.
Cut cut_as(const Shape& shape, int64_t m, int64_t n, int halves, int subs, int64_t steps, int splits, bool staged) {
  Cut c = {};
  c.rows = shape.rows;
  c.cols = shape.cols / subs;
  c.tiles_m = (int)((m + c.rows - 1) / c.rows);
  c.tiles_n = (int)((n + c.cols - 1) / c.cols);
  c.halves = halves;
  c.steps = (int)((steps + splits - 1) / splits);
  c.splits = (int)((steps + c.steps - 1) / c.steps);
  c.staged = staged;
  return c;
}
// The shares' way through memory: written and read. In binary32's products of two matrices,
// whose steps are the longest, the other tiles of a CU hide the writing where it has several:
// where that changes the cut, 65 sizes drawn over the operator's range, calls take 0.998 of
// the time in the mean, 0.86 to 1.15 (777x1023x2731: 108 us in two shares, 117 in one). It
// does not hold in 16 bits (71 sizes: 1.04, up to 1.28) or for the loss's gradient in
// binary32 (39 sizes: 1.004).
double join_time(int type, const Cut& c, int64_t m, int64_t n, int subs) {
  const double bytes = type == CKM_F32 && subs == 2 && c.rows < 256 && c.blocks() > 2 * kCUs ? 4.0 : 8.0;
  return c.splits > 1 ? kJoin + bytes * c.splits * m * n * c.halves * subs / kSharesAUs : 0.0;
}

// The cheapest cut by a model of the time: a CU takes one tile after the other, each as
// many steps of k at the shape's measured time (longer where a CU has one tile and so
// half its waves) and a fixed part (start, first loads, stores); no less than the
// operands take from memory; shares are written and read once more. The steps' times
// are those of these products (us; rows of a tile, tiles of a CU):
//   bf16 2048x2048x4096   128 rows, one: 45, two shares 33; 64, two: 42; 16, eight: 113
//   f32 2048x2048x1024    128 rows, one: 75; 64, two: 71; 16, eight: 97
//   bf16 2048x8192x4096   256 rows, one: 101 (1357 TFLOP/s); 128, four: 128; 64, eight: 161
//   bf16 1x16384x2048     16 rows 12, 64 rows 15 (67 MB)
double time_of(int type, const Shape& shape, const Cut& c, int64_t m, int64_t n, int subs, int64_t bytes, Staged staged) {
  constexpr double kSteps[] = {1.0, 1.4, 2.5}, kReads[] = {1.0, 1.2, 5.0};   // by way of registers, of lines that are cut
  const double rounds = std::ceil(c.blocks() / kCUs);
  const Time& time = shape.step(type);
  const double step = (rounds > 1.0 ? time.more : time.one) * kSteps[staged];
  // where a CU holds two tiles, one's fixed part is half hidden behind the other's steps
  const double fixed = shape.fixed * (shape.rows == 256 ? rounds : 1.0 + 0.5 * (rounds - 1.0));
  return std::max(rounds * c.steps * step + fixed, kReads[staged] * bytes / kBytesAUs + shape.fixed) +
         join_time(type, c, m, n, subs);
}

Cut cut_product(int type, int64_t m, int64_t n, int halves, int subs, int64_t steps, int64_t bytes, bool split,
                bool a_along_k) {
  Cut best = {};
  for (const Shape& shape : kShapes) {
    if (shape.rows < 64 && !a_along_k) continue;
    for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256}) {
      Cut c = cut_as(shape, m, n, halves, subs, steps, splits, false);
      if (splits > 1 && (!split || steps / splits < 4 || c.blocks() > 2048)) break;
      c.time = time_of(type, shape, c, m, n, subs, bytes, kStraight);
      if (!best.rows || c.time <= best.time) best = c;
    }
  }
  return best;
}

Cut cut_like(int type, int64_t m, int64_t n, int halves, int subs, int64_t steps, int64_t bytes, bool a_along_k,
             Staged staged, const Cut& as) {
  Cut best = {};
  for (const Shape& shape : kShapes) {
    if ((shape.rows < 64 && !a_along_k) || (shape.rows == 256 && staged)) continue;
    Cut c = cut_as(shape, m, n, halves, subs, steps, as.splits, staged != kStraight);
    c.time = time_of(type, shape, c, m, n, subs, bytes, staged);
    if (!best.rows || c.time <= best.time) best = c;
  }
  return best;
}

bool cut_together(int type, Cut& a, int64_t m_a, int64_t n_a, int64_t steps_a, Cut& b, int64_t m_b, int64_t n_b,
                  int64_t steps_b, int64_t bytes) {
  // long products have the larger tiles' rate to lose, and little to gain (f16
  // 2048x2048x8192, gated gradient: 404 us apart, 448 together)
  constexpr double kLong = 60.0, kGain = 0.92;
  if (a.time + b.time > kLong) return false;
  const Shape& shape_b = kShapes[1];
  Cut d = cut_as(shape_b, m_b, n_b, b.halves, 1, steps_b, 1, false);
  const Time& time_b = shape_b.step(type);
  double least = kGain * (a.time + b.time + kLaunch);
  bool found = false;
  Cut best = {};
  for (int k = 1; k <= 2; ++k) {
    const Shape& shape = kShapes[k];
    const Time& time = shape.step(type);
    for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
      const Cut c = cut_as(shape, m_a, n_a, 1, 1, steps_a, splits, false);
      if (splits > 1 && (steps_a / splits < 4 || c.blocks() > 2048)) break;
      // all the work shared out evenly, no less than the longest tile
      const double work = (c.blocks() * (c.steps * time.more + shape.fixed) + d.blocks() * (d.steps * time_b.more + shape_b.fixed)) / kCUs;
      const double longest = std::max(c.steps * time.one + shape.fixed, d.steps * time_b.one + shape_b.fixed);
      const double t = std::max({work, longest, bytes / kBytesAUs + shape.fixed}) + join_time(type, c, m_a, n_a, 1);
      if (t < least) {
        least = t;
        best = c;
        found = true;
      }
    }
  }
  if (!found) return false;
  a = best;
  a.time = least;
  b = d;
  b.time = 0.0;
  return true;
}

static bool share(const Place& a, const Place& b) {
  if (!a.p || !b.p || !a.rows || !b.rows || !a.cols || !b.cols) return false;
  const __int128 pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
  const __int128 ca = (__int128)a.cols * a.elt, cb = (__int128)b.cols * b.elt, ra = (__int128)a.ld * a.elt, rb = (__int128)b.ld * b.elt;
  if (pa + (a.rows - 1) * ra + ca <= pb || pb + (b.rows - 1) * rb + cb <= pa) return false;
  if (a.rows == 1 || b.rows == 1 || ra != rb || ra < ca || ra < cb) return true;
  // rows of one stride: from a's columns to b's, around the stride
  const __int128 by = ((pb - pa) % ra + ra) % ra;
  return by < ca || by + cb > ra;
}

ckm_status check_apart(std::initializer_list<Place> outputs, std::initializer_list<Place> inputs) {
  for (const Place* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Place& i : inputs)
      if (share(*o, i)) return set_error(CKM_E_INVALID_ARG, "%s overlaps %s", o->name, i.name);
    for (const Place* q = o + 1; q != outputs.end(); ++q)
      if (share(*o, *q)) return set_error(CKM_E_INVALID_ARG, "%s overlaps %s", o->name, q->name);
  }
  return CKM_OK;
}

ckm_status check_blocks(const Cut& c) {
  constexpr int64_t kMost = ((int64_t)1 << 32) / 512 - 1;   // a launch's threads are counted in 32 bits
  return c.blocks() <= kMost ? CKM_OK : set_error(CKM_E_UNSUPPORTED, "a product of %lld tiles", (long long)c.blocks());
}

void PackArgs::add(const void* src, int64_t rows, int64_t cols, int64_t ld_src, void* dst, int64_t ld) {
  const uint32_t groups = (uint32_t)((ld + kVec - 1) / kVec);
  const int64_t total = rows * groups;
  one[count++] = {src, dst, total, ld_src, ld, groups, (int32_t)cols,
                  (uint32_t)std::min<int64_t>((total + kBlock - 1) / kBlock, 1 << 16)};
}

void launch_pack(int type, const PackArgs& a, hipStream_t s) {
  const uint32_t blocks = a.one[0].blocks + a.one[1].blocks + a.one[2].blocks + (a.most ? 1 : 0);
  if (blocks == 0) return;
  switch (type) {
    case CKM_F32: ckm_pack_kernel<float><<<blocks, kBlock, 0, s>>>(a); break;
    case CKM_F16: ckm_pack_kernel<_Float16><<<blocks, kBlock, 0, s>>>(a); break;
    default: ckm_pack_kernel<__bf16><<<blocks, kBlock, 0, s>>>(a); break;
  }
}

void launch_zero(int type, void* dst, int64_t rows, int64_t cols, int64_t ld, hipStream_t s) {
  const int64_t total = rows * cols;
  const uint32_t grid = (uint32_t)std::min<int64_t>((total + kBlock - 1) / kBlock, 1 << 16);
  if (total == 0) return;
  if (type == CKM_F32) ckm_zero_kernel<<<grid, kBlock, 0, s>>>(total, cols, (float*)dst, ld);
  else ckm_zero_kernel<<<grid, kBlock, 0, s>>>(total, cols, (uint16_t*)dst, ld);
}

void launch_join(int type, const ResultArgs& a, int splits, hipStream_t s) {
  switch (type) {
    case CKM_F32: join<float>(a, splits, s); break;
    case CKM_F16: join<_Float16>(a, splits, s); break;
    default: join<__bf16>(a, splits, s); break;
  }
}

}  // namespace ckm
