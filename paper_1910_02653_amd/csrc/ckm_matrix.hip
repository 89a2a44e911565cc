// What the operators' products share: how they are cut into tiles and shares of k,
// copies of operands that cannot be loaded straight to LDS, and the sums of shares.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "ckm_matrix.h"

namespace ckm {
namespace {

constexpr int kBlock = 256;

// A thread a group of eight columns of the copy.
template <typename T>
__global__ void __launch_bounds__(kBlock) ckm_pack_kernel(int64_t total, uint32_t groups, int32_t cols, const T* src,
                                                          int64_t ld_src, T* dst, int64_t ld,
                                                          const int64_t* targets, int64_t vocab) {
  for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock) {
    const int64_t row = at / groups;
    const int col = (int)(at - row * groups) * kVec;
    Raw8<T> r = zero_group<T>();
    const bool live = !targets || (targets[row] >= 0 && targets[row] < vocab);
    if (live && col < cols) r = load_left(src + row * ld_src + col, cols - col);
    store_part<false>(dst + row * ld, r, col, (int)ld);
  }
}

template <typename T>
void pack(const void* src, int64_t rows, int64_t cols, int64_t ld_src, void* dst, int64_t ld, hipStream_t s,
          const int64_t* targets, int64_t vocab) {
  const uint32_t groups = (uint32_t)((ld + kVec - 1) / kVec);
  const int64_t total = rows * groups;
  if (total == 0) return;
  ckm_pack_kernel<T><<<(uint32_t)std::min<int64_t>((total + kBlock - 1) / kBlock, 1 << 16), kBlock, 0, s>>>(
      total, groups, (int32_t)cols, (const T*)src, ld_src, (T*)dst, ld, targets, vocab);
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

Cut cut_product(int64_t m, int64_t n, int halves, int64_t steps, int) {
  const auto tiles = [&](int64_t t) { return ((m + t - 1) / t) * ((n + t - 1) / t) * halves; };
  Cut c = {};
  c.rows = c.cols = tiles(256) >= 192 ? 256 : 128;
  c.halves = halves;
  c.tiles_m = (int)((m + c.rows - 1) / c.rows);
  c.tiles_n = (int)((n + c.cols - 1) / c.cols);
  const int64_t blocks = tiles(c.rows);
  int64_t splits = std::max<int64_t>(1, std::min<int64_t>(512 / blocks, steps / 8));
  c.steps = (int)((steps + splits - 1) / splits);
  c.splits = (int)((steps + c.steps - 1) / c.steps);
  return c;
}

ckm_status check_blocks(const Cut& c) {
  return c.blocks() <= INT32_MAX ? CKM_OK
                                 : set_error(CKM_E_UNSUPPORTED, "a product of %lld tiles", (long long)c.blocks());
}

void launch_pack(int type, const void* src, int64_t rows, int64_t cols, int64_t ld_src, void* dst, int64_t ld,
                 hipStream_t s, const int64_t* targets, int64_t vocab) {
  switch (type) {
    case CKM_F32: pack<float>(src, rows, cols, ld_src, dst, ld, s, targets, vocab); break;
    case CKM_F16: pack<_Float16>(src, rows, cols, ld_src, dst, ld, s, targets, vocab); break;
    default: pack<__bf16>(src, rows, cols, ld_src, dst, ld, s, targets, vocab); break;
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
