// Dropout from the counter-based generator, with an optional residual sum:
// y = r + D(x), D(x) = x 65536 / keep where the element's draw is below keep,
// else 0. Its gradient is the same map of dy, so one kernel serves both, and
// the mask exists only in registers.
//
// Bound by memory: each element is read once and written once, and the draws,
// about 50 instructions for eight elements, hide behind that. A thread takes one
// group of eight; two and four groups a thread, their loads first, were slower at
// every size (bf16 16384x8192: 91, 96, 100 us; f16 4096x4096 with a residual
// 17, 20, 20). bf16 16384x8192 moves 5.9 TB/s, where a large copy moves 5.2.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "ckm_ops.h"

namespace ckm {
namespace {

constexpr int kDropBlock = 256;

// Groups are numbered row by row, `groups` to a row. A block takes 256
// consecutive ones at a time; the division by `groups` is made once for the
// block's first group, and a thread's place follows from it without one: with
// magic = floor(2^32 / groups) + 1, q = hi(at * magic) is exact for at * groups
// < 2^32 and groups > 1; where a row holds 512 groups or more, a block crosses one
// row border at most (magic 0). kFlat: rows of whole groups without gaps, so that
// a group's number is its address and the loads need not wait for its place.
template <typename T, bool kRes, bool kFlat>
__global__ void __launch_bounds__(kDropBlock) ckm_dropout_kernel(int64_t total, uint32_t groups, uint32_t magic,
                                                                 int32_t cols, const T* x, int64_t ld_x, const T* res,
                                                                 int64_t ld_res, DropArgs drop, T* y, int64_t ld_y) {
  const DropSite site = drop_site(drop);
  for (int64_t base = (int64_t)blockIdx.x * kDropBlock; base < total; base += (int64_t)gridDim.x * kDropBlock) {
    const int64_t g = base + threadIdx.x;
    const int64_t row0 = base / groups;
    const uint32_t at = (uint32_t)(base - row0 * groups) + threadIdx.x;
    const uint32_t q = groups == 1 ? at : magic ? __umulhi(at, magic) : (at >= groups ? 1u : 0u);
    const uint32_t group = at - q * groups;
    const int64_t row = row0 + q;
    if (g >= total) continue;
    const int col = (int)(group * kVec);
    Raw8<T> vx, vr;
    if constexpr (kFlat) {
      vx = load8(x + g * kVec);
      if constexpr (kRes) vr = load8(res + g * kVec);
    } else {
      vx = load_cols<false>(x + row * ld_x, col, cols);
      if constexpr (kRes) vr = load_cols<false>(res + row * ld_res, col, cols);
    }
    fix_tail<kFlat>(vx, col, cols);
    if (drop.on) drop_choice(vx, drop, site, group, (uint32_t)row);
    float v[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = (float)vx.get(j) * drop.scale;
    if constexpr (kRes) {
      fix_tail<kFlat>(vr, col, cols);
#pragma unroll
      for (int j = 0; j < kVec; ++j) v[j] += (float)vr.get(j);
    }
    if constexpr (kFlat)
      store_part<true>(y + g * kVec, rounded8<T>(v), 0, kVec);
    else
      store_part<false>(y + row * ld_y, rounded8<T>(v), col, cols);
  }
}

template <typename T>
void launch_dropout(int64_t rows, int64_t cols, const void* x, int64_t ld_x, const void* res, int64_t ld_res,
                    const DropArgs& drop, void* y, int64_t ld_y, hipStream_t stream) {
  const uint32_t groups = (uint32_t)((cols + kVec - 1) / kVec);
  const int64_t total = rows * groups;
  const uint32_t magic = groups == 1 || groups >= 2 * kDropBlock ? 0u : (uint32_t)((((uint64_t)1 << 32) / groups) + 1);
  const dim3 grid((uint32_t)std::min<int64_t>((total + kDropBlock - 1) / kDropBlock, 1 << 20));
  const auto go = [&](auto with_res, auto flat) {
    ckm_dropout_kernel<T, decltype(with_res)::value, decltype(flat)::value><<<grid, kDropBlock, 0, stream>>>(
        total, groups, magic, (int32_t)cols, (const T*)x, ld_x, (const T*)res, ld_res, drop, (T*)y, ld_y);
  };
  const bool flat =
      cols % kVec == 0 && (rows == 1 || (ld_x == cols && ld_y == cols && (!res || ld_res == cols)));
  if (res && flat) go(std::true_type{}, std::true_type{});
  else if (res) go(std::true_type{}, std::false_type{});
  else if (flat) go(std::false_type{}, std::true_type{});
  else go(std::false_type{}, std::false_type{});
}

}  // namespace

ckm_status drop_args(const ckm_drop* d, DropArgs* out) {
  *out = DropArgs();
  if (!d) return CKM_OK;
  if (d->keep > 65536u) return set_error(CKM_E_INVALID_ARG, "drop: keep = %u > 65536", d->keep);
  if ((uintptr_t)d->d_site % 8) return set_error(CKM_E_INVALID_ARG, "drop: d_site is not aligned to 8 bytes");
  out->k0 = (uint32_t)d->seed;
  out->k1 = (uint32_t)(d->seed >> 32);
  out->site = d->site;
  out->d_site = d->d_site;
  out->keep = d->keep;
  out->scale = d->keep ? 65536.0f / (float)d->keep : 0.0f;
  out->on = d->keep < 65536u;
  return CKM_OK;
}

ckm_status check_matrix(const void* p, const char* name, int64_t rows, int64_t cols, int64_t ld, size_t elt,
                        bool output) {
  if (!p) return set_error(CKM_E_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)p % elt) return set_error(CKM_E_INVALID_ARG, "%s is not aligned to its %zu-byte elements", name, elt);
  if (ld < 0 || (output && rows > 1 && ld < cols))
    return set_error(CKM_E_INVALID_ARG, "%s: row stride %lld for rows of %lld", name, (long long)ld, (long long)cols);
  if (rows > 1 && ld > (INT64_MAX / 8 - cols) / (rows - 1))
    return set_error(CKM_E_INVALID_ARG, "%s: row stride %lld passes the address range", name, (long long)ld);
  return CKM_OK;
}

ckm_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CKM_OK : set_error(CKM_E_DEVICE, "%s: %s (%d)", what, hipGetErrorString(e), (int)e);
}

}  // namespace ckm

extern "C" ckm_status ckm_dropout_async(ckm_dtype type, int64_t rows, int64_t cols, const void* d_x, int64_t ld_x,
                                        const void* d_residual, int64_t ld_residual, const ckm_drop* drop, void* d_y,
                                        int64_t ld_y, void* stream) {
  using namespace ckm;
  if (!dtype_ok(type)) return set_error(CKM_E_INVALID_ARG, "unknown type %d", (int)type);
  if (rows < 0 || cols < 0) return set_error(CKM_E_INVALID_ARG, "rows = %lld, cols = %lld", (long long)rows, (long long)cols);
  if (rows > CKM_MAX_ROWS || cols > CKM_MAX_COLS)
    return set_error(CKM_E_UNSUPPORTED, "rows = %lld, cols = %lld", (long long)rows, (long long)cols);
  if (!drop) return set_error(CKM_E_INVALID_ARG, "drop is NULL");
  DropArgs args;
  ckm_status st = drop_args(drop, &args);
  if (st != CKM_OK) return st;
  if (rows == 0 || cols == 0) return CKM_OK;
  const size_t elt = dtype_bytes(type);
  if ((st = check_matrix(d_x, "x", rows, cols, ld_x, elt, false)) != CKM_OK) return st;
  if (d_residual && (st = check_matrix(d_residual, "residual", rows, cols, ld_residual, elt, false)) != CKM_OK) return st;
  if ((st = check_matrix(d_y, "y", rows, cols, ld_y, elt, true)) != CKM_OK) return st;
  const hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case CKM_F32: launch_dropout<float>(rows, cols, d_x, ld_x, d_residual, ld_residual, args, d_y, ld_y, s); break;
    case CKM_F16: launch_dropout<_Float16>(rows, cols, d_x, ld_x, d_residual, ld_residual, args, d_y, ld_y, s); break;
    default: launch_dropout<__bf16>(rows, cols, d_x, ld_x, d_residual, ld_residual, args, d_y, ld_y, s); break;
  }
  return launched("dropout launch");
}
