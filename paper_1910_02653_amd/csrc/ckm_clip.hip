// The 2-norm over many tensors, and the tensors scaled so that it is at most a given
// one: norm = sqrt(sum g^2), y = g min(1, max_norm / (norm + eps)).
//
// A launch takes up to 112 tensors in its arguments: no table on the device has to be
// written before it, and a captured call keeps its own. The tensors are cut into chunks
// of 8192 elements, which the blocks of a launch take in turn; each block leaves one
// sum. The blocks of the scaling add these sums themselves, all in the same order, which
// spares a launch; of long lists, whose sums are many times as many, one block does it
// once (40000 tensors of 64 elements: 3.3 ms of launches instead of 8.9). Squares and sums
// are binary64: no gradient of binary32 or bfloat16 is too large or too small for its square.
//
// Bound by memory: every element is read twice and written once. f16 24 blocks of
// width 2048 (2.4 GB) 1375 us: the norm 409 (5.9 TB/s), the scaling 928 (5.2). The norm of
// 1 GiB takes 182 us in f16 and bf16, 184 in f32; with the scaling 576, 573 and 605. A
// small list costs its two launches, 10 us, and the host's walk over the list, 24.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

#include "ckm_ops.h"

namespace ckm {
namespace {

constexpr int kBlock = 256, kTensors = 112;
constexpr int kGroups = 4;                       // of a thread in a chunk
constexpr int kChunk = kBlock * kGroups * kVec;  // elements
constexpr int kBlocks = 2048;                    // of a launch, and of all sums but for long lists

struct Entry {
  const void* in;
  void* out;
  int64_t count;
  int32_t type;
  int32_t first;   // chunk
};
struct Table {
  int32_t tensors, chunks;
  Entry e[kTensors];
};

// kBack: the last chunks first, which the sums read last and which are in the caches.
template <bool kBack, typename F>
__device__ __forceinline__ void each_chunk(const Table& t, F&& f) {
  for (int k = blockIdx.x; k < t.chunks; k += gridDim.x) {
    const int c = kBack ? t.chunks - 1 - k : k;
    int lo = 0, hi = t.tensors;   // the last entry that starts at or before c
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (t.e[mid].first <= c) lo = mid;
      else hi = mid;
    }
    f(t.e[lo], (int64_t)(c - t.e[lo].first) * kChunk);
  }
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
  for (int by = 1; by < 64; by *= 2) v += __shfl_xor(v, by);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <typename T>
__device__ __forceinline__ double squares(const T* p, int64_t from, int64_t count) {
  Raw8<T> r[kGroups];
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = from + (i * kBlock + threadIdx.x) * kVec;
    r[i] = zero_group<T>();
    if (at < count) r[i] = load_left(p + at, (int)min(count - at, (int64_t)kVec));
  }
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const double v = (double)(float)r[i].get(j);
      sum = fma(v, v, sum);
    }
  }
  return sum;
}

__global__ void __launch_bounds__(kBlock) ckm_norm_parts_kernel(Table t, double* parts) {
  __shared__ double lds[kBlock / 64];
  double sum = 0.0;
  each_chunk<false>(t, [&](const Entry& e, int64_t from) {
    if (e.type == CKM_F32) sum += squares((const float*)e.in, from, e.count);
    else if (e.type == CKM_F16) sum += squares((const _Float16*)e.in, from, e.count);
    else sum += squares((const __bf16*)e.in, from, e.count);
  });
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__device__ __forceinline__ double sum_of(const double* parts, int n, double* lds) {
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kBlock) sum += parts[k];
  return block_sum(sum, lds);
}
__device__ __forceinline__ double norm_of(const double* parts, int n, double* lds) { return sqrt(sum_of(parts, n, lds)); }

__global__ void __launch_bounds__(kBlock) ckm_norm_join_kernel(const double* parts, int n, float* norm) {
  __shared__ double lds[kBlock / 64];
  const double v = norm_of(parts, n, lds);
  if (threadIdx.x == 0) *norm = (float)v;
}

// The same sum, in the same order, for norm_of one value.
__global__ void __launch_bounds__(kBlock) ckm_sum_join_kernel(const double* parts, int n, double* all) {
  __shared__ double lds[kBlock / 64];
  const double v = sum_of(parts, n, lds);
  if (threadIdx.x == 0) *all = v;
}

// factor 2^shift: a factor below binary32's normal range has lost digits there, or all.
template <typename T>
__device__ __forceinline__ void scaled(const Entry& e, int64_t from, float factor, int shift) {
  Raw8<T> r[kGroups];
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = from + (i * kBlock + threadIdx.x) * kVec;
    if (at < e.count) r[i] = load_left((const T*)e.in + at, (int)min(e.count - at, (int64_t)kVec));
  }
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int64_t at = from + (i * kBlock + threadIdx.x) * kVec;
    if (at >= e.count) continue;
    float v[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = ldexpf((float)r[i].get(j) * factor, shift);
    store_part<false>((T*)e.out + at, rounded8<T>(v), 0, (int)min(e.count - at, (int64_t)kVec));
  }
}

__global__ void __launch_bounds__(kBlock) ckm_clip_kernel(Table t, const double* parts, int n, double max_norm,
                                                          double eps, float* norm) {
  __shared__ double lds[kBlock / 64];
  const double v = norm_of(parts, n, lds);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  // NaN stays; a max_norm of inf bounds nothing, a norm of inf neither
  const double f = max_norm == INFINITY && v == INFINITY ? 1.0 : max_norm / (v + eps);
  int shift = 0;
  const float factor = f > 1.0 ? 1.0f : f < 0x1p-126 ? (float)frexp(f, &shift) : (float)f;
  each_chunk<true>(t, [&](const Entry& e, int64_t from) {
    if (factor == 1.0f && shift == 0 && e.out == e.in) return;
    if (e.type == CKM_F32) scaled<float>(e, from, factor, shift);
    else if (e.type == CKM_F16) scaled<_Float16>(e, from, factor, shift);
    else scaled<__bf16>(e, from, factor, shift);
  });
}

int launches(int64_t tensors) { return (int)((tensors + kTensors - 1) / kTensors); }
// Blocks of a launch: a list of many launches leaves fewer sums a launch.
int most_blocks(int64_t tensors) { return std::max(128, kBlocks / std::max(1, launches(tensors))); }

// Calls f(table, blocks, blocks of the launches before) for each launch, from the last
// one to the first if kBack; returns the number of blocks.
template <bool kBack, typename F>
int each_launch(int64_t count, const ckm_tensor* t, F&& f) {
  const int most = most_blocks(count);
  int blocks = 0;
  Table table;
  for (int64_t at = 0; at < count; at += kTensors) {
    const int64_t k = kBack ? (count - 1) / kTensors * kTensors - at : at;
    table.tensors = (int32_t)std::min<int64_t>(kTensors, count - k);
    int64_t chunks = 0;
    int used = 0;
    for (int i = 0; i < table.tensors; ++i) {
      const ckm_tensor& v = t[k + i];
      if (!v.count) continue;
      table.e[used++] = {v.d_in, v.d_out, v.count, (int32_t)v.type, (int32_t)chunks};
      chunks += (v.count + kChunk - 1) / kChunk;
    }
    if (!used) continue;
    table.tensors = used;
    table.chunks = (int32_t)chunks;
    const int n = (int)std::min<int64_t>(chunks, most);
    f(table, n, blocks);
    blocks += n;
  }
  return blocks;
}

ckm_status check_tensors(int64_t count, const ckm_tensor* t) {
  if (count < 0) return set_error(CKM_E_INVALID_ARG, "%lld tensors", (long long)count);
  if (count > CKM_MAX_TENSORS) return set_error(CKM_E_UNSUPPORTED, "%lld tensors", (long long)count);
  if (count && !t) return set_error(CKM_E_INVALID_ARG, "tensors is NULL");
  int64_t chunks = 0;   // of a launch
  for (int64_t k = 0; k < count; ++k) {
    if (k % kTensors == 0) chunks = 0;
    if (t[k].type < 0 || t[k].type > CKM_BF16 || !dtype_ok((int)t[k].type))
      return set_error(CKM_E_INVALID_ARG, "tensor %lld: unknown type %lld", (long long)k, (long long)t[k].type);
    if (t[k].count < 0) return set_error(CKM_E_INVALID_ARG, "tensor %lld: %lld elements", (long long)k, (long long)t[k].count);
    if (t[k].count > INT64_MAX / 8) return set_error(CKM_E_UNSUPPORTED, "tensor %lld: %lld elements", (long long)k, (long long)t[k].count);
    if (!t[k].count) continue;
    if (!t[k].d_in) return set_error(CKM_E_INVALID_ARG, "tensor %lld is NULL", (long long)k);
    if ((uintptr_t)t[k].d_in % dtype_bytes((int)t[k].type))
      return set_error(CKM_E_INVALID_ARG, "tensor %lld is not aligned to its elements", (long long)k);
    chunks += (t[k].count + kChunk - 1) / kChunk;
    if (chunks > INT32_MAX - kBlocks) return set_error(CKM_E_UNSUPPORTED, "tensor %lld: %lld elements", (long long)k, (long long)t[k].count);
  }
  return CKM_OK;
}

// Outputs: there, and none over another tensor's input or output.
ckm_status check_outputs(int64_t count, const ckm_tensor* t) {
  struct Span {
    uintptr_t from, to;
    int64_t of;
    bool out;
  };
  std::vector<Span> spans;
  spans.reserve(2 * count);
  for (int64_t k = 0; k < count; ++k) {
    if (!t[k].count) continue;
    const size_t elt = dtype_bytes((int)t[k].type), bytes = t[k].count * elt;
    if (!t[k].d_out) return set_error(CKM_E_INVALID_ARG, "tensor %lld: out is NULL", (long long)k);
    if ((uintptr_t)t[k].d_out % elt) return set_error(CKM_E_INVALID_ARG, "tensor %lld: out is not aligned to its elements", (long long)k);
    spans.push_back({(uintptr_t)t[k].d_out, (uintptr_t)t[k].d_out + bytes, k, true});
    if (t[k].d_out != t[k].d_in) spans.push_back({(uintptr_t)t[k].d_in, (uintptr_t)t[k].d_in + bytes, k, false});
  }
  std::sort(spans.begin(), spans.end(), [](const Span& p, const Span& q) { return p.from < q.from; });
  // the span of each kind that reaches furthest so far
  const Span *in = nullptr, *out = nullptr;
  for (const Span& s : spans) {
    const Span* over = out && out->to > s.from ? out : s.out && in && in->to > s.from ? in : nullptr;
    if (over)
      return set_error(CKM_E_INVALID_ARG, "the output of tensor %lld overlaps tensor %lld",
                       (long long)(s.out ? s.of : over->of), (long long)(s.out ? over->of : s.of));
    const Span*& last = s.out ? out : in;
    if (!last || s.to > last->to) last = &s;
  }
  return CKM_OK;
}

// The norm: there, and not inside a tensor or, given outputs, one of them.
ckm_status check_norm(int64_t count, const ckm_tensor* t, const float* norm, bool outputs) {
  if (!norm || (uintptr_t)norm % 4) return set_error(CKM_E_INVALID_ARG, "norm is NULL or not aligned to 4 bytes");
  const uintptr_t at = (uintptr_t)norm;
  for (int64_t k = 0; k < count; ++k) {
    const size_t bytes = t[k].count * dtype_bytes((int)t[k].type);
    const auto over = [&](const void* p) { return bytes && (uintptr_t)p < at + 4 && at < (uintptr_t)p + bytes; };
    if (over(t[k].d_in) || (outputs && over(t[k].d_out)))
      return set_error(CKM_E_INVALID_ARG, "norm overlaps tensor %lld", (long long)k);
  }
  return CKM_OK;
}

// The blocks' sums, and the sum of them.
size_t parts_bytes(int64_t count) { return count ? ((size_t)launches(count) * most_blocks(count) + 1) * sizeof(double) : 0; }

ckm_status check_parts(int64_t count, void* work, size_t work_bytes) {
  const size_t need = parts_bytes(count);
  if (need && (!work || work_bytes < need))
    return set_error(CKM_E_INVALID_ARG, "work buffer of %zu bytes, %zu needed", work ? work_bytes : (size_t)0, need);
  if ((uintptr_t)work % 8) return set_error(CKM_E_INVALID_ARG, "work is not aligned to 8 bytes");
  return CKM_OK;
}

int launch_parts(int64_t count, const ckm_tensor* t, double* parts, hipStream_t s) {
  return each_launch<false>(count, t, [&](const Table& table, int blocks, int before) {
    ckm_norm_parts_kernel<<<blocks, kBlock, 0, s>>>(table, parts + before);
  });
}

}  // namespace
}  // namespace ckm

extern "C" ckm_status ckm_norm_workspace_size(int64_t count, size_t* bytes) {
  using namespace ckm;
  if (!bytes) return set_error(CKM_E_INVALID_ARG, "bytes is NULL");
  if (count < 0) return set_error(CKM_E_INVALID_ARG, "%lld tensors", (long long)count);
  if (count > CKM_MAX_TENSORS) return set_error(CKM_E_UNSUPPORTED, "%lld tensors", (long long)count);
  *bytes = parts_bytes(count);
  return CKM_OK;
}

extern "C" ckm_status ckm_norm_async(int64_t count, const ckm_tensor* tensors, float* d_norm, void* d_work,
                                     size_t work_bytes, void* stream) {
  using namespace ckm;
  ckm_status st = check_tensors(count, tensors);
  if (st != CKM_OK) return st;
  if ((st = check_norm(count, tensors, d_norm, false)) != CKM_OK) return st;
  if ((st = check_parts(count, d_work, work_bytes)) != CKM_OK) return st;
  const int n = launch_parts(count, tensors, (double*)d_work, (hipStream_t)stream);
  ckm_norm_join_kernel<<<1, kBlock, 0, (hipStream_t)stream>>>((const double*)d_work, n, d_norm);
  return launched("norm launch");
}

extern "C" ckm_status ckm_clip_async(int64_t count, const ckm_tensor* tensors, double max_norm, double eps,
                                     float* d_norm, void* d_work, size_t work_bytes, void* stream) {
  using namespace ckm;
  try {
    ckm_status st = check_tensors(count, tensors);
    if (st != CKM_OK) return st;
    if (!(max_norm >= 0.0)) return set_error(CKM_E_INVALID_ARG, "max_norm = %g", max_norm);
    if (!(eps >= 0.0 && std::isfinite(eps))) return set_error(CKM_E_INVALID_ARG, "eps = %g", eps);
    if ((st = check_norm(count, tensors, d_norm, true)) != CKM_OK) return st;
    if ((st = check_outputs(count, tensors)) != CKM_OK) return st;
    if ((st = check_parts(count, d_work, work_bytes)) != CKM_OK) return st;
    const hipStream_t s = (hipStream_t)stream;
    double* parts = (double*)d_work;
    int n = launch_parts(count, tensors, parts, s);
    if (n > kBlocks) {
      double* all = parts + (size_t)launches(count) * most_blocks(count);
      ckm_sum_join_kernel<<<1, kBlock, 0, s>>>(parts, n, all);
      parts = all;
      n = 1;
    }
    if (n == 0) {
      ckm_norm_join_kernel<<<1, kBlock, 0, s>>>(parts, 0, d_norm);
    } else {
      each_launch<true>(count, tensors, [&](const Table& table, int blocks, int before) {
        ckm_clip_kernel<<<blocks, kBlock, 0, s>>>(table, parts, n, max_norm, eps, before == 0 ? d_norm : nullptr);
      });
    }
    return launched("clip launch");
  } catch (...) {
    return set_error(CKM_E_NOMEM, "no host memory to check %lld tensors", (long long)count);
  }
}
