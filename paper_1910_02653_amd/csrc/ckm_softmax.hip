// Softmax of attention scores with scale, masks and dropout in one pass, and its
// gradient.
//
//   forward   t = scale x + mask over the visible keys, m = max t, z = 1 / sum
//             exp(t - m), y = D(exp(t - m) z); a row that sees nothing gives
//             zeros and the statistics (0, 0)
//   gradient  p = exp(t - m) z from the scores and the statistics, g = D(dy),
//             dx = scale p (g - sum p g)
//
// Neither the probabilities before the dropout nor its mask are ever stored: the
// gradient makes both again from the scores and the statistics, the mask bit for bit.
// Logits, statistics and sums are in binary32. exp(v), v = t - m <= 0, is 2^(v log2 e).
// Its relative error beside the unit's last place, with u = 2^-24: in binary32 u,
// since what the product's rounding loses is made good (four more operations a score:
// f32 16x1024x1024 27 us with and without, 128 single queries on 32768 keys 11.1 -> 12); in
// the 16-bit types, whose own rounding is far coarser, 1.3 u |v| where logits are formed
// (the factor and the product) and 3.3 u |v| where they are not (scale log2 e, the
// difference of the scores, the product).
//
// Bound by memory, the dropout's draws a close second: f16 16x2048x2048 without
// causal mask moves 269 MB in 50 us (5.4 TB/s, where a large copy moves 5.2), causal
// 202 MB in 44 us, its gradient 269 MB in 55 us. What it took: a row's loads all in
// flight before its arithmetic; the arithmetic of a score down to a maximum, a
// difference, 2^v, a sum and three products; the dropout's choice on packed halves; one
// row set a block and no loop, whose invariants had cost a third of the registers
// (gradient 73 -> 56 us); scores held as the words they were loaded as.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "ckm_ops.h"

namespace ckm {
namespace {

// Rows in memory: elements between batches, heads, queries; where those make one
// stride from row to row, that.
struct Strided {
  const void* p;
  int64_t s[3];
  int64_t row;   // -1: there is no such stride
};

struct SoftmaxArgs {
  int64_t rows;
  int32_t heads, queries, keys;
  Strided x, dy, y; // y: probabilities, or the scores' gradient
  float* stats;     // [rows][2]: m, z (read by the gradient)
  float scale;
  bool causal;
  const int32_t* lengths;
  int mask_kind;
  Strided mask;
  DropArgs drop;
  bool places;      // a row's batch, head and query matter: masks, or rows without one stride
};

struct Row {
  int64_t n;        // its number
  int32_t b, h, i;
  int32_t seen;     // keys seen are below this (masks aside)
};
__device__ __forceinline__ Row row_of(const SoftmaxArgs& a, int64_t row) {
  Row r = {row, 0, 0, 0, a.keys};
  if (!a.places) return r;
  const uint32_t bh = (uint32_t)row / (uint32_t)a.queries;
  r.i = (uint32_t)row - bh * a.queries;
  r.b = bh / (uint32_t)a.heads;
  r.h = bh - r.b * a.heads;
  int32_t seen = a.keys;
  if (a.lengths) seen = min(seen, a.lengths[r.b]);
  if (a.causal) seen = min(seen, r.i + (a.keys - a.queries) + 1);
  r.seen = max(seen, 0);
  return r;
}
__device__ __forceinline__ int64_t offset_of(const Strided& t, const Row& r) {
  return t.row >= 0 ? r.n * t.row : r.b * t.s[0] + r.h * t.s[1] + r.i * t.s[2];
}

constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0x1.62e43p-1f, kLn2Low = (float)(0.693147180559945309 - (double)kLn2);
// exp(t - m), t <= m. In binary32, what the rounding of p = v log2 e lost goes in as a
// factor 1 + (v - p ln 2); for v = -inf that is NaN, and the 0 before it stays.
template <typename T>
__device__ __forceinline__ float exp_of(float t, float m) {
  const float v = t - m, p = v * kLog2e, e = __builtin_amdgcn_exp2f(p);
  if constexpr (sizeof(T) == 2) return e;
  return fmaf(e, fmaxf(fmaf(-p, kLn2Low, fmaf(-p, kLn2, v)), -1.0f), e);
}

// A row's largest logit m as its exponentials use it, where no logits are formed. In
// the 16-bit types exp(scale x - m) is 2^((x - top) scale log2 e), top the largest
// score: exactly 1 there, as where t - m is formed, so that a row that sees one
// key has probability 1 and gradient 0. The gradient finds top from m: the score
// next to m / scale, which lies within a few 2^-24 of one (or is taken as it is).
template <typename T>
struct Top {
  float m, top, sl;
  __device__ __forceinline__ Top(float m_, float top_, float scale) : m(m_), top(top_), sl(scale * kLog2e) {}
  __device__ __forceinline__ Top(float m_, float scale) : m(m_), top(0.0f), sl(scale * kLog2e) {
    if constexpr (sizeof(T) == 2) {
      const float q = fmaxf(m / scale, kLowest), near = (float)rounded<T>(q);
      top = fabsf(q - near) <= 0x1p-20f * fabsf(q) ? near : q;
    }
  }
};
// exp(scale x - m) of a group's scores.
template <typename T>
__device__ __forceinline__ void exps8(float (&e)[kVec], const Raw8<T>& x, const Top<T>& top, float scale) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    if constexpr (sizeof(T) == 2)
      e[j] = __builtin_amdgcn_exp2f(((float)x.get(j) - top.top) * top.sl);
    else
      e[j] = exp_of<T>((float)x.get(j) * scale, top.m);
  }
}
// The largest of a group's scores.
template <typename T>
__device__ __forceinline__ float top8(const Raw8<T>& x) {
  if constexpr (std::is_same<T, _Float16>::value) {   // two at a time
    typedef _Float16 Half2 __attribute__((ext_vector_type(2)));
    const auto two = [&](int k) { return __builtin_bit_cast(Half2, x.w[k]); };
    const Half2 m = __builtin_elementwise_max(__builtin_elementwise_max(two(0), two(1)),
                                              __builtin_elementwise_max(two(2), two(3)));
    return fmaxf((float)m.x, (float)m.y);
  } else {
    float m = (float)x.get(0);
#pragma unroll
    for (int j = 1; j < kVec; ++j) m = fmaxf(m, (float)x.get(j));
    return m;
  }
}

// What a row's logits are made of: the scores alone (kPlain: with a scale that is
// not positive, or near the range's end), a mask of truth values or of values to
// add. Without a mask and with an ordinary scale (kNoMask) no logits are formed.
enum : int { kNoMask = 0, kBool = 1, kAdd = 2, kPlain = 3 };
int mask_form(int mask_kind, float scale) {
  return mask_kind == CKM_MASK_BOOL  ? kBool
         : mask_kind == CKM_MASK_ADD ? kAdd
         : scale > 1e-30f && scale < 1e30f ? kNoMask : kPlain;
}
template <int kMask, typename T>
using MaskType = std::conditional_t<kMask == kBool, uint8_t, T>;

template <int kMask, typename T>
__device__ __forceinline__ const MaskType<kMask, T>* mask_row(const SoftmaxArgs& a, const Row& r) {
  return (const MaskType<kMask, T>*)a.mask.p + offset_of(a.mask, r);
}
// The logits of a group; -inf where a key is not seen. Scores there are not used,
// whatever they hold. left: seen keys from the group's first on.
template <int kMask, typename T>
__device__ __forceinline__ void logits8(float (&t)[kVec], const SoftmaxArgs& a, const Raw8<T>& x,
                                        const Raw8<MaskType<kMask, T>>& m, int left) {
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    bool seen = j < left;
    float add = 0.0f;
    if constexpr (kMask == kAdd) {
      add = (float)m.get(j);
      seen &= add != -__builtin_inff();
    }
    if constexpr (kMask == kBool) seen &= m.get(j) != 0;
    const float v = kMask == kAdd ? fmaf((float)x.get(j), a.scale, add) : (float)x.get(j) * a.scale;
    t[j] = seen ? v : -__builtin_inff();
  }
}

// The gradient that reaches a group's probabilities through the dropout, but for
// its factor, which the row's sum and the result take together; 0 where a mask
// left the exponential 0.
template <int kMask, typename T>
__device__ __forceinline__ void grads8(float (&g)[kVec], const SoftmaxArgs& a, DropSite site, Raw8<T> dy,
                                       const float (&e)[kVec], int64_t row, int col) {
  if (a.drop.on) drop_choice(dy, a.drop, site, col / kVec, (uint32_t)row);
#pragma unroll
  for (int j = 0; j < kVec; ++j) g[j] = kMask != kNoMask && e[j] == 0.0f ? 0.0f : (float)dy.get(j);
}

constexpr int softmax_block(int lanes) { return lanes < 256 ? 256 : lanes; }

// A row in the registers of kLanes threads, kPer groups each. kEven: rows of
// whole groups. With kNoMask the unseen scores of a row's last group are set to
// -inf once.
template <typename T, int kLanes, int kPer, bool kBack, int kMask, bool kEven>
__global__ void __launch_bounds__(softmax_block(kLanes)) ckm_softmax_kernel(SoftmaxArgs a) {
  constexpr int kBlock = softmax_block(kLanes), kRowsAt = kBlock / kLanes;
  __shared__ float lds[kLanes > 64 ? 2 * kBlock / 64 : 1];
  const int lane = threadIdx.x % kLanes;
  const DropSite site = drop_site(a.drop);
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRowsAt + row_in_block<kLanes>();
  const bool live = row < a.rows;
  const Row r = row_of(a, live ? row : a.rows - 1);
  const T* x = (const T*)a.x.p + offset_of(a.x, r);
  const T* dy = (const T*)a.dy.p + offset_of(a.dy, r);
  constexpr bool kMasked = kMask == kBool || kMask == kAdd;
  const MaskType<kMask, T>* mask = kMasked ? mask_row<kMask, T>(a, r) : nullptr;
  T* y = (T*)const_cast<void*>(a.y.p) + offset_of(a.y, r);
  const int seen = live ? r.seen : 0, keys = live ? a.keys : 0;
  // every load of the row first, then the arithmetic
  Raw8<T> rx[kPer], rd[kBack ? kPer : 1];
  Raw8<MaskType<kMask, T>> rm[kMasked ? kPer : 1];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int col = (lane + i * kLanes) * kVec;
    if (col < seen) {
      rx[i] = load_cols<kEven>(x, col, a.keys);
      if constexpr (kBack) rd[i] = load_cols<kEven>(dy, col, a.keys);
      if constexpr (kMasked) rm[i] = load_cols<kEven>(mask, col, a.keys);
    }
  }
  float t[kPer][kVec];   // logits, then exponentials
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int col = (lane + i * kLanes) * kVec;
    if (col < seen) {
      fix_tail<kEven>(rx[i], col, a.keys);
      if constexpr (kBack) fix_tail<kEven>(rd[i], col, a.keys);
      if constexpr (kMask != kNoMask) {
        if constexpr (kMasked) fix_tail<kEven>(rm[i], col, a.keys);
        logits8<kMask>(t[i], a, rx[i], rm[kMasked ? i : 0], seen - col);
      } else {
        hide(rx[i], seen - col, (T)-__builtin_inff());
        if constexpr (kBack) hide(rd[i], seen - col, (T)0);
      }
    }
  }
  if constexpr (!kBack) {
    float m = kLowest;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec;
      if (col >= seen) continue;
      if constexpr (kMask != kNoMask) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) m = fmaxf(m, t[i][j]);
      } else {
        m = fmaxf(m, top8(rx[i]));
      }
    }
    m = reduce_row<OpMax, kLanes, kBlock>(m, lds, 0);
    float most = m;   // a score, with kNoMask
    if constexpr (kMask == kNoMask) {
      m *= a.scale;
      // a logit past the range (binary16 scores have none) is an infinite one, as where
      // logits are formed
      if constexpr (std::is_same<T, __bf16>::value)
        most = m == __builtin_inff() ? __builtin_nanf("") : m == -__builtin_inff() ? __builtin_inff() : most;
      m = fmaxf(m, kLowest);
    }
    const Top<T> top(m, most, a.scale);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec;
      if (col >= seen) continue;
      if constexpr (kMask == kNoMask) exps8(t[i], rx[i], top, a.scale);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        if constexpr (kMask != kNoMask) t[i][j] = exp_of<T>(t[i][j], m);
        sum += t[i][j];
      }
    }
    sum = reduce_row<OpSum, kLanes, kBlock>(sum, lds, 1);
    const float z = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (live && lane == 0 && a.stats) {
      a.stats[2 * row] = sum == 0.0f ? 0.0f : m;
      a.stats[2 * row + 1] = z;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int group = lane + i * kLanes, col = group * kVec;
      if (col >= keys) continue;
      Raw8<T> o = zero_group<T>();
      if (col < seen) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) t[i][j] *= z;
        o = dropped8<T>(t[i], a.drop, site, group, (uint32_t)row);
      }
      store_part<kEven>(y, o, col, keys);
    }
  } else {
    const float m = live ? a.stats[2 * row] : 0.0f, z = live ? a.stats[2 * row + 1] : 0.0f;
    const Top<T> top(m, a.scale);
    float g[kPer][kVec];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec;
      if (col >= seen) continue;
      if constexpr (kMask != kNoMask) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) t[i][j] = exp_of<T>(t[i][j], m);
      } else {
        exps8(t[i], rx[i], top, a.scale);
      }
      grads8<kMask>(g[i], a, site, rd[i], t[i], row, col);
#pragma unroll
      for (int j = 0; j < kVec; ++j) sum = fmaf(t[i][j], g[i][j], sum);
    }
    // p = e z: the row's z goes into its sum and its factor
    const float by = a.scale * a.drop.scale * z;
    sum = reduce_row<OpSum, kLanes, kBlock>(sum, lds, 0) * z;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int col = (lane + i * kLanes) * kVec;
      if (col >= keys) continue;
      float o[kVec] = {};
      if (col < seen) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = t[i][j] * ((g[i][j] - sum) * by);
      }
      store_part<kEven>(y, rounded8<T>(o), col, keys);
    }
  }
}

// ---------------------------------------------------------------------------
// Long rows, and few of them: a row is cut into `splits` shares of `chunk` keys
// (a multiple of a block's 2048). The first launch leaves each share's maximum
// and sum of exponentials (the gradient: its sum of e g); the second joins a row's
// shares in each of its blocks and makes the share's outputs.
// ---------------------------------------------------------------------------

constexpr int kSplitBlock = 256, kSplitSpan = kSplitBlock * kVec, kMaxSplits = kSplitBlock;
constexpr int kSplitPer = 2;   // spans loaded together

// The groups of a share that a thread holds at a time: kSplitPer from `col` on, a
// span apart.
template <typename T, bool kBack, int kMask>
struct Span {
  static constexpr bool kMasked = kMask == kBool || kMask == kAdd;
  Raw8<T> x[kSplitPer], dy[kBack ? kSplitPer : 1];
  Raw8<MaskType<kMask, T>> m[kMasked ? kSplitPer : 1];
  float t[kSplitPer][kVec];   // logits (not with kNoMask), then exponentials

  __device__ __forceinline__ void load(const SoftmaxArgs& a, const T* px, const T* pdy, const MaskType<kMask, T>* pm,
                                       int col, int to) {
#pragma unroll
    for (int i = 0; i < kSplitPer; ++i) {
      const int c = col + i * kSplitSpan;
      if (c < to) {
        x[i] = load_cols<false>(px, c, a.keys);
        if constexpr (kBack) dy[i] = load_cols<false>(pdy, c, a.keys);
        if constexpr (kMasked) m[i] = load_cols<false>(pm, c, a.keys);
      }
    }
#pragma unroll
    for (int i = 0; i < kSplitPer; ++i) {
      const int c = col + i * kSplitSpan;
      if (c < to) {
        fix_tail<false>(x[i], c, a.keys);
        if constexpr (kBack) fix_tail<false>(dy[i], c, a.keys);
        if constexpr (kMasked) fix_tail<false>(m[i], c, a.keys);
        if constexpr (kMask == kNoMask) {
          hide(x[i], to - c, (T)-__builtin_inff());
          if constexpr (kBack) hide(dy[i], to - c, (T)0);
        } else {
          logits8<kMask>(t[i], a, x[i], m[kMasked ? i : 0], to - c);
        }
      }
    }
  }
  __device__ __forceinline__ float largest(const SoftmaxArgs& a, int i) const {
    if constexpr (kMask == kNoMask) return top8(x[i]) * a.scale;
    float v = t[i][0];
#pragma unroll
    for (int j = 1; j < kVec; ++j) v = fmaxf(v, t[i][j]);
    return v;
  }
  __device__ __forceinline__ void exps(const SoftmaxArgs& a, const Top<T>& top, int i) {
    if constexpr (kMask == kNoMask) {
      exps8(t[i], x[i], top, a.scale);
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j) t[i][j] = exp_of<T>(t[i][j], top.m);
    }
  }
};

template <typename T, bool kBack, int kMask, bool kJoin>
__global__ void __launch_bounds__(kSplitBlock) ckm_softmax_split_kernel(SoftmaxArgs a, int splits, int32_t chunk,
                                                                        float2* part) {
  __shared__ float lds[2 * kSplitBlock / 64];
  const int64_t item = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (item >= a.rows * splits) return;
  const int64_t row = item / splits;
  const int share = (int)(item - row * splits);
  const DropSite site = drop_site(a.drop);
  const Row r = row_of(a, row);
  const T* x = (const T*)a.x.p + offset_of(a.x, r);
  const T* dy = (const T*)a.dy.p + offset_of(a.dy, r);
  const MaskType<kMask, T>* mask = nullptr;
  if constexpr (kMask == kBool || kMask == kAdd) mask = mask_row<kMask, T>(a, r);
  const int from = share * chunk, first = from + (int)threadIdx.x * kVec;
  const int seen = min(r.seen, from + chunk);   // below 2^31: chunk holds at most 2^30 keys and a block's
  Span<T, kBack, kMask> s;
  if constexpr (!kJoin) {
    const float m = kBack ? a.stats[2 * row] : 0.0f;
    const Top<T> given(m, a.scale);
    float top = kLowest, sum = 0.0f;
    for (int col = first; col < seen; col += kSplitPer * kSplitSpan) {
      s.load(a, x, dy, mask, col, seen);
      float now = top;
      if constexpr (!kBack) {
#pragma unroll
        for (int i = 0; i < kSplitPer; ++i)
          if (col + i * kSplitSpan < seen) now = fmaxf(now, s.largest(a, i));
        sum *= exp_of<T>(top, now);
        top = now;
      }
      const Top<T> at = kBack ? given : Top<T>(now, a.scale);
#pragma unroll
      for (int i = 0; i < kSplitPer; ++i) {
        const int c = col + i * kSplitSpan;
        if (c >= seen) continue;
        s.exps(a, at, i);
        if constexpr (kBack) {
          float g[kVec];
          grads8<kMask>(g, a, site, s.dy[i], s.t[i], row, c);
#pragma unroll
          for (int j = 0; j < kVec; ++j) sum = fmaf(s.t[i][j], g[j], sum);
        } else {
#pragma unroll
          for (int j = 0; j < kVec; ++j) sum += s.t[i][j];
        }
      }
    }
    if constexpr (!kBack) {
      const float all = reduce_row<OpMax, kSplitBlock, kSplitBlock>(top, lds, 0);
      sum *= exp_of<T>(top, all);
      top = all;
    }
    sum = reduce_row<OpSum, kSplitBlock, kSplitBlock>(sum, lds, 1);
    if (threadIdx.x == 0) part[item] = {top, sum};
  } else {
    T* y = (T*)const_cast<void*>(a.y.p) + offset_of(a.y, r);
    const int to = (int)min((int64_t)a.keys, (int64_t)from + chunk);
    // the share's first groups, which do not wait for the shares' sums
    if (first < seen) s.load(a, x, dy, mask, first, seen);
    float2 mine = {kLowest, 0.0f};
    if ((int)threadIdx.x < splits) mine = part[row * splits + threadIdx.x];
    float m, z, sum, by = 1.0f;
    if constexpr (!kBack) {
      m = reduce_row<OpMax, kSplitBlock, kSplitBlock>(mine.x, lds, 0);
      sum = reduce_row<OpSum, kSplitBlock, kSplitBlock>(mine.y * exp_of<T>(mine.x, m), lds, 1);
      z = sum == 0.0f ? 0.0f : 1.0f / sum;
      if (share == 0 && threadIdx.x == 0 && a.stats) {
        a.stats[2 * row] = sum == 0.0f ? 0.0f : m;
        a.stats[2 * row + 1] = z;
      }
    } else {
      m = a.stats[2 * row];
      z = a.stats[2 * row + 1];
      by = a.scale * a.drop.scale * z;
      sum = reduce_row<OpSum, kSplitBlock, kSplitBlock>(mine.y, lds, 0) * z;
    }
    const Top<T> top(m, a.scale);
    for (int col = first; col < to; col += kSplitPer * kSplitSpan) {
      if (col != first && col < seen) s.load(a, x, dy, mask, col, seen);
#pragma unroll
      for (int i = 0; i < kSplitPer; ++i) {
        const int c = col + i * kSplitSpan;
        if (c >= to) continue;
        Raw8<T> o = zero_group<T>();
        if (c < seen) {
          s.exps(a, top, i);
          if constexpr (kBack) {
            float g[kVec];
            grads8<kMask>(g, a, site, s.dy[i], s.t[i], row, c);
#pragma unroll
            for (int j = 0; j < kVec; ++j) s.t[i][j] *= (g[j] - sum) * by;
            o = rounded8<T>(s.t[i]);
          } else {
#pragma unroll
            for (int j = 0; j < kVec; ++j) s.t[i][j] *= z;
            o = dropped8<T>(s.t[i], a.drop, site, c / kVec, (uint32_t)row);
          }
        }
        store_part<false>(y, o, c, a.keys);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// launch rules
// ---------------------------------------------------------------------------

// Shares of a row, 1 when a row stays whole in registers, which is faster wherever
// it fits, for few rows too: f16, 16 rows of 16384 keys 4.3 us whole, 6.8 in eight
// shares; 8 of 32768 5.3, 8 of 33000 in shares 6.6. Shares fill the chip with about
// 1024 blocks (32 rows of 131072: 9.9 us; with twice as many, half as long, 14.5).
// The number fixes the order of the sums, so it depends on the sizes alone.
constexpr int kWholeKeys = 32768;
int softmax_splits(int64_t rows, int64_t keys) {
  if (keys <= kWholeKeys) return 1;
  const int64_t spans = (keys + kSplitSpan - 1) / kSplitSpan;
  const int64_t wanted = std::max<int64_t>(2, (1024 + rows - 1) / std::max<int64_t>(rows, 1));
  return (int)std::min<int64_t>(std::min<int64_t>((spans + kSplitPer - 1) / kSplitPer, wanted), kMaxSplits);
}
// One set of work to a block, in two dimensions: a launch has fewer than 2^32
// threads in each.
dim3 grid_of(int64_t blocks) {
  const int64_t wide = std::min<int64_t>(blocks, 1 << 20);
  return dim3((uint32_t)wide, (uint32_t)((blocks + wide - 1) / wide));
}

template <typename T, bool kBack, int kLanes, int kPer>
void launch_whole_as(const SoftmaxArgs& a, hipStream_t s) {
  constexpr int kBlock = softmax_block(kLanes), kRowsAt = kBlock / kLanes;
  const dim3 grid = grid_of((a.rows + kRowsAt - 1) / kRowsAt);
  switch (mask_form(a.mask_kind, a.scale)) {
    case kBool: ckm_softmax_kernel<T, kLanes, kPer, kBack, kBool, false><<<grid, kBlock, 0, s>>>(a); break;
    case kAdd: ckm_softmax_kernel<T, kLanes, kPer, kBack, kAdd, false><<<grid, kBlock, 0, s>>>(a); break;
    case kPlain: ckm_softmax_kernel<T, kLanes, kPer, kBack, kPlain, false><<<grid, kBlock, 0, s>>>(a); break;
    default:
      if (a.keys % kVec == 0)
        ckm_softmax_kernel<T, kLanes, kPer, kBack, kNoMask, true><<<grid, kBlock, 0, s>>>(a);
      else
        ckm_softmax_kernel<T, kLanes, kPer, kBack, kNoMask, false><<<grid, kBlock, 0, s>>>(a);
  }
}

template <typename T, bool kBack, int kMask>
void launch_split_as(const SoftmaxArgs& a, int splits, void* work, hipStream_t s) {
  const int64_t spans = ((int64_t)a.keys + kSplitSpan - 1) / kSplitSpan;
  const int32_t chunk = (int32_t)((spans + splits - 1) / splits * kSplitSpan);
  const dim3 grid = grid_of(a.rows * splits);
  ckm_softmax_split_kernel<T, kBack, kMask, false><<<grid, kSplitBlock, 0, s>>>(a, splits, chunk, (float2*)work);
  ckm_softmax_split_kernel<T, kBack, kMask, true><<<grid, kSplitBlock, 0, s>>>(a, splits, chunk, (float2*)work);
}

// Threads and groups a thread for whole rows. Forward: four groups a thread, so that
// what a row costs once (its place, two sums, its statistics) is shared by more
// columns. Measured against two groups on twice the threads, with dropout (us):
// bf16 64x16x256x300 73.6 / 88.6, 4x16x1024x1024 causal 41.8 / 44.5, f16
// 16x2048x2048 causal 43.1 / 45.7 (one group 66.3), bf16 4x4096x4096 causal 41.4 /
// 44.0 (one 64.3), 4096x16384 causal 51.1 / 58.0; against it 16x16x512x512 causal 49.3 /
// 46.2. The gradient holds a row's exponentials and gradients, and is faster with two
// groups: f16 16x2048x2048 54.1, four 55.0, one 60.3; bf16 2x4096x8192 64.9, four 65.8.
template <typename T, bool kBack>
void launch_softmax(const SoftmaxArgs& a, int splits, void* work, hipStream_t s) {
  if (splits > 1) {
    switch (mask_form(a.mask_kind, a.scale)) {
      case kBool: return launch_split_as<T, kBack, kBool>(a, splits, work, s);
      case kAdd: return launch_split_as<T, kBack, kAdd>(a, splits, work, s);
      case kPlain: return launch_split_as<T, kBack, kPlain>(a, splits, work, s);
      default: return launch_split_as<T, kBack, kNoMask>(a, splits, work, s);
    }
  }
  const int groups = (a.keys + kVec - 1) / kVec;
  if (groups <= 16) return launch_whole_as<T, kBack, 16, 1>(a, s);
  if (groups <= 32) return launch_whole_as<T, kBack, 16, 2>(a, s);
  if constexpr (kBack) {
    if (groups <= 64) launch_whole_as<T, true, 32, 2>(a, s);
    else if (groups <= 128) launch_whole_as<T, true, 64, 2>(a, s);
    else if (groups <= 256) launch_whole_as<T, true, 128, 2>(a, s);
    else if (groups <= 512) launch_whole_as<T, true, 256, 2>(a, s);
    else if (groups <= 1024) launch_whole_as<T, true, 512, 2>(a, s);
    else if (groups <= 2048) launch_whole_as<T, true, 1024, 2>(a, s);
    else launch_whole_as<T, true, 1024, 4>(a, s);
  } else {
    if (groups <= 64) launch_whole_as<T, false, 16, 4>(a, s);
    else if (groups <= 128) launch_whole_as<T, false, 32, 4>(a, s);
    else if (groups <= 256) launch_whole_as<T, false, 64, 4>(a, s);
    else if (groups <= 512) launch_whole_as<T, false, 128, 4>(a, s);
    else if (groups <= 1024) launch_whole_as<T, false, 256, 4>(a, s);
    else if (groups <= 2048) launch_whole_as<T, false, 512, 4>(a, s);
    else launch_whole_as<T, false, 1024, 4>(a, s);
  }
}

template <bool kBack>
void launch_typed(int type, const SoftmaxArgs& a, int splits, void* work, hipStream_t s) {
  switch (type) {
    case CKM_F32: launch_softmax<float, kBack>(a, splits, work, s); break;
    case CKM_F16: launch_softmax<_Float16, kBack>(a, splits, work, s); break;
    default: launch_softmax<__bf16, kBack>(a, splits, work, s); break;
  }
}

// Strides of a [batch, heads, queries] array of rows of `keys` elements: not
// negative, offsets within the address range, and for an output no two rows
// that share an element (each stride spans everything with smaller ones).
ckm_status check_strides(const char* name, const int64_t* stride, const ckm_scores& c, bool output) {
  if (!stride) return set_error(CKM_E_INVALID_ARG, "%s strides are NULL", name);
  const int64_t dim[3] = {c.batch, c.heads, c.queries};
  int order[3] = {0, 1, 2};
  __int128 last = 0;
  for (int k = 0; k < 3; ++k) {
    if (stride[k] < 0) return set_error(CKM_E_INVALID_ARG, "%s: negative stride %lld", name, (long long)stride[k]);
    last += (__int128)(dim[k] - 1) * stride[k];
  }
  if (last > INT64_MAX / 8 - c.keys) return set_error(CKM_E_INVALID_ARG, "%s: strides pass the address range", name);
  if (!output) return CKM_OK;
  std::sort(order, order + 3, [&](int p, int q) { return stride[p] < stride[q]; });
  int64_t span = c.keys;   // elements from the first to past the last one
  for (const int k : order) {
    if (dim[k] == 1) continue;
    if (stride[k] < span) return set_error(CKM_E_INVALID_ARG, "%s: rows overlap (stride %lld)", name, (long long)stride[k]);
    span += (dim[k] - 1) * stride[k];
  }
  return CKM_OK;
}

ckm_status check_scores(const ckm_scores* c, int64_t* rows) {
  if (!c) return set_error(CKM_E_INVALID_ARG, "scores is NULL");
  if (c->batch < 0 || c->heads < 0 || c->queries < 0 || c->keys < 0)
    return set_error(CKM_E_INVALID_ARG, "scores of %lld x %lld x %lld x %lld", (long long)c->batch, (long long)c->heads,
                     (long long)c->queries, (long long)c->keys);
  if (c->batch > CKM_MAX_ROWS || c->heads > CKM_MAX_ROWS || c->queries > CKM_MAX_ROWS ||
      (__int128)c->batch * c->heads * c->queries > CKM_MAX_ROWS || c->keys > CKM_MAX_COLS)
    return set_error(CKM_E_UNSUPPORTED, "scores of %lld x %lld x %lld x %lld", (long long)c->batch, (long long)c->heads,
                     (long long)c->queries, (long long)c->keys);
  *rows = c->batch * c->heads * c->queries;
  return CKM_OK;
}

ckm_status softmax(bool back, ckm_dtype type, const ckm_scores* c, const void* x, const int64_t* x_stride,
                   const void* dy, const int64_t* dy_stride, const ckm_drop* drop, void* y, const int64_t* y_stride,
                   float* stats, void* work, size_t work_bytes, void* stream) {
  if (!dtype_ok(type)) return set_error(CKM_E_INVALID_ARG, "unknown type %d", (int)type);
  SoftmaxArgs a = {};
  ckm_status st = check_scores(c, &a.rows);
  if (st != CKM_OK) return st;
  if (!(c->scale >= -3.4e38f && c->scale <= 3.4e38f)) return set_error(CKM_E_INVALID_ARG, "scale = %g", (double)c->scale);
  if (c->flags & ~CKM_SCORES_CAUSAL) return set_error(CKM_E_INVALID_ARG, "unknown flags 0x%x", c->flags);
  if (c->mask_kind != CKM_MASK_NONE && c->mask_kind != CKM_MASK_BOOL && c->mask_kind != CKM_MASK_ADD)
    return set_error(CKM_E_INVALID_ARG, "unknown mask kind %d", c->mask_kind);
  if ((st = drop_args(drop, &a.drop)) != CKM_OK) return st;
  if (a.rows == 0 || (back && c->keys == 0)) return CKM_OK;
  const size_t elt = dtype_bytes(type);
  // a NULL or misaligned array, then its strides
  const auto check = [&](const void* p, const char* name, const int64_t* stride, size_t bytes, bool output) {
    const ckm_status s = check_matrix(p, name, 1, c->keys, 0, bytes, false);
    return s != CKM_OK ? s : check_strides(name, stride, *c, output);
  };
  if (c->keys > 0) {
    if ((st = check(x, "x", x_stride, elt, false)) != CKM_OK) return st;
    if (back && (st = check(dy, "dy", dy_stride, elt, false)) != CKM_OK) return st;
    if ((st = check(y, back ? "dx" : "y", y_stride, elt, true)) != CKM_OK) return st;
    if (c->mask_kind != CKM_MASK_NONE &&
        (st = check(c->d_mask, "mask", c->mask_stride, c->mask_kind == CKM_MASK_ADD ? elt : 1, false)) != CKM_OK)
      return st;
  }
  if (back && !stats) return set_error(CKM_E_INVALID_ARG, "stats is NULL");
  if ((uintptr_t)stats % 4) return set_error(CKM_E_INVALID_ARG, "stats is not aligned to 4 bytes");
  if ((uintptr_t)c->d_lengths % 4) return set_error(CKM_E_INVALID_ARG, "lengths is not aligned to 4 bytes");
  const int splits = softmax_splits(a.rows, c->keys);
  const size_t need = splits > 1 ? (size_t)a.rows * splits * sizeof(float2) : 0;
  if (need > 0 && (!work || work_bytes < need))
    return set_error(CKM_E_INVALID_ARG, "work buffer of %zu bytes, %zu needed", work ? work_bytes : (size_t)0, need);
  if ((uintptr_t)work % 8) return set_error(CKM_E_INVALID_ARG, "work is not aligned to 8 bytes");
  a.heads = (int32_t)c->heads;
  a.queries = (int32_t)c->queries;
  a.keys = (int32_t)c->keys;
  const auto strided = [&](const void* p, const int64_t* s) {
    Strided v = {p, {0, 0, 0}, 0};
    if (!s) return v;
    for (int k = 0; k < 3; ++k) v.s[k] = s[k];
    // one stride d for all rows: heads lie queries d apart, batches heads queries d
    const int64_t d = c->queries > 1 ? s[2] : c->heads > 1 ? s[1] : s[0];
    v.row = d;
    if (c->queries > 1 && c->heads > 1 && s[1] != (__int128)c->queries * d) v.row = -1;
    if (c->batch > 1 && c->heads * c->queries > 1 && s[0] != (__int128)c->heads * c->queries * d) v.row = -1;
    return v;
  };
  a.x = strided(x, x_stride);
  a.dy = strided(dy, dy_stride);
  a.y = strided(y, y_stride);
  a.stats = stats;
  a.scale = c->scale;
  a.causal = c->flags & CKM_SCORES_CAUSAL;
  a.lengths = c->d_lengths;
  a.mask_kind = c->mask_kind;
  a.mask = strided(c->d_mask, c->mask_kind == CKM_MASK_NONE ? nullptr : c->mask_stride);
  a.places = a.causal || a.lengths || a.x.row < 0 || a.dy.row < 0 || a.y.row < 0 || a.mask.row < 0;
  if (back)
    launch_typed<true>(type, a, splits, work, (hipStream_t)stream);
  else
    launch_typed<false>(type, a, splits, work, (hipStream_t)stream);
  return launched(back ? "softmax gradient launch" : "softmax launch");
}

}  // namespace
}  // namespace ckm

extern "C" ckm_status ckm_softmax_workspace_size(const ckm_scores* scores, size_t* bytes) {
  using namespace ckm;
  if (!bytes) return set_error(CKM_E_INVALID_ARG, "bytes is NULL");
  int64_t rows = 0;
  const ckm_status st = check_scores(scores, &rows);
  if (st != CKM_OK) return st;
  const int splits = rows ? softmax_splits(rows, scores->keys) : 1;
  *bytes = splits > 1 ? (size_t)rows * splits * sizeof(float2) : 0;
  return CKM_OK;
}

extern "C" ckm_status ckm_softmax_async(ckm_dtype type, const ckm_scores* scores, const void* d_x,
                                        const int64_t* x_stride, const ckm_drop* drop, void* d_y,
                                        const int64_t* y_stride, float* d_stats, void* d_work, size_t work_bytes,
                                        void* stream) {
  return ckm::softmax(false, type, scores, d_x, x_stride, nullptr, nullptr, drop, d_y, y_stride, d_stats, d_work,
                      work_bytes, stream);
}

extern "C" ckm_status ckm_softmax_backward_async(ckm_dtype type, const ckm_scores* scores, const void* d_dy,
                                                 const int64_t* dy_stride, const void* d_x, const int64_t* x_stride,
                                                 const float* d_stats, const ckm_drop* drop, void* d_dx,
                                                 const int64_t* dx_stride, void* d_work, size_t work_bytes,
                                                 void* stream) {
  return ckm::softmax(true, type, scores, d_x, x_stride, d_dy, dy_stride, drop, d_dx, dx_stride,
                      const_cast<float*>(d_stats), d_work, work_bytes, stream);
}
