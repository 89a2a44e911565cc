// Device helpers and launch declarations shared by the training-node operators:
// dropout (ckm_dropout.hip), layer norm (ckm_layer_norm.hip), the attention softmax
// (ckm_softmax.hip), the matrix operators (ckm_matrix.h) and the norm over many
// tensors (ckm_clip.hip).
//
// A thread loads and stores groups of eight consecutive columns: 16 bytes of a 16-bit
// type, and exactly the eight draws of one Philox output.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "ckm.h"
#include "ckm_internal.h"

// Products and sums are fused where the code says so (fmaf) and nowhere else: an
// operator then gives the same bits in each of its kernels' forms, and one with a
// dropout or a residual inside the bits of the operators one after the other.
#pragma clang fp contract(off)

namespace ckm {

constexpr int kVec = 8;   // columns of a group

// A dropout as the kernels take it: on is false without one, and when every
// element is kept (keep = 65536, factor 1).
struct DropArgs {
  uint32_t k0 = 0, k1 = 0;            // Philox key: the seed
  uint64_t site = 0;                  // counter words 2 and 3, plus *d_site when given
  const uint64_t* d_site = nullptr;
  uint32_t keep = 65536;              // a draw below this keeps the element
  float scale = 1.0f;                 // 65536 / keep
  bool on = false;
};

// Checks a caller's ckm_drop (NULL: no dropout) and converts it.
ckm_status drop_args(const ckm_drop* d, DropArgs* out);
// Checks that a matrix of rows x cols elements of `elt` bytes behind `p` is
// addressable: aligned to its type, row stride (elements) not negative, and at
// least cols for an output of more than one row.
ckm_status check_matrix(const void* p, const char* name, int64_t rows, int64_t cols, int64_t ld, size_t elt,
                        bool output);
inline size_t dtype_bytes(int t) { return t == CKM_F32 ? 4 : 2; }
inline bool dtype_ok(int t) { return t == CKM_F32 || t == CKM_F16 || t == CKM_BF16; }
// CKM_OK, or CKM_E_DEVICE with the launch's error.
ckm_status launched(const char* what);

// ---- device side ----------------------------------------------------------

// A group as it is stored, in whole words: joined and moved as words, it stays in
// the registers it was loaded into, and a load need not be waited for to take it
// apart. Rows of odd length or stride start anywhere: addresses need only be
// aligned to an element, which the hardware's loads and stores take.
template <typename T>
struct Raw8 {
  static constexpr int kWords = kVec * sizeof(T) / 4, kIn = 4 / sizeof(T);   // words, elements in one
  uint32_t w[kWords];
  __device__ __forceinline__ T get(int j) const {
    if constexpr (sizeof(T) == 4)
      return __builtin_bit_cast(T, w[j]);
    else if constexpr (sizeof(T) == 2)
      return __builtin_bit_cast(T, (uint16_t)(w[j / 2] >> (16 * (j % 2))));
    else
      return (T)(w[j / 4] >> (8 * (j % 4)));
  }
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <typename T>
__device__ __forceinline__ Raw8<T> group_of(uint32_t word) {
  Raw8<T> r;
#pragma unroll
  for (int k = 0; k < Raw8<T>::kWords; ++k) r.w[k] = word;
  return r;
}
template <typename T>
__device__ __forceinline__ Raw8<T> zero_group() {
  return group_of<T>(0u);
}
// kCount elements from kFrom on.
template <typename T, int kFrom, int kCount>
__device__ __forceinline__ void load_piece(Raw8<T>& r, const T* p) {
  constexpr int kBytes = kCount * sizeof(T), kAt = kFrom * sizeof(T);
  if constexpr (kBytes >= 4) {
    __builtin_memcpy(&r.w[kAt / 4], p + kFrom, kBytes);
  } else if constexpr (kBytes == 2) {
    uint16_t v;
    __builtin_memcpy(&v, p + kFrom, 2);
    r.w[kAt / 4] |= (uint32_t)v << (kAt % 4 * 8);
  } else {
    r.w[kAt / 4] |= (uint32_t)(uint8_t)p[kFrom] << (kAt % 4 * 8);
  }
}
template <typename T, int kFrom, int kCount>
__device__ __forceinline__ void store_piece(T* p, const Raw8<T>& r) {
  constexpr int kBytes = kCount * sizeof(T), kAt = kFrom * sizeof(T);
  if constexpr (kBytes >= 4) {
    __builtin_memcpy(p + kFrom, &r.w[kAt / 4], kBytes);
  } else {
    const uint16_t v = (uint16_t)(r.w[kAt / 4] >> (kAt % 4 * 8));
    __builtin_memcpy(p + kFrom, &v, 2);
  }
}
// Calls f(from, count) for the pieces of four, two and one elements of n < 8.
template <typename F>
__device__ __forceinline__ void pieces(int n, F&& f) {
  using std::integral_constant;
  if (n & 4) {
    f(integral_constant<int, 0>{}, integral_constant<int, 4>{});
    if (n & 2) {
      f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
      if (n & 1) f(integral_constant<int, 6>{}, integral_constant<int, 1>{});
    } else if (n & 1) {
      f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    }
  } else if (n & 2) {
    f(integral_constant<int, 0>{}, integral_constant<int, 2>{});
    if (n & 1) f(integral_constant<int, 2>{}, integral_constant<int, 1>{});
  } else if (n & 1) {
    f(integral_constant<int, 0>{}, integral_constant<int, 1>{});
  }
}
// Column `col` on of a row of `cols` columns: one load for a whole group. In rows
// that are not of whole groups (kEven false) the last one is loaded where it ends
// with the row, and fix_tail moves its elements into place, after the loads that
// a kernel wants in flight together. Rows of fewer than eight go by pieces.
template <bool kEven, typename T>
__device__ __forceinline__ Raw8<T> load_cols(const T* row, int col, int cols) {
  if constexpr (kEven) {
    return load8(row + col);
  } else {
    if (cols >= kVec) return load8(row + min(col, cols - kVec));
    Raw8<T> r = zero_group<T>();
    pieces(cols, [&](auto from, auto count) { load_piece<T, decltype(from)::value, decltype(count)::value>(r, row); });
    return r;
  }
}
template <bool kEven, typename T>
__device__ __forceinline__ void fix_tail(Raw8<T>& r, int col, int cols) {
  if constexpr (!kEven) {
    if (cols >= kVec && col + kVec > cols) {
      constexpr int kWords = Raw8<T>::kWords, kIn = Raw8<T>::kIn;
      const int by = kVec - cols % kVec;   // elements to move down, the same for every such group
      const auto down = [&](int n) {       // by n words
#pragma unroll
        for (int k = 0; k < kWords; ++k) r.w[k] = k + n < kWords ? r.w[k + n] : 0u;
      };
      if (by & 4) down(4 / kIn);
      if constexpr (kIn <= 2)
        if (by & 2) down(2 / kIn);
      if constexpr (kIn == 1) {
        if (by & 1) down(1);
      } else {
        const uint32_t bits = by % kIn * (32 / kIn);
#pragma unroll
        for (int k = 0; k < kWords; ++k)
          r.w[k] = __builtin_amdgcn_alignbit(k + 1 < kWords ? r.w[k + 1] : 0u, r.w[k], bits);
      }
    }
  }
}
// Stores a group at column `col` of a row, the last one of a row that is not of
// whole groups in pieces.
template <bool kEven, typename T>
__device__ __forceinline__ void store_part(T* row, const Raw8<T>& r, int col, int cols) {
  T* p = row + col;
  if (kEven || col + kVec <= cols) {
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
    pieces(cols % kVec,
           [&](auto from, auto count) { store_piece<T, decltype(from)::value, decltype(count)::value>(p, r); });
  }
}
// The first `left` elements of eight in memory, 1 or more; zeros past them.
template <typename T>
__device__ __forceinline__ Raw8<T> load_left(const T* p, int left) {
  if (left >= kVec) return load8(p);
  Raw8<T> r = zero_group<T>();
  pieces(left, [&](auto from, auto count) { load_piece<T, decltype(from)::value, decltype(count)::value>(r, p); });
  return r;
}
// Puts `value` in the place of a group's elements past the first `left`.
template <typename T>
__device__ __forceinline__ void hide(Raw8<T>& r, int left, T value) {
  if (left >= kVec) return;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) r.w[j] = j < left ? r.w[j] : __builtin_bit_cast(uint32_t, value);
  } else {
    const uint32_t v = __builtin_bit_cast(uint16_t, value) * 0x10001u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t keep = left >= 2 * k + 2 ? ~0u : left > 2 * k ? 0xFFFFu : 0u;
      r.w[k] = (r.w[k] & keep) | (v & ~keep);
    }
  }
}
// v rounded to T, nearest even. For binary16 the empty statement keeps the compiler
// from fusing the conversion with a product before it, which rounds once and not
// twice: it does that for some elements of a kernel and not for others.
template <typename T>
__device__ __forceinline__ T rounded(float v) {
  if constexpr (std::is_same<T, _Float16>::value) asm("" : "+v"(v));
  return (T)v;
}
template <typename T>
__device__ __forceinline__ Raw8<T> rounded8(const float (&v)[kVec]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 2) {   // two at a time
    typedef float Two __attribute__((ext_vector_type(2)));
    typedef T Half2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float lo = v[2 * k], hi = v[2 * k + 1];
      if constexpr (std::is_same<T, _Float16>::value) asm("" : "+v"(lo), "+v"(hi));   // as in rounded()
      r.w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((Two{lo, hi}), Half2));
    }
  } else {
#pragma unroll
    for (int j = 0; j < kVec; ++j) r.w[j] = __float_as_uint(v[j]);
  }
  return r;
}

// Philox4x32-10 (Salmon et al., SC'11) of counter (group, row, site), the
// generator and draw order of the rounding: draw j is 16-bit half (j mod 2)
// of word j / 2.
struct DropSite {
  uint32_t s0, s1;
};
__device__ __forceinline__ DropSite drop_site(const DropArgs& d) {
  uint64_t s = d.site;
  if (d.d_site) s += *d.d_site;
  return {(uint32_t)s, (uint32_t)(s >> 32)};
}
__device__ __forceinline__ uint32_t drop_xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);   // truth table of a ^ b ^ c
}
// The group's eight draws, two to a word, low half first.
__device__ __forceinline__ void draws8(uint32_t (&x)[4], const DropArgs& d, DropSite s, uint32_t group, uint32_t row) {
  uint32_t c0 = group, c1 = row, c2 = s.s0, c3 = s.s1, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0;
    const uint64_t p1 = (uint64_t)0xCD9E8D57u * c2;
    const uint32_t n0 = drop_xor3((uint32_t)(p1 >> 32), c1, k0);
    const uint32_t n2 = drop_xor3((uint32_t)(p0 >> 32), c3, k1);
    c0 = n0;
    c1 = (uint32_t)p1;
    c2 = n2;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  x[0] = c0;
  x[1] = c1;
  x[2] = c2;
  x[3] = c3;
}
// All ones in the halves whose draw is below keep (keep < 65536), by saturating
// differences of the two 16-bit halves at once: no lane masks, whose use right
// after a comparison stalls.
__device__ __forceinline__ uint32_t kept_halves(uint32_t draws, uint32_t keep) {
  typedef uint16_t Half2 __attribute__((ext_vector_type(2)));
  const Half2 k = {(uint16_t)keep, (uint16_t)keep}, one = {1, 1};
  const Half2 below = __builtin_elementwise_min(__builtin_elementwise_sub_sat(k, __builtin_bit_cast(Half2, draws)), one);
  return __builtin_bit_cast(uint32_t, (Half2)-below);
}
// Applies the dropout's choice to a group as it is stored, before or after the
// factor: dropped elements become 0 whatever they hold, NaN and infinities too.
template <typename T>
__device__ __forceinline__ void drop_choice(Raw8<T>& r, const DropArgs& d, DropSite s, uint32_t group, uint32_t row) {
  uint32_t x[4];
  draws8(x, d, s, group, row);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r.w[k] &= kept_halves(x[k], d.keep);
  } else {
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      r.w[j] = ((j & 1) ? x[j >> 1] >> 16 : x[j >> 1] & 0xFFFFu) < d.keep ? r.w[j] : 0u;
  }
}
// D of eight values, rounded to T.
template <typename T>
__device__ __forceinline__ Raw8<T> dropped8(const float (&v)[kVec], const DropArgs& d, DropSite s, uint32_t group,
                                            uint32_t row) {
  float o[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) o[j] = v[j] * d.scale;
  Raw8<T> r = rounded8<T>(o);
  if (d.on) drop_choice(r, d, s, group, row);
  return r;
}

// The row of a block's rows that this thread works on: the same for a whole wave
// where a row has 64 threads or more, and then in a scalar register.
template <int kLanes>
__device__ __forceinline__ int row_in_block() {
  if constexpr (kLanes >= 64)
    return __builtin_amdgcn_readfirstlane(threadIdx.x) / kLanes;
  else
    return threadIdx.x / kLanes;
}

// Sums and maxima over the kLanes threads of a row. Within 16 lanes by lane
// permutations, over a wave by reading its four 16-lane rows, over more waves
// through LDS. Every thread of the row gets the result, by one order of
// additions that depends on kLanes alone.
template <int kCtrl>
__device__ __forceinline__ float dpp_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true));
}
struct OpSum {
  __device__ __forceinline__ static float of(float a, float b) { return a + b; }
};
struct OpMax {
  __device__ __forceinline__ static float of(float a, float b) { return fmaxf(a, b); }
};
template <typename Op>
__device__ __forceinline__ float reduce16(float x) {
  x = Op::of(x, dpp_move<0xB1>(x));    // lanes xor 1
  x = Op::of(x, dpp_move<0x4E>(x));    // lanes xor 2
  x = Op::of(x, dpp_move<0x141>(x));   // the other four of eight
  x = Op::of(x, dpp_move<0x140>(x));   // the other eight of sixteen
  return x;
}
template <typename Op>
__device__ __forceinline__ float reduce32(float x) {
  x = reduce16<Op>(x);
  // both of the pair's rows of 16 lanes, in every lane of the two
  const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return Op::of(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
__device__ __forceinline__ float lane_of(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
template <typename Op>
__device__ __forceinline__ float reduce64(float x) {
  x = reduce16<Op>(x);
  return Op::of(Op::of(lane_of(x, 0), lane_of(x, 16)), Op::of(lane_of(x, 32), lane_of(x, 48)));
}
// Over kWaves (a power of two up to 16) values in LDS, `step` apart: each lane
// reads one.
template <typename Op, int kWaves>
__device__ __forceinline__ float reduce_waves(const float* at, int step) {
  float x = at[(threadIdx.x % kWaves) * step];
  if constexpr (kWaves > 1) x = Op::of(x, dpp_move<0xB1>(x));
  if constexpr (kWaves > 2) x = Op::of(x, dpp_move<0x4E>(x));
  if constexpr (kWaves > 4) x = Op::of(x, dpp_move<0x141>(x));
  if constexpr (kWaves > 8) x = Op::of(x, dpp_move<0x140>(x));
  return lane_of(x, 0);
}
// kCount values at once, one barrier. kLanes 16, 32, 64, or a power of two of waves
// that divides the block's kBlock threads. lds: 2 kCount kBlock / 64 floats; `turn`
// (0 or 1) picks the half, and a kernel's reductions take turns: a wave can write a
// half again only after the barrier of the reduction between, which every reader of
// it has reached. All threads of the block take part.
template <typename Op, int kLanes, int kBlock, int kCount>
__device__ __forceinline__ void reduce_rows(float (&v)[kCount], float* lds, int turn) {
#pragma unroll
  for (int k = 0; k < kCount; ++k)
    v[k] = kLanes == 16 ? reduce16<Op>(v[k]) : kLanes == 32 ? reduce32<Op>(v[k]) : reduce64<Op>(v[k]);
  if constexpr (kLanes > 64) {
    constexpr int kWaves = kLanes / 64;
    float* at = lds + turn * (kCount * kBlock / 64);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < kCount; ++k) at[kCount * (threadIdx.x >> 6) + k] = v[k];
    }
    __syncthreads();
    at += row_in_block<kLanes>() * (kCount * kWaves);
#pragma unroll
    for (int k = 0; k < kCount; ++k) v[k] = reduce_waves<Op, kWaves>(at + k, kCount);
  }
}
template <typename Op, int kLanes, int kBlock>
__device__ __forceinline__ float reduce_row(float x, float* lds, int turn) {
  float v[1] = {x};
  reduce_rows<Op, kLanes, kBlock>(v, lds, turn);
  return v[0];
}

}  // namespace ckm
