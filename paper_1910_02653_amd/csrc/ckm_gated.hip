// Gated feed-forward: h = act(x Wg) (x Wu), both projections, the activation and the
// product in one kernel, and its gradient.
//
//   forward   g = x Wg, u = x Wu (binary32, in registers), h = act(g) u
//   gradient  g and u again, dg = dh u act'(g), du = dh act(g), dx = dg Wg' + du Wu',
//             dWg = x' dg, dWu = x' du
//
// A tile of the forward product has as many columns of Wg as of Wu, the same ones,
// and a wave holds both of an element. The gradient writes dg and du, side by side in
// a row and rounded to the tensors' type, which the products after it multiply (a
// rounding more than the formulas': one part in 2^9 of each term in bfloat16,
// independent of one another); dx is one product over both, dWg and dWu one launch,
// and where there are few tiles all three.
//
// binary16's range may be too small for dg and du where dx and dW are well inside it: they
// are products of two factors, and dW sums many rows. Each block leaves the largest finite
// |dg|, |du| it has seen; a second launch takes the largest of all and, if it is past the
// range or below 2^-6 (elements less than 2^-8 of it have begun to lose digits), computes
// dg and du again times the power of two that brings it between 2^14 and 2^15. The results
// are multiplied by the inverse. In range, which is the rule, its blocks return at once: f16
// 2048x2048x8192 408 us without it and 412 with it, 512x1024x2048 33 and 36; out of range 553 and 45.
//
// Bound by the products: f16 2048x2048x8192 119 us (1150 TFLOP/s; the library's product
// alone 117 to 137), its gradient 398 (the least of a trace: recomputation 136 and 5 for the
// second launch, dx 135 and 13 for its shares, dW 123); bf16 8192x4096x16384 1610 to 1650 us
// (1330 to 1370); f32 2048x1024x4096 256 us and 758, 134 to 136 of 154 TFLOP/s. A tile's end,
// activation and stores, is 6 to 10 us of some 58 and not hidden: one block is on a CU. A
// single token is bound by reading the weights: f16 1x2048x8192 14.7 us, 67 MB; f32 27.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "ckm_matrix.h"

namespace ckm {
namespace {

enum { kForward, kBackward, kAgain, kShares };   // what a kernel makes of g and u; again: dg and du times a power of two
template <typename T>
constexpr bool kHeld = std::is_same<T, _Float16>::value;   // dg and du times a power of two where they need it

struct GatedArgs {
  ProductArgs p;
  int32_t act;
  int32_t tiles_m, tiles_n, steps;
  const void* dh;
  int64_t ld_dh;
  void* out;         // h, or dg | du
  int64_t ld_out;
  int32_t up;        // where du begins in a row of dg | du
  float* slab;       // [split][g, u][m][ld_slab]
  int64_t ld_slab;
  float* most;       // kHeld: the blocks' largest |dg|, |du|,
  int32_t mosts;     // so many,
  float* alpha;      // and one over the power of two that dg and du are held times
};

// The exponent of the power of two for a largest value.
__device__ __forceinline__ int held_by(float most) {
  if (most == 0.0f || (most >= 0x1p-6f && most <= 65504.0f)) return 0;
  return max(-126, min(126, 14 - ((int)(__float_as_uint(most) >> 23) - 127)));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// The largest of a block's threads' values, for the block; lds: its threads have passed their last use of it.
template <int kThreads>
__device__ __forceinline__ void leave_most(const GatedArgs& a, float most, float* lds) {
  most = reduce_row<OpMax, kThreads, kThreads>(most, lds, 0);
  if (threadIdx.x == 0) a.most[blockIdx.x] = most;
}
// The power of two for all blocks' values, 1 if dg and du are as they have to be.
template <int kThreads>
__device__ __forceinline__ float held_times(const GatedArgs& a, float* lds) {
  float most = 0.0f;
  for (int k = threadIdx.x; k < a.mosts; k += kThreads) most = fmaxf(most, a.most[k]);
  const int e = held_by(reduce_row<OpMax, kThreads, kThreads>(most, lds, 0));
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.alpha = power_of_two(-e);
  return power_of_two(__builtin_amdgcn_readfirstlane(e));
}

// act(z) and its derivative. The normal distribution's lower side is e^(-z^2 / 2) t q(t),
// t = 1 / (1 + 0.44 |z| / sqrt 2), q a polynomial fitted to erfc(x) e^(x^2) / 2: no
// difference of numbers near 1 (half of 1 + erf(z / sqrt 2) in binary32 is off by 3e-4 at
// -4, by 4 % at -5, and 0 from -6 on). For 16-bit results, whose rounding is far above: the
// logistic function by the hardware's 2^x and 1 / x (some 2^-21), and q of degree 7
// (2.3e-7, in binary32's arithmetic 4.3e-7; at z = -12.6 the exponential's rounded argument
// adds 7e-6). For binary32: degree 9 (1e-8), and the exponential corrected by the rounding
// of z^2: within 10 units of 2^-24 of the value down to z = -12.9, where it is subnormal.
template <typename T>
__device__ __forceinline__ void activation(int act, float z, float& a, float& da) {
  constexpr bool kFull = std::is_same<T, float>::value;
  if (act == CKM_ACT_SILU) {
    const float s = kFull ? 1.0f / (1.0f + expf(-z))
                          : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
    a = z * s;
    da = s * (1.0f + z * (1.0f - s));
  } else if (act == CKM_ACT_GELU) {
    float c, e;
    if constexpr (kFull) {
      const float y = fminf(fabsf(z), 16.0f);   // past it e is 0
      const float d = fmaf(0.31112698f, y, 1.0f), r = __builtin_amdgcn_rcpf(d), t = fmaf(r, fmaf(-d, r, 1.0f), r);
      const float y2 = y * y;
      e = expf(-0.5f * y2);
      e = fmaf(e, -0.5f * fmaf(y, y, -y2), e);
      float q = -0.0194131676f;
      q = fmaf(q, t, 0.0947795957f);
      q = fmaf(q, t, -0.161439314f);
      q = fmaf(q, t, 0.0886825845f);
      q = fmaf(q, t, -0.0116111515f);
      q = fmaf(q, t, 0.0601861700f);
      q = fmaf(q, t, 0.0888089538f);
      q = fmaf(q, t, 0.111705750f);
      q = fmaf(q, t, 0.124182113f);
      q = fmaf(q, t, 0.124118462f);
      c = q * t * e;
      c = z < 0.0f ? c : 1.0f - c;
    } else {
      const float t = __builtin_amdgcn_rcpf(fmaf(0.31112698f, fabsf(z), 1.0f));
      e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
      float q = 0.035749969f;
      q = fmaf(q, t, -0.13957664f);
      q = fmaf(q, t, 0.14943397f);
      q = fmaf(q, t, -0.011147469f);
      q = fmaf(q, t, 0.10849696f);
      q = fmaf(q, t, 0.10846730f);
      q = fmaf(q, t, 0.12446772f);
      q = fmaf(q, t, 0.12410826f);
      c = q * t * e;
      c = z < 0.0f ? c : 1.0f - c;
    }
    a = z * c;
    da = c + z * (0.39894228f * e);
  } else {
    a = z > 0.0f ? z : z != z ? z : 0.0f;
    da = z > 0.0f ? 1.0f : z != z ? z : 0.0f;
  }
}

template <typename T, int kCount>
__device__ __forceinline__ void gated_of(int act, float (&g)[kCount], const float (&u)[kCount]) {   // h in g's place
#pragma unroll
  for (int k = 0; k < kCount; ++k) {
    float a, da;
    activation<T>(act, g[k], a, da);
    g[k] = a * u[k];
  }
}
template <typename T, int kCount>
__device__ __forceinline__ void gated_back_of(int act, const Raw8<T>& dh, float (&g)[kCount], float (&u)[kCount]) {   // dg, du
#pragma unroll
  for (int k = 0; k < kCount; ++k) {
    float a, da;
    activation<T>(act, g[k], a, da);
    const float d = (float)dh.get(k);
    g[k] = d * u[k] * da;
    u[k] = d * a;
  }
}

// What becomes of eight columns of g and u. held: the largest finite |dg|, |du| so far, or (again) what they are
// multiplied by.
template <typename T, int kMode>
__device__ __forceinline__ void finish(const GatedArgs& a, int64_t m, int n, float (&g)[8], float (&u)[8], float& held) {
  if constexpr (kMode == kForward) {
    if (n >= a.p.n) return;
    gated_of<T>(a.act, g, u);
    store_part<false>((T*)a.out + m * a.ld_out, rounded8<T>(g), n, a.p.n);
  } else {   // zeros to the end of dg's last group
    if (n >= a.up) return;
    const int left = a.p.n - n;
    gated_back_of<T>(a.act, load_left((const T*)a.dh + m * a.ld_dh + n, left), g, u);
    if constexpr (kMode == kAgain) {
#pragma unroll
      for (int k = 0; k < 8; ++k) g[k] *= held, u[k] *= held;
    } else if constexpr (kHeld<T>) {
      float most = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(fmaxf(most, fabsf(g[k])), fabsf(u[k]));   // a NaN counts for nothing
      if (most == INFINITY) {
        most = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (fabsf(g[k]) < INFINITY) most = fmaxf(most, fabsf(g[k]));
          if (fabsf(u[k]) < INFINITY) most = fmaxf(most, fabsf(u[k]));
        }
      }
      held = fmaxf(held, most);
    }
    T* row = (T*)a.out + m * a.ld_out;
    store_part<false>(row, rounded8<T>(g), n, a.up);
    store_part<false>(row + a.up, rounded8<T>(u), n, a.up);
  }
}

template <class P, int kMode>
__device__ __forceinline__ void gated_tile(const GatedArgs& a, int block, int thread, char* lds, float& held) {
  using T = typename P::T;
  const P p(thread);
  const int tiles = a.tiles_m * a.tiles_n, split = block / tiles;
  int tm, tn;
  tile_of(block % tiles, a.tiles_m, a.tiles_n, tm, tn);
  const int all = (a.p.k + P::kStep - 1) / P::kStep, from = split * a.steps;
  F4 acc[P::kFN][P::kFM];
  p.run(acc, a.p, tm * P::kM, tn * P::kSubN, from, min(all, from + a.steps), (LdsChar*)lds);
  if constexpr (kMode == kForward) {   // half as much goes through LDS
#pragma unroll
    for (int j = 0; j < P::kFS; ++j)
#pragma unroll
      for (int i = 0; i < P::kFM; ++i) {
        float g[4], u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = acc[j][i][k], u[k] = acc[j + P::kFS][i][k];
        gated_of<T>(a.act, g, u);
        acc[j][i] = F4{g[0], g[1], g[2], g[3]};
      }
    p.template each8<1>(acc, (LdsChar*)lds, [&](int row, int col, float (&v)[1][8]) {
      const int m = tm * P::kM + row, n = tn * P::kSubN + col;
      if (m < a.p.m && n < a.p.n) store_part<false>((T*)a.out + m * a.ld_out, rounded8<T>(v[0]), n, a.p.n);
    });
  } else {
    p.template each8<2>(acc, (LdsChar*)lds, [&](int row, int col, float (&v)[2][8]) {
      const int m = tm * P::kM + row, n = tn * P::kSubN + col;
      if (m >= a.p.m) return;
      if constexpr (kMode == kBackward || kMode == kAgain) {
        finish<T, kMode>(a, m, n, v[0], v[1], held);
      } else if (n < a.p.n) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          F4* at = (F4*)(a.slab + (((int64_t)split * 2 + s) * a.p.m + m) * a.ld_slab + n);
          at[0] = F4{v[s][0], v[s][1], v[s][2], v[s][3]};
          at[1] = F4{v[s][4], v[s][5], v[s][6], v[s][7]};
        }
      }
    });
  }
}

template <class P, int kMode>
__global__ void __launch_bounds__(P::kThreads, P::kWaveSlots) ckm_gated_kernel(GatedArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
  float held = 0.0f;
  gated_tile<P, kMode>(a, blockIdx.x, threadIdx.x, lds, held);
  if constexpr (kMode == kBackward && kHeld<typename P::T>) {
    __syncthreads();
    leave_most<P::kThreads>(a, held, (float*)lds);
  }
}
// dg and du again, where the first time's do not fit: a block takes several tiles.
template <class P>
__global__ void __launch_bounds__(P::kThreads, P::kWaveSlots) ckm_gated_again_kernel(GatedArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
  float held = held_times<P::kThreads>(a, (float*)lds);
  if (held == 1.0f) return;
  for (int block = blockIdx.x; block < a.tiles_m * a.tiles_n; block += gridDim.x) {
    __syncthreads();   // the tile before has been read from lds
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));   // a lane's places are worked out for each tile: kept over the loop they take registers that are not there
    gated_tile<P, kAgain>(a, block, thread, lds, held);
  }
}

// The shares of g and u added in their order, and what kMode makes of them; a thread
// eight columns.
template <typename T, int kMode>
__global__ void __launch_bounds__(256) ckm_gated_join_kernel(GatedArgs a, int splits, int64_t total, uint32_t eights) {
  const int64_t one = (int64_t)a.p.m * a.ld_slab;
  constexpr bool kLeaves = kMode == kBackward && kHeld<T>;
  __shared__ float lds[kLeaves || kMode == kAgain ? 8 : 1];
  float held = 0.0f;
  if constexpr (kMode == kAgain) {
    held = held_times<256>(a, lds);
    if (held == 1.0f) return;
  }
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
    const int64_t m = at / eights;
    const int n = (int)(at - m * eights) * 8;
    float v[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float* p = a.slab + s * one + m * a.ld_slab + n;
      F4 x = ((const F4*)p)[0], y = ((const F4*)p)[1];
#pragma unroll 8
      for (int k = 1; k < splits; ++k) {
        x += ((const F4*)(p + 2 * k * one))[0];
        y += ((const F4*)(p + 2 * k * one))[1];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) v[s][k] = x[k], v[s][k + 4] = y[k];
    }
    finish<T, kMode>(a, m, n, v[0], v[1], held);
  }
  if constexpr (kLeaves) leave_most<256>(a, held, lds);
}

// Blocks of the join of shares.
int64_t join_blocks(int64_t m, int64_t n) { return std::min<int64_t>((m * ((n + 7) / 8) + 255) / 256, 1 << 16); }
// The blocks that leave a largest |dg|, |du|.
int64_t leaving(const Cut& cut, int64_t m, int64_t n) { return cut.splits > 1 ? join_blocks(m, n) : cut.blocks(); }

template <typename T, int kMode>
void launch_both(GatedArgs a, const Cut& cut, hipStream_t s) {
  a.tiles_m = cut.tiles_m;
  a.tiles_n = cut.tiles_n;
  a.steps = cut.steps;
  with_shape<T, true, false, 2>(cut, [&](auto p) {
    using P = typename decltype(p)::Shape;
    const uint32_t blocks = (uint32_t)cut.blocks();
    if (cut.splits > 1) {
      ckm_gated_kernel<P, kShares><<<blocks, P::kThreads, 0, s>>>(a);
      return;
    }
    ckm_gated_kernel<P, kMode><<<blocks, P::kThreads, 0, s>>>(a);
    if constexpr (kMode == kBackward && kHeld<T>)
      ckm_gated_again_kernel<P><<<std::min(blocks, 256u * P::kBlocks), P::kThreads, 0, s>>>(a);
  });
  if (cut.splits > 1) {
    const uint32_t eights = (uint32_t)((a.p.n + 7) / 8), blocks = (uint32_t)join_blocks(a.p.m, a.p.n);
    const int64_t total = a.p.m * (int64_t)eights;
    ckm_gated_join_kernel<T, kMode><<<blocks, 256, 0, s>>>(a, cut.splits, total, eights);
    if constexpr (kMode == kBackward && kHeld<T>)
      ckm_gated_join_kernel<T, kAgain><<<std::min(blocks, 1024u), 256, 0, s>>>(a, cut.splits, total, eights);
  }
}

// Where a call's parts lie in its work buffer.
struct GatedPlan {
  bool pack_x, pack_w;
  int64_t ld_x, ld_w;        // of the operands as multiplied
  int64_t inner, ld_d;       // columns of dg, padded to whole groups; a row of dg | du
  Cut both, dx, dw;
  bool together;             // dx and the weights' gradients in a launch
  size_t x, w, d, most, alpha, slab, total;
  double time;               // the model's, us
};

// packed: operands that cannot be loaded as they are are copied, or else staged. The cuts of
// k are those of operands that can be loaded, in either form.
GatedPlan plan_as(int type, const ckm_gated& c, bool back, bool ragged_x, bool ragged_w, bool packed) {
  const size_t elt = dtype_bytes(type);
  const int64_t group = 16 / elt, step = kStepBytes / elt;
  GatedPlan p = {};
  p.pack_x = ragged_x && packed;
  p.pack_w = ragged_w && packed;
  p.inner = whole(c.inner, group);
  p.ld_d = row_of(2 * p.inner, elt);
  p.ld_x = p.pack_x || c.rows == 1 ? whole(c.hidden, group) : c.ld_x;   // a single row may have any stride
  p.ld_w = p.pack_w || c.hidden == 1 ? p.inner : c.ld_gate;
  const int64_t steps_h = (c.hidden + step - 1) / step, steps_f = (c.inner + step - 1) / step;
  const int64_t x_bytes = c.rows * c.hidden * elt, w_bytes = 2 * c.hidden * c.inner * elt, h_bytes = c.rows * c.inner * elt;
  const bool staged_x = ragged_x && !packed, staged_w = ragged_w && !packed;
  p.both = cut_product(type, c.rows, c.inner, 1, 2, steps_h, x_bytes + w_bytes, true, true);
  if (staged_x || staged_w)
    p.both = cut_like(type, c.rows, c.inner, 1, 2, steps_h, x_bytes + w_bytes, true,
                      staged_w ? kStagedAcross : kStagedAlong, p.both);
  p.time = p.both.time + (p.pack_x || p.pack_w ? copy_time((p.pack_x ? x_bytes : 0) + (p.pack_w ? w_bytes : 0)) : 0.0);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at = whole(at + bytes, 256);
    return here;
  };
  if (p.pack_x) p.x = take(c.rows * p.ld_x * elt);
  if (p.pack_w) p.w = take(2 * c.hidden * p.ld_w * elt);
  size_t slab = p.both.splits > 1 ? (size_t)p.both.splits * 2 * c.rows * whole(c.inner, 8) * 4 : 0;
  if (back) {
    const int64_t steps_m = (c.rows + step - 1) / step, dx_bytes = 2 * h_bytes + w_bytes, dw_bytes = dx_bytes + x_bytes;
    p.dx = cut_product(type, c.rows, c.hidden, 1, 1, 2 * steps_f, dx_bytes, true, true);
    p.dw = cut_product(type, c.hidden, c.inner, 2, 1, steps_m, dw_bytes, true, false);
    p.together = cut_together(type, p.dx, c.rows, c.hidden, 2 * steps_f, p.dw, c.hidden, c.inner, steps_m,
                              dw_bytes + w_bytes);
    if (staged_x || staged_w) {
      p.together = false;
      p.dx = cut_like(type, c.rows, c.hidden, 1, 1, 2 * steps_f, dx_bytes, true, staged_w ? kStagedAlong : kStraight, p.dx);
      p.dw = cut_like(type, c.hidden, c.inner, 2, 1, steps_m, dw_bytes, false, staged_x ? kStagedAcross : kStraight, p.dw);
    }
    p.time += p.dx.time + p.dw.time;
    p.d = take(c.rows * p.ld_d * elt);
    if (type == CKM_F16) {
      p.most = take(leaving(p.both, c.rows, c.inner) * sizeof(float));
      p.alpha = take(sizeof(float));
    }
    if (p.dx.splits > 1) slab = std::max(slab, (size_t)p.dx.splits * c.rows * whole(c.hidden, 8) * 4);
    if (p.dw.splits > 1) slab = std::max(slab, (size_t)p.dw.splits * 2 * c.hidden * whole(c.inner, 8) * 4);
  }
  p.slab = take(slab);
  p.total = at;
  return p;
}

GatedPlan plan_of(int type, const ckm_gated& c, bool back) {
  const size_t elt = dtype_bytes(type);
  const bool x = !loadable(c.d_x, c.rows, c.hidden, c.ld_x, elt, true);
  const bool w = c.ld_gate != c.ld_up || !loadable(c.d_gate, c.hidden, c.inner, c.ld_gate, elt, back) ||
                 !loadable(c.d_up, c.hidden, c.inner, c.ld_up, elt, back);
  const GatedPlan p = plan_as(type, c, back, x, w, true);
  if ((!x && !w) || (c.ld_gate != c.ld_up && c.hidden > 1) || !stageable(c.rows, c.ld_x, elt) ||
      !stageable(c.hidden, c.ld_gate, elt))
    return p;
  const GatedPlan q = plan_as(type, c, back, x, w, false);
  return q.time < p.time ? q : p;
}

template <typename T>
void launch_gated(int type, const ckm_gated& c, const GatedPlan& plan, const void* dh, int64_t ld_dh, void* out,
                  int64_t ld_out, void* dgate, int64_t ld_dgate, void* dup, int64_t ld_dup, char* work, hipStream_t s) {
  const bool back = dh != nullptr;
  const void *x = c.d_x, *wg = c.d_gate, *wu = c.d_up;
  PackArgs packs = {};
  if (plan.pack_x) {
    packs.add(x, c.rows, c.hidden, c.ld_x, work + plan.x, plan.ld_x);
    x = work + plan.x;
  }
  if (plan.pack_w) {
    T* to = (T*)(work + plan.w);
    packs.add(wg, c.hidden, c.inner, c.ld_gate, to, plan.ld_w);
    packs.add(wu, c.hidden, c.inner, c.ld_up, to + c.hidden * plan.ld_w, plan.ld_w);
    wg = to;
    wu = to + c.hidden * plan.ld_w;
  }
  launch_pack(type, packs, s);
  float* slab = (float*)(work + plan.slab);
  GatedArgs a = {};
  a.p = {{x, x, plan.ld_x}, {wg, wu, plan.ld_w}, (int32_t)c.rows, (int32_t)c.inner, (int32_t)c.hidden, 1};
  a.act = c.act;
  a.dh = dh;
  a.ld_dh = ld_dh;
  a.slab = slab;
  a.ld_slab = whole(c.inner, 8);
  if (!back) {
    a.out = out;
    a.ld_out = ld_out;
    launch_both<T, kForward>(a, plan.both, s);
    return;
  }
  T* d = (T*)(work + plan.d);
  a.out = d;
  a.ld_out = plan.ld_d;
  a.up = (int32_t)plan.inner;
  if (kHeld<T>) {
    a.most = (float*)(work + plan.most);
    a.mosts = (int32_t)leaving(plan.both, c.rows, c.inner);
    a.alpha = (float*)(work + plan.alpha);
  }
  launch_both<T, kBackward>(a, plan.both, s);
  // dx = dg Wg' + du Wu'
  ResultArgs rx = {}, rw = {};
  rx.p = {{d, d + plan.inner, plan.ld_d}, {wg, wu, plan.ld_w}, (int32_t)c.rows, (int32_t)c.hidden, (int32_t)c.inner, 2};
  rx.c[0] = out;
  rx.ld_c[0] = ld_out;
  rx.factor = rw.factor = 1.0f;
  rx.alpha = rw.alpha = a.alpha;
  rx.halves = 1;
  if (plan.dx.splits > 1) rx.slab = slab;
  rx.ld_slab = whole(c.hidden, 8);
  // dWg = x' dg, dWu = x' du
  rw.p = {{x, x, plan.ld_x}, {d, d + plan.inner, plan.ld_d}, (int32_t)c.hidden, (int32_t)c.inner, (int32_t)c.rows, 1};
  rw.c[0] = dgate;
  rw.c[1] = dup;
  rw.ld_c[0] = ld_dgate;
  rw.ld_c[1] = ld_dup;
  rw.halves = 2;
  if (plan.dw.splits > 1) rw.slab = slab;
  rw.ld_slab = whole(c.inner, 8);
  if (plan.together && out && dgate) {
    launch_two<T, true>(rx, plan.dx, rw, plan.dw, s);
  } else if (out) {
    launch_product<T, true, true>(rx, plan.dx, s);
  }
  if (out && plan.dx.splits > 1) launch_join(type, rx, plan.dx.splits, s);
  if (dgate && !(plan.together && out)) {
    launch_product<T, false, false>(rw, plan.dw, s);
    if (plan.dw.splits > 1) launch_join(type, rw, plan.dw.splits, s);
  }
}

ckm_status check_gated(ckm_dtype type, const ckm_gated* c) {
  if (!dtype_ok(type)) return set_error(CKM_E_INVALID_ARG, "unknown type %d", (int)type);
  if (!c) return set_error(CKM_E_INVALID_ARG, "gated is NULL");
  if (c->rows < 0 || c->hidden < 1 || c->inner < 1)
    return set_error(CKM_E_INVALID_ARG, "gated of %lld rows, %lld x %lld", (long long)c->rows, (long long)c->hidden,
                     (long long)c->inner);
  if (c->rows > CKM_MAX_MATRIX_ROWS || c->hidden > CKM_MAX_MATRIX_COLS || c->inner > CKM_MAX_MATRIX_COLS)
    return set_error(CKM_E_UNSUPPORTED, "gated of %lld rows, %lld x %lld", (long long)c->rows, (long long)c->hidden,
                     (long long)c->inner);
  if (c->act != CKM_ACT_SILU && c->act != CKM_ACT_GELU && c->act != CKM_ACT_RELU)
    return set_error(CKM_E_INVALID_ARG, "unknown activation %d", (int)c->act);
  const size_t elt = dtype_bytes(type);
  ckm_status st;
  if (c->rows && (st = check_matrix(c->d_x, "x", c->rows, c->hidden, c->ld_x, elt, false)) != CKM_OK) return st;
  if ((st = check_matrix(c->d_gate, "w_gate", c->hidden, c->inner, c->ld_gate, elt, false)) != CKM_OK) return st;
  return check_matrix(c->d_up, "w_up", c->hidden, c->inner, c->ld_up, elt, false);
}

ckm_status gated(ckm_dtype type, const ckm_gated* c, bool back, const void* dh, int64_t ld_dh, void* out,
                 int64_t ld_out, void* dgate, int64_t ld_dgate, void* dup, int64_t ld_dup, void* work,
                 size_t work_bytes, void* stream) {
  ckm_status st = check_gated(type, c);
  if (st != CKM_OK) return st;
  const size_t elt = dtype_bytes(type);
  const hipStream_t s = (hipStream_t)stream;
  if (back) {
    if ((dgate == nullptr) != (dup == nullptr))
      return set_error(CKM_E_INVALID_ARG, "one of dw_gate and dw_up is NULL and the other is not");
    if (dgate && (st = check_matrix(dgate, "dw_gate", c->hidden, c->inner, ld_dgate, elt, true)) != CKM_OK) return st;
    if (dup && (st = check_matrix(dup, "dw_up", c->hidden, c->inner, ld_dup, elt, true)) != CKM_OK) return st;
  }
  const Place x = {"x", c->d_x, c->rows, c->hidden, c->ld_x, elt}, wg = {"w_gate", c->d_gate, c->hidden, c->inner, c->ld_gate, elt},
              wu = {"w_up", c->d_up, c->hidden, c->inner, c->ld_up, elt};
  const auto apart = [&] {
    return back ? check_apart({{"dx", out, c->rows, c->hidden, ld_out, elt},
                               {"dw_gate", dgate, c->hidden, c->inner, ld_dgate, elt},
                               {"dw_up", dup, c->hidden, c->inner, ld_dup, elt}},
                              {x, wg, wu, {"dh", dh, c->rows, c->inner, ld_dh, elt}})
                : check_apart({{"h", out, c->rows, c->inner, ld_out, elt}}, {x, wg, wu});
  };
  if (c->rows == 0) {
    if ((st = apart()) != CKM_OK) return st;
    if (dgate) {
      launch_zero(type, dgate, c->hidden, c->inner, ld_dgate, s);
      launch_zero(type, dup, c->hidden, c->inner, ld_dup, s);
      return launched("gated gradient launch");
    }
    return CKM_OK;
  }
  if (back && (st = check_matrix(dh, "dh", c->rows, c->inner, ld_dh, elt, false)) != CKM_OK) return st;
  if ((out || !back) &&
      (st = check_matrix(out, back ? "dx" : "h", c->rows, back ? c->hidden : c->inner, ld_out, elt, true)) != CKM_OK)
    return st;
  if (back && !out && !dgate) return CKM_OK;
  if ((st = apart()) != CKM_OK) return st;
  const GatedPlan plan = plan_of(type, *c, back);
  if ((st = check_blocks(plan.both)) != CKM_OK) return st;
  if (back && ((st = check_blocks(plan.dx)) != CKM_OK || (st = check_blocks(plan.dw)) != CKM_OK)) return st;
  if (plan.total && (!work || work_bytes < plan.total))
    return set_error(CKM_E_INVALID_ARG, "work buffer of %zu bytes, %zu needed", work ? work_bytes : (size_t)0,
                     plan.total);
  if ((uintptr_t)work % 16) return set_error(CKM_E_INVALID_ARG, "work is not aligned to 16 bytes");
  const auto go = [&](auto t) {
    launch_gated<decltype(t)>(type, *c, plan, dh, ld_dh, out, ld_out, dgate, ld_dgate, dup, ld_dup, (char*)work, s);
  };
  switch (type) {
    case CKM_F32: go(0.0f); break;
    case CKM_F16: go((_Float16)0); break;
    default: go((__bf16)0.0f); break;
  }
  return launched(back ? "gated gradient launch" : "gated launch");
}

}  // namespace
}  // namespace ckm

extern "C" ckm_status ckm_gated_workspace_size(ckm_dtype type, const ckm_gated* gated, int32_t backward, size_t* bytes) {
  using namespace ckm;
  if (!bytes) return set_error(CKM_E_INVALID_ARG, "bytes is NULL");
  const ckm_status st = check_gated(type, gated);
  if (st != CKM_OK) return st;
  *bytes = gated->rows ? plan_of(type, *gated, backward != 0).total : 0;
  return CKM_OK;
}

extern "C" ckm_status ckm_gated_async(ckm_dtype type, const ckm_gated* gated, void* d_h, int64_t ld_h, void* d_work,
                                      size_t work_bytes, void* stream) {
  return ckm::gated(type, gated, false, nullptr, 0, d_h, ld_h, nullptr, 0, nullptr, 0, d_work, work_bytes, stream);
}

extern "C" ckm_status ckm_gated_backward_async(ckm_dtype type, const ckm_gated* gated, const void* d_dh, int64_t ld_dh,
                                               void* d_dx, int64_t ld_dx, void* d_dgate, int64_t ld_dgate, void* d_dup,
                                               int64_t ld_dup, void* d_work, size_t work_bytes, void* stream) {
  return ckm::gated(type, gated, true, d_dh, ld_dh, d_dx, ld_dx, d_dgate, ld_dgate, d_dup, ld_dup, d_work, work_bytes,
                    stream);
}
