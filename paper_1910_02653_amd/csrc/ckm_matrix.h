// Tiled matrix products for the operators that multiply: C[m][n] = sum over k of
// A[m][k] B[k][n], of which a block computes a tile kM x kN into registers, in
// binary32, and an operator's kernel makes of it what it needs.
//
// Along k a block goes by steps of 128 bytes (64 elements of 16 bits, 32 of
// binary32). A step's operand tiles are loaded straight into LDS, kStages steps
// ahead; a wave reads its fragments of 16 x 64 bytes from there half a step ahead
// of the matrix instructions that take them. Each step has one barrier: the next
// step's tiles have landed, and every wave has read this step's, whose place the
// loads after it take.
//
// An operand lies along k (rows of m or n, k contiguous) or across it (rows of k, m
// or n contiguous). A fragment across k is read with the transposing LDS load.
// Places past m, n or k read as zeros: the loads' range check sees to rows, a
// comparison to columns.
//
// What bounds it (256 x 256 columns, 8 waves of 128 x 64, two stages of 64 KB; bf16
// 4096x4096x8192 209 us, 1312 TFLOP/s; a large library product reaches 1220 to 1560 by
// layout). A block alone on the card takes 2600 cycles a step, of which the matrix
// instructions are 2048, the loads' issue some 340 (64 of them, each of which holds its wave
// for 20 to 30 cycles), the reads and the barrier 180. With all CUs at work the clock
// falls as the matrix units fill: 1.9 GHz at two thirds. Measured and not taken:
// 32 x 32 matrix instructions (277 instead of 290 us alone, but 1.73 GHz and 246 instead
// of 227 us on the whole card); four waves of 128 x 128 (260 us; with the sums pinned
// to accumulation registers 209 to 230); stages of half a step, four of them (230);
// a third stage of A alone (no difference); a wave priority around the matrix
// instructions, reads earlier or later, the barrier before the last of them (all within
// 3 %); loads at once at the step's begin (232 instead of 209).
#pragma once

#include <initializer_list>

#include "ckm_ops.h"

namespace ckm {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef int I4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char LdsChar;

constexpr int kStepBytes = 128;                    // of k, in one step
constexpr uint32_t kNowhere = 0x80000000u;         // an offset past every range
constexpr int64_t kMaxRowBytes = (int64_t)1 << 22; // a tile's rows then stay within 2^31 bytes

// An operand in memory: up to two matrices of one row stride (parts of k one after
// the other, or of n side by side).
struct Operand {
  const void *p, *q;   // the first, the second
  int64_t ld;          // elements
};

struct ProductArgs {
  Operand a, b;
  int32_t m, n, k;      // of one part
  int32_t parts;        // 1, or 2: k of the first, then k of the second
};

// Whether a matrix of rows of `cols` elements can be loaded straight to LDS: whole
// groups of 16 bytes, and for one along k no group that ends past the row.
inline bool loadable(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t elt, bool along_k) {
  return (uintptr_t)p % 16 == 0 && (rows == 1 || (ld * elt % 16 == 0 && ld >= cols && ld * (int64_t)elt <= kMaxRowBytes)) &&
         (!along_k || cols * elt % 16 == 0);
}

#define CKM_WAIT_LOADS(n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory")

// A tile of kRows rows (or columns) by one step in LDS: kRows x 128 bytes, loaded
// by kWaves waves, 1024 bytes a load. Groups of 16 bytes are permuted within a row of
// the tile so that the lanes of a fragment's read meet in no bank.
template <typename T, int kRows, bool kAlongK, int kWaves>
struct TileLoad {
  static constexpr int kElt = sizeof(T), kStep = kStepBytes / kElt, kGroup = 16 / kElt;
  static constexpr int kBytes = kRows * kStepBytes;
  static constexpr int kRowBytes = kAlongK ? kStepBytes : kRows * kElt;
  static constexpr int kLoads = kBytes / 1024;
  static constexpr int kPer = (kLoads + kWaves - 1) / kWaves;   // of a wave; a few are made twice where waves are many
  static_assert(kRowBytes <= 1024 && kBytes % 1024 == 0, "rows of a tile in one load");
  static_assert(kAlongK || kRowBytes >= 128, "");

  uint32_t off[kPer];
  uint32_t kpos;   // along k: the first element's k within the step

  // The permutation of row r across k, in groups.
  __device__ __forceinline__ static int turned(int r) {
    if constexpr (sizeof(T) == 4) return 4 * ((r >> 2) & 3) & (kRowBytes / 16 - 1);
    else if constexpr (kRowBytes >= 256) return 2 * ((r & 3) | ((r >> 3) & 1) << 2);
    else return 2 * (((r >> 1) & 1) | ((r >> 3) & 1) << 1);
  }

  __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int valid) {
#pragma unroll
    for (int t = 0; t < kPer; ++t) {
      const int at = (wave * kPer + t) % kLoads * 1024 + lane * 16;
      const int row = at / kRowBytes, slot = at % kRowBytes / 16;
      const int group = kAlongK ? slot ^ (row & 7) : slot ^ turned(row);
      off[t] = (uint32_t)(row * (uint32_t)(ld * kElt) + group * 16);
      if constexpr (kAlongK) kpos = group * kGroup;   // the same for every t
      else if (group * kGroup >= valid) off[t] = kNowhere;
    }
  }

  // The loads of one step: `base` the tile's first element, `valid` rows (along k) or
  // columns of the tile that are there, `left` the k that are left.
  struct Step {
    I4 rsrc;        // of a buffer that ends where the tile does: what is loaded past it is zero
    int left;
    uint32_t lds;   // where to
  };
  __device__ __forceinline__ Step step(const char* base, int64_t ld, int valid, int left, uint32_t lds) const {
    const int64_t row = ld * kElt;
    const int have = min(left, kStep);
    // whole groups along k (what follows the row's end in its last one is zero or not there); across k whole words
    const int64_t range = have <= 0 ? 0 : kAlongK ? (min(valid, kRows) - 1) * row + ((have * kElt + 15) & ~15)
                                                  : (have - 1) * row + ((min(valid, kRows) * kElt + 3) & ~3);
    return {{__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)base),
             __builtin_amdgcn_readfirstlane((int)(uint32_t)((uintptr_t)base >> 32)),
             __builtin_amdgcn_readfirstlane((int)range), 0x00020000},
            left, lds};
  }
  // Load t of a wave's kPer. The compiler does not know of it: the product waits by count.
  __device__ __forceinline__ void load(const Step& s, int t, int wave) const {
    const uint32_t o = kAlongK && (int)kpos >= s.left ? kNowhere : off[t];
    const uint32_t to = __builtin_amdgcn_readfirstlane(s.lds + (wave * kPer + t) % kLoads * 1024);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 ::"s"(to), "v"(o), "s"(s.rsrc) : "memory", "m0");
  }
};

// The same tile by way of registers, for rows that start anywhere (groups of 16 bytes
// at any address, and what is past the range element by element).
template <typename T, int kRows, bool kAlongK, int kWaves>
struct TileStage {
  using Load = TileLoad<T, kRows, kAlongK, kWaves>;
  static constexpr int kPer = Load::kPer, kGroup = Load::kGroup;
  I4 held[kPer];

  __device__ __forceinline__ static int place(int t, int wave, int lane) {   // in the tile
    return (wave * kPer + t) % Load::kLoads * 1024 + lane * 16;
  }
  __device__ __forceinline__ void fetch(const char* base, int64_t ld, int valid, int left, int wave, int lane) {
#pragma unroll
    for (int t = 0; t < kPer; ++t) {
      const int at = place(t, wave, lane), row = at / Load::kRowBytes, slot = at % Load::kRowBytes / 16;
      const int first = (kAlongK ? slot ^ (row & 7) : slot ^ Load::turned(row)) * kGroup;
      const int n = kAlongK ? (row < valid ? left - first : 0) : (row < left ? valid - first : 0);
      held[t] = I4{0, 0, 0, 0};
      const T* p = (const T*)base + row * ld + first;
      if (n >= kGroup) {
        __builtin_memcpy(&held[t], p, 16);
      } else if (n > 0) {
        const Raw8<T> r = load_left(p, n);
#pragma unroll
        for (int k = 0; k < 4; ++k) held[t][k] = r.w[k];
      }
    }
  }
  __device__ __forceinline__ void put(LdsChar* tile, int wave, int lane) const {
    typedef __attribute__((address_space(3))) I4 LdsI4;
#pragma unroll
    for (int t = 0; t < kPer; ++t) *(LdsI4*)(tile + place(t, wave, lane)) = held[t];
  }
};

// A lane's view of a tile: fragment f (16 rows or columns), half a step each.
template <typename T, int kRows, bool kAlongK>
struct TileRead {
  static constexpr int kElt = sizeof(T);
  static constexpr int kRowBytes = kAlongK ? kStepBytes : kRows * kElt;
  uint32_t at;   // of fragment 0 of the wave, first half

  __device__ __forceinline__ void init(int lane, int first) {   // first: of the wave's fragments
    const int i = lane & 15, g = lane >> 4;
    if constexpr (kAlongK) {
      at = (first * 16 + i) * kStepBytes + ((g ^ (i & 7)) * 16);
    } else if constexpr (sizeof(T) == 4) {
      at = 4 * g * kRowBytes + i * 4 + ((first * 64) ^ (TileLoad<T, kRows, false, 1>::turned(4 * g) * 16));
    } else {
      const int k = 8 * g + i / 4;
      at = k * kRowBytes + ((first * 32) ^ (TileLoad<T, kRows, false, 1>::turned(k) * 16)) + (i % 4) * 8;
    }
  }

  // The fragment's 16 bytes a lane: k = 64 bytes x half + 16 bytes x (lane / 16) on, along k.
  __device__ __forceinline__ I4 get(LdsChar* tile, int f, int half) const {
    typedef __attribute__((address_space(3))) I4 LdsI4;
    typedef __attribute__((address_space(3))) int LdsInt;
    typedef short S4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) S4 LdsS4;
    if constexpr (kAlongK) {
      return *(LdsI4*)(tile + (at ^ (half * 64)) + f * 16 * kStepBytes);
    } else if constexpr (sizeof(T) == 4) {
      LdsChar* p = tile + (at ^ (f * 64)) + half * 16 * kRowBytes;
      return I4{*(LdsInt*)p, *(LdsInt*)(p + kRowBytes), *(LdsInt*)(p + 2 * kRowBytes), *(LdsInt*)(p + 3 * kRowBytes)};
    } else {
      LdsChar* p = tile + (at ^ (f * 32)) + half * 32 * kRowBytes;
      struct Both {
        S4 lo, hi;
      } v = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)p),
             __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)(p + 4 * kRowBytes))};
      return __builtin_bit_cast(I4, v);
    }
  }
};

// acc += over half a step: rows of the result are p's, columns q's.
template <typename T>
__device__ __forceinline__ F4 mma(F4 acc, I4 p, I4 q) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(p[j]), __int_as_float(q[j]), acc, 0, 0, 0);
    return acc;
  } else if constexpr (std::is_same<T, _Float16>::value) {
    typedef _Float16 H8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, p), __builtin_bit_cast(H8, q), acc, 0, 0, 0);
  } else {
    typedef __bf16 B8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, p), __builtin_bit_cast(B8, q), acc, 0, 0, 0);
  }
}

// Between a wave's LDS stores and its other lanes' loads of them, and such loads and the
// next stores there. The hardware keeps a wave's order; the compiler, which sees that one
// lane's addresses differ, may not. No instruction of its own.
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A block's product: kM x kN of C by kWavesM x kWavesN waves. kSubs = 2: the tile's
// columns are kN / 2 of each of two matrices, and each wave has as many of both.
// kStaged: operands by way of registers (TileStage).
template <typename T_, int kM_, int kN_, int kWavesM_, int kWavesN_, int kStages_, bool kAK_, bool kBK_, int kSubs_,
          bool kStaged_ = false>
struct Product {
  using T = T_;
  static constexpr int kM = kM_, kN = kN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kStages = kStages_, kSubs = kSubs_;
  static constexpr bool kAK = kAK_, kBK = kBK_, kStaged = kStaged_;
  static constexpr int kWaves = kWavesM * kWavesN, kThreads = 64 * kWaves, kStep = kStepBytes / sizeof(T);
  static constexpr int kFM = kM / kWavesM / 16, kFN = kN / kWavesN / 16, kFS = kFN / kSubs;
  static constexpr int kSubN = kN / kSubs;
  using LoadA = TileLoad<T, kM, kAK, kWaves>;
  using LoadB = TileLoad<T, kSubN, kBK, kWaves>;
  static constexpr int kStage = LoadA::kBytes + kSubs * LoadB::kBytes;
  static constexpr int kLds = kStages * kStage;
  static constexpr int kPer = LoadA::kPer + kSubs * LoadB::kPer;   // loads of a wave in a step
  static_assert(kM % (16 * kWavesM) == 0 && kN % (16 * kWavesN * kSubs) == 0 && kStages >= 2, "");

  // waves of a SIMD, as many blocks as fit a CU's 160 KB
  static constexpr int kBlocks = 163840 / kLds < 1 ? 1 : 163840 / kLds > 4 ? 4 : 163840 / kLds;
  static constexpr int kWaveSlots = kBlocks * kWaves / 4 > 4 ? 4 : kBlocks * kWaves / 4;

  int wave, lane, wm, wn;

  __device__ __forceinline__ Product(int thread = threadIdx.x) {
    wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    lane = thread & 63;
    wm = wave / kWavesN;
    wn = wave % kWavesN;
  }
  // The row and first column (of four) of acc[j][i] in the tile; columns of sub j / kFS.
  __device__ __forceinline__ int row(int i) const { return (wm * kFM + i) * 16 + (lane & 15); }
  __device__ __forceinline__ int col(int j) const { return (wn * kFS + j % kFS) * 16 + (lane >> 4) * 4; }

  // Calls f(row, column, v[kOut][8]) for every eight consecutive columns of the tile's
  // rows (of the first kOut matrices'), which a wave's lanes have side by side: the
  // sums go through LDS, each wave's by itself. Stores of the four columns that a lane
  // has in registers touch 16 rows in 32 bytes each: a tile of 256 x 256 in bfloat16 takes
  // 8.5 us instead of 5.2.
  template <int kOut, typename F>
  __device__ __forceinline__ void each8(const F4 (&acc)[kFN][kFM], LdsChar* lds, F&& f) const {
    typedef __attribute__((address_space(3))) F4 LdsF4;
    constexpr int kRow = kOut * kFS * 64, kRoom = kLds / kWaves;   // bytes of a row, of a wave
    constexpr int kFit = kRoom / (16 * kRow), kLanes = kFS * 2;   // fragments that fit
    constexpr int kPass = kFit >= kFM ? kFM : kFit >= 4 ? 4 : kFit >= 2 ? 2 : 1;
    static_assert(kFit >= 1 && kFM % kPass == 0, "");
    LdsChar* room = lds + wave * kRoom;
    // groups of 16 bytes permuted against meetings in a bank
    constexpr int kTurn = kRow < 128 ? kRow / 16 - 1 : 7;
    const auto at = [&](int r, int group) { return (LdsF4*)(room + r * kRow + ((group ^ (r & kTurn)) * 16)); };
#pragma unroll
    for (int i0 = 0; i0 < kFM; i0 += kPass) {
#pragma unroll
      for (int i = 0; i < kPass; ++i)
#pragma unroll
        for (int j = 0; j < kOut * kFS; ++j) *at(i * 16 + (lane & 15), j * 4 + (lane >> 4)) = acc[j][i0 + i];
      lanes_meet();
      constexpr int kEights = kPass * 16 * kLanes;
#pragma unroll
      for (int t = 0; t < (kEights + 63) / 64; ++t) {
        if (kEights % 64 != 0 && t * 64 + lane >= kEights) break;
        const int r = (t * 64 + lane) / kLanes, q = lane % kLanes;
        float v[kOut][8];
#pragma unroll
        for (int s = 0; s < kOut; ++s) {
          const F4 x = *at(r, s * kFS * 4 + 2 * q), y = *at(r, s * kFS * 4 + 2 * q + 1);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[s][k] = x[k], v[s][k + 4] = y[k];
        }
        f((wm * kFM + i0) * 16 + r, wn * kFS * 16 + 8 * q, v);
      }
      if (i0 + kPass < kFM) lanes_meet();
    }
  }

  // The tile from (m0, n0) on over steps [step0, step1) of k; every wave has passed
  // its last read of `lds` when this returns, and no load is under way.
  __device__ __forceinline__ void run(F4 (&acc)[kFN][kFM], const ProductArgs& a, int m0, int n0, int step0, int step1,
                                      LdsChar* lds) const {
    LoadA la;
    LoadB lb;
    const int validm = a.m - m0, validn = a.n - n0;
    la.init(wave, lane, a.a.ld, validm);
    lb.init(wave, lane, a.b.ld, validn);
    const int per = (a.k + kStep - 1) / kStep;   // steps of a part
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    // where a step's tiles begin, and the k that are left there
    const auto part_of = [&](int step) { return kSubs == 1 && step >= per; };
    const auto k_of = [&](int step) { return (int64_t)(part_of(step) ? step - per : step) * kStep; };
    const auto left_of = [&](int step) { return step < step1 ? (int)(a.k - k_of(step)) : 0; };
    const auto from_a = [&](int step) {
      const int64_t k = k_of(step);
      return (const char*)((const T*)(part_of(step) ? a.a.q : a.a.p) + (kAK ? (int64_t)m0 * a.a.ld + k : k * a.a.ld + m0));
    };
    const auto from_b = [&](int step, int sub) {
      const int64_t k = k_of(step);
      return (const char*)((const T*)((kSubs == 1 ? part_of(step) : sub == 1) ? a.b.q : a.b.p) +
                           (kBK ? (int64_t)n0 * a.b.ld + k : k * a.b.ld + n0));
    };
    struct Steps {
      typename LoadA::Step a;
      typename LoadB::Step b[kSubs];
    };
    const auto step_of = [&](int stage, int step) {
      Steps r;
      const uint32_t to = lds0 + stage * kStage;
      r.a = la.step(from_a(step), a.a.ld, validm, left_of(step), to);
#pragma unroll
      for (int s = 0; s < kSubs; ++s)
        r.b[s] = lb.step(from_b(step, s), a.b.ld, validn, left_of(step), to + LoadA::kBytes + s * LoadB::kBytes);
      return r;
    };
    TileStage<T, kM, kAK, kWaves> sa;
    TileStage<T, kSubN, kBK, kWaves> sb[kSubs];
    const auto fetch = [&](int step) {
      const int left = left_of(step);
      sa.fetch(from_a(step), a.a.ld, validm, left, wave, lane);
#pragma unroll
      for (int s = 0; s < kSubs; ++s) sb[s].fetch(from_b(step, s), a.b.ld, validn, left, wave, lane);
    };
    const auto put = [&](int stage) {
      sa.put(lds + stage * kStage, wave, lane);
#pragma unroll
      for (int s = 0; s < kSubs; ++s) sb[s].put(lds + stage * kStage + LoadA::kBytes + s * LoadB::kBytes, wave, lane);
    };
    // load number t of a wave's kPer in a step
    const auto load = [&](const Steps& r, int t) {
      if (t < LoadA::kPer) la.load(r.a, t, wave);
      else lb.load(r.b[(t - LoadA::kPer) / LoadB::kPer], (t - LoadA::kPer) % LoadB::kPer, wave);
    };
    TileRead<T, kM, kAK> ra;
    TileRead<T, kSubN, kBK> rb;
    ra.init(lane, wm * kFM);
    rb.init(lane, wn * kFS);
    I4 fa[2][kFM], fb[2][kFN];
    const auto read_a = [&](int set, int i, int stage) { fa[set][i] = ra.get(lds + stage * kStage, i, set); };
    const auto read_b = [&](int set, int j, int stage) {
      fb[set][j] = rb.get(lds + stage * kStage + LoadA::kBytes + j / kFS * LoadB::kBytes, j % kFS, set);
    };
    // The matrix instructions of one half step, among them the reads of the next and, in
    // the second half, the loads, one at a time: a wave that issues a load does nothing
    // else for some 30 cycles.
    const auto half = [&](auto set_, int stage, const Steps* r) {
      constexpr int set = decltype(set_)::value, next = 1 - set;
#pragma unroll
      for (int i = 0; i < kFM; ++i) {
        read_a(next, i, stage);
#pragma unroll
        for (int j = i * kFN / kFM; j < (i + 1) * kFN / kFM; ++j) read_b(next, j, stage);
#pragma unroll
        for (int j = 0; j < kFN; ++j) acc[j][i] = mma<T>(acc[j][i], fb[set][j], fa[set][i]);
        if constexpr (set == 1 && !kStaged) {
#pragma unroll
          for (int t = i * kPer / kFM; t < (i + 1) * kPer / kFM; ++t) load(*r, t);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
#pragma unroll
    for (int j = 0; j < kFN; ++j)
#pragma unroll
      for (int i = 0; i < kFM; ++i) acc[j][i] = F4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (kStaged) {
#pragma unroll
      for (int s = 0; s < kStages; ++s) {
        fetch(step0 + s);
        if (s < kStages - 1) put(s);   // the last one stays in registers
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    } else {
#pragma unroll
      for (int s = 0; s < kStages; ++s) {
        const Steps r = step_of(s, step0 + s);
#pragma unroll
        for (int t = 0; t < kPer; ++t) load(r, t);
      }
      CKM_WAIT_LOADS((kStages - 1) * kPer);
      asm volatile("s_barrier" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < kFM; ++i) read_a(0, i, 0);
#pragma unroll
    for (int j = 0; j < kFN; ++j) read_b(0, j, 0);
    int stage = 0;
    for (int s = step0; s < step1; ++s) {
      const int next = stage + 1 == kStages ? 0 : stage + 1;
      half(std::integral_constant<int, 0>{}, stage, nullptr);
      if constexpr (kStaged) {
        put(stage == 0 ? kStages - 1 : stage - 1);   // the place of the step before, kStages - 1 ahead
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        fetch(s + kStages);
        half(std::integral_constant<int, 1>{}, next, nullptr);
      } else {
        const Steps r = step_of(stage, s + kStages);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 2) * kPer) : "memory");
        half(std::integral_constant<int, 1>{}, next, &r);
      }
      stage = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
};

template <class S>
struct Tag {
  using Shape = S;
};

// The place in a grid of tiles_m x tiles_n that block `b` of them takes. Blocks go to
// the eight dies in turn, so each die gets a range of its own, and goes through it in
// columns of up to eight tiles of m, which share the operands' tiles in its cache.
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int total = tiles_m * tiles_n, per = total / 8, rest = total % 8;
  const int die = b % 8, at = die * per + min(die, rest) + b / 8;
  const int band = at / (8 * tiles_n), first = band * 8, high = min(8, tiles_m - first);
  const int in = at - first * tiles_n;
  tm = first + in % high;
  tn = in / high;
}

// Up to four consecutive elements of a row at column `col`, rounded to T.
template <typename T>
__device__ __forceinline__ void store4(T* row, int col, int cols, F4 v) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 r;
#pragma unroll
  for (int k = 0; k < 4; ++k) r[k] = rounded<T>(v[k]);
  if (col + 4 <= cols) {
    __builtin_memcpy(row + col, &r, sizeof(r));
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (col + k < cols) row[col + k] = r[k];
  }
}

// How a product of m x n is cut: the shape of a tile, and shares of k, whose sums are
// joined in a fixed order.
struct Cut {
  int rows;                  // of a tile: names its shape (with_shape)
  int cols;                  // of n (of each matrix's, for kSubs = 2)
  int tiles_m, tiles_n;      // of one half
  int halves, splits, steps; // results side by side; steps of k in a share
  bool staged;               // operands whose rows start anywhere
  double time;               // the model's, us
  int64_t blocks() const { return (int64_t)tiles_m * tiles_n * halves * splits; }
};
// subs: 2 when a tile's columns are of two matrices (n then counts one's). bytes: of
// the operands. split: whether shares of k are possible. a_along_k: tiles of 16 rows are
// for an A along k alone.
Cut cut_product(int type, int64_t m, int64_t n, int halves, int subs, int64_t steps, int64_t bytes, bool split,
                bool a_along_k);
// The best cut of the same product with the shares of `as`, which cut_product gave, for
// operands that cannot be loaded straight to LDS too: the sums' order, and so every bit of
// a result, goes by the sizes and not by where operands lie (left to the model, f16
// 16x2048x2048 has three shares or four).
enum Staged { kStraight, kStagedAlong, kStagedAcross };   // with rows of k, or of m or n
Cut cut_like(int type, int64_t m, int64_t n, int halves, int subs, int64_t steps, int64_t bytes, bool a_along_k,
             Staged staged, const Cut& as);
// Cuts of two products that share a launch, in place of the two given, if the model has
// them done sooner; whether that is so. The first's tiles have 64 or 128 rows, the
// second's 128, and no shares.
bool cut_together(int type, Cut& a, int64_t m_a, int64_t n_a, int64_t steps_a, Cut& b, int64_t m_b, int64_t n_b,
                  int64_t steps_b, int64_t bytes);
// Whether they can be staged: a tile's rows then stay within 2^31 bytes too.
inline bool stageable(int64_t rows, int64_t ld, size_t elt) { return rows == 1 || ld * (int64_t)elt <= kMaxRowBytes; }
// The model's time of copying `bytes` of operands in a launch, us.
inline double copy_time(int64_t bytes) { return 5.0 + 2.0 * bytes / 4.0e6; }

__host__ __device__ inline int64_t whole(int64_t n, int64_t of) { return (n + of - 1) / of * of; }
// Elements from row to row of a matrix in the work buffer: 128 bytes past a multiple of
// 256, so that a tile's rows are spread over the memory's channels.
inline int64_t row_of(int64_t cols, size_t elt) { return (whole(cols * elt, 256) + 128) / elt; }
// A matrix that a call writes or reads, and whether two share an element: by their
// ranges, and where their rows lie at one stride by the columns.
struct Place {
  const char* name;
  const void* p;
  int64_t rows, cols, ld;
  size_t elt;
};
ckm_status check_apart(std::initializer_list<Place> outputs, std::initializer_list<Place> inputs);
// CKM_E_UNSUPPORTED for a grid past what a launch counts.
ckm_status check_blocks(const Cut& c);

// Calls f with the shape of a cut's tiles: 256 x 256 columns where there are enough of
// them, smaller ones to fill the CUs, 16 rows for single tokens, whose weights are read
// once. A tile of two matrices has waves of 128 columns, 64 of each, so that a wave's
// rows of the result are whole lines of memory. The largest shape has no registers left
// to stage operands in.
template <typename T, bool kAK, bool kBK, int kSubs, typename F>
void with_shape(const Cut& cut, F&& f) {
  if (cut.staged) {
    if (cut.rows == 128) f(Tag<Product<T, 128, 128, 2, 2, 2, kAK, kBK, kSubs, true>>());
    else if (cut.rows == 64) f(Tag<Product<T, 64, 128, 2, 2, 3, kAK, kBK, kSubs, true>>());
    else if constexpr (kAK) f(Tag<Product<T, 16, 128, 1, 4, 4, kAK, kBK, kSubs, true>>());
  } else if (cut.rows == 256) {
    f(Tag<Product<T, 256, 256, kSubs == 2 ? 4 : 2, kSubs == 2 ? 2 : 4, 2, kAK, kBK, kSubs>>());
  } else if (cut.rows == 128) {
    f(Tag<Product<T, 128, 128, 2, 2, 2, kAK, kBK, kSubs>>());
  } else if (cut.rows == 64) {
    f(Tag<Product<T, 64, 128, 2, 2, 3, kAK, kBK, kSubs>>());
  } else if constexpr (kAK) {
    f(Tag<Product<T, 16, 128, 1, 4, 4, kAK, kBK, kSubs>>());
  }
}

// Up to three copies in a launch: rows of cols elements into rows of `ld` (whole groups),
// zeros between; with targets, a row whose target is outside [0, vocab) as zeros.
struct PackArgs {
  struct One {
    const void* src;
    void* dst;
    int64_t total, ld_src, ld;   // total: groups of eight columns
    uint32_t groups;             // of a row
    int32_t cols;
    uint32_t blocks;
  } one[3];
  int count;
  const int64_t* targets;
  int64_t vocab;
  // with `most`, one more block: the largest finite |dloss| of rows that have a target,
  // 1 if that is 0
  const float* dloss;
  float* most;
  int64_t rows;
  void add(const void* src, int64_t rows, int64_t cols, int64_t ld_src, void* dst, int64_t ld);
};
void launch_pack(int type, const PackArgs& a, hipStream_t s);
// Zeros in rows of cols elements.
void launch_zero(int type, void* dst, int64_t rows, int64_t cols, int64_t ld, hipStream_t s);

// ---- a product alone, into a result or into shares --------------------------
struct ResultArgs {
  ProductArgs p;          // n: of one half
  void* c[2];             // the result's halves; or
  float* slab;            // shares [split][half][m][ld_slab] in binary32, when not NULL
  int64_t ld_c[2], ld_slab;
  bool add;               // to what the slab holds
  const float* alpha;     // NULL, or a factor on the device,
  float factor;           // times this
  int32_t tiles_m, tiles_n, halves, steps;   // Cut
};

// A block's tile of a result. Two results side by side: half h takes b's p or q (parts
// is 1 then).
template <class P, bool kSlab>
__device__ __forceinline__ void product_tile(const ResultArgs& a, int block, char* lds) {
  const P p;
  const int tiles = a.tiles_m * a.tiles_n * a.halves, split = block / tiles;
  int tm, tn;
  tile_of(block % tiles, a.tiles_m, a.tiles_n * a.halves, tm, tn);
  const int half = tn / a.tiles_n;
  tn -= half * a.tiles_n;
  ProductArgs product = a.p;
  if (half) product.b.p = product.b.q;
  const int all = (a.p.k + P::kStep - 1) / P::kStep * a.p.parts, from = split * a.steps;
  F4 acc[P::kFN][P::kFM];
  p.run(acc, product, tm * P::kM, tn * P::kN, from, min(all, from + a.steps), (LdsChar*)lds);
  const float factor = kSlab ? 1.0f : a.alpha ? a.factor * *a.alpha : a.factor;
  typename P::T* c = (typename P::T*)(half ? a.c[1] : a.c[0]);
  const int64_t ld_c = half ? a.ld_c[1] : a.ld_c[0];
  const int64_t row0 = kSlab ? ((int64_t)split * a.halves + half) * a.p.m : 0;
  p.template each8<1>(acc, (LdsChar*)lds, [&](int row, int col, float (&v)[1][8]) {
    const int m = tm * P::kM + row, n = tn * P::kN + col;
    if (m >= a.p.m || n >= a.p.n) return;
    if constexpr (kSlab) {   // rows of whole eights
      F4* at = (F4*)(a.slab + (row0 + m) * a.ld_slab + n);
      F4 x = {v[0][0], v[0][1], v[0][2], v[0][3]}, y = {v[0][4], v[0][5], v[0][6], v[0][7]};
      if (a.add) x += at[0], y += at[1];
      at[0] = x;
      at[1] = y;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[0][k] *= factor;
      store_part<false>(c + m * ld_c, rounded8<typename P::T>(v[0]), n, a.p.n);
    }
  });
}

template <class P, bool kSlab>
__global__ void __launch_bounds__(P::kThreads, P::kWaveSlots) ckm_product_kernel(ResultArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
  product_tile<P, kSlab>(a, blockIdx.x, lds);
}
// Two results that need not wait for one another, each with blocks of its own: where
// neither fills the CUs.
template <class P, bool kSlab, class Q>
__global__ void __launch_bounds__(P::kThreads, 2) ckm_two_products_kernel(ResultArgs a, int blocks_a, ResultArgs b) {
  static_assert(P::kThreads == Q::kThreads, "");
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds > Q::kLds ? P::kLds : Q::kLds];
  if ((int)blockIdx.x < blocks_a) product_tile<P, kSlab>(a, blockIdx.x, lds);
  else product_tile<Q, false>(b, blockIdx.x - blocks_a, lds);
}

// Adds the shares of a result in their order.
void launch_join(int type, const ResultArgs& a, int splits, hipStream_t s);

inline void set_cut(ResultArgs& a, const Cut& cut) {
  a.tiles_m = cut.tiles_m;
  a.tiles_n = cut.tiles_n;
  a.halves = cut.halves;
  a.steps = cut.steps;
}

template <typename T, bool kAK, bool kBK>
void launch_product(ResultArgs a, const Cut& cut, hipStream_t s) {
  set_cut(a, cut);
  with_shape<T, kAK, kBK, 1>(cut, [&](auto p) {
    using P = typename decltype(p)::Shape;
    if (a.slab) ckm_product_kernel<P, true><<<(uint32_t)cut.blocks(), P::kThreads, 0, s>>>(a);
    else ckm_product_kernel<P, false><<<(uint32_t)cut.blocks(), P::kThreads, 0, s>>>(a);
  });
}

// a: A along k, B along k or across it (kBK); b: both across. The cuts are together's.
template <typename T, bool kBK>
void launch_two(ResultArgs a, const Cut& cut_a, ResultArgs b, const Cut& cut_b, hipStream_t s) {
  set_cut(a, cut_a);
  set_cut(b, cut_b);
  using Q = Product<T, 128, 128, 2, 2, 2, false, false, 1>;
  const auto go = [&](auto p) {
    using P = typename decltype(p)::Shape;
    const uint32_t blocks = (uint32_t)(cut_a.blocks() + cut_b.blocks());
    const int blocks_a = (int)cut_a.blocks();
    if (a.slab) ckm_two_products_kernel<P, true, Q><<<blocks, P::kThreads, 0, s>>>(a, blocks_a, b);
    else ckm_two_products_kernel<P, false, Q><<<blocks, P::kThreads, 0, s>>>(a, blocks_a, b);
  };
  if (cut_a.rows == 128) go(Tag<Product<T, 128, 128, 2, 2, 2, true, kBK, 1>>());
  else go(Tag<Product<T, 64, 128, 2, 2, 3, true, kBK, 1>>());
}

}  // namespace ckm
