// rmsnorm.hip -- residual addition, root-mean-square norm and quantization of its
// result in one pass (gfx950): what stands in front of a quantized linear.
//
//   h = bf16(x + residual)                       (h = x without a residual)
//   y_j = fl(fl(h_j r) w_j), r = fl(1 / fl(sqrt(fl(mean_j h_j^2) + eps)))
//   y as bf16, or quantized from its fp32 values: FP8, NVFP4, MXFP4, MXFP8
//
// The norm is that of the stored sum h, so what a caller keeps and what was normed
// are the same numbers, and y can be computed again from h. The squares are summed
// in fp32, a thread's own first, then over the lanes and waves, in an order that only the
// row's length decides.
//
// HBM-bound: x and the residual are read once, h and y written once. A row stays in
// the registers of the threads that share it (packed bf16, 16 elements a unit: a whole
// NVFP4 block, half an MX one, and a 16-byte store of FP8 codes), from the loads to the
// codes. Rows of any alignment and length: units are loaded with wide loads that
// need no alignment, a shorter last one shifted into place (load16). Static FP8 with a
// residual, inputs in turn past the memory-side cache: 4608 x 3072 21.1 us (4.7 TB/s),
// 16384 x 4096 85 us (5.5 TB/s), 1 x 1024 2.6 us (one launch's latency); of three inputs
// in turn 4608 x 3072 18.4 (5.4 TB/s).
//
// A tensor scale taken from y (dynamic FP8, NVFP4) needs the largest |y| of all
// rows before the first code: one workgroup does a tensor of few rows in one launch;
// otherwise a first launch writes h and a maximum per workgroup, parked in the code
// buffer, and the last one norms h again, with the same steps, and codes it. Between
// them k_norm_scale makes the scale of the maxima; or, for tensors of moderate size, the
// first launch leaves its maxima at the start of every workgroup's own codes, where
// the last finds them (launch_dynamic).
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace qg {

enum { F_BF16 = 0, F_FP8 = 1, F_NVFP4 = 2, F_MXFP4 = 3, F_MXFP8 = 4, F_AMAX = 5 };  // qg_format; F_AMAX: h and max |y| alone

// ---------------------------------------------------------------- 16 elements of a row
// Elements [c, c + 16) of a row of cols, zero from cols on. EVEN: cols % 16 == 0, every
// unit whole (an instance of its own: with the code for shorter units behind branches
// the others take 10 % longer, 4608 x 3072 23.4 us against 20.6). A row's last unit, if
// shorter, is loaded as the row's last 16 elements and shifted down, the same in every
// row: one latency, where a condition on each element made 16 loads follow each other
// (300 x 1001 5.1 us against 4.6; a row of fewer than 16 elements still takes them).
template <int N>  // words; down by `words` of them
__device__ __attribute__((always_inline)) inline void shift_down(uint32_t (&w)[N], int words) {
#pragma unroll
  for (int k = N / 2; k > 0; k >>= 1)
    if (words & k) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = i + k < N ? w[i + k < N ? i + k : 0] : 0u;
    }
}
template <bool EVEN>
__device__ __attribute__((always_inline)) inline void load16(const uint16_t* row, int c, int cols, uint32_t (&w)[8]) {
  if (EVEN || cols - c >= 16) {
    __builtin_memcpy(w, row + c, 32);
  } else if (cols >= 16) {
    const int gone = 16 - cols % 16;
    __builtin_memcpy(w, row + (cols - 16), 32);
    shift_down(w, gone >> 1);
    if (gone & 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = (w[i] >> 16) | (i < 7 ? w[i < 7 ? i + 1 : 0] << 16 : 0u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t lo = (2 * i < cols) ? (uint32_t)row[2 * i] : 0u;
      const uint32_t hi = (2 * i + 1 < cols) ? (uint32_t)row[2 * i + 1] : 0u;
      w[i] = lo | (hi << 16);
    }
  }
}
template <bool EVEN>
__device__ __attribute__((always_inline)) inline void store16(uint16_t* p, int cnt, const uint32_t (&w)[8]) {
  if (EVEN || cnt >= 16) {
    __builtin_memcpy(p, w, 32);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < cnt) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
  }
}

template <bool EVEN>
__device__ __attribute__((always_inline)) inline void load_weight(const NormArgs& a, int c, float (&v)[16]) {
  if (a.w_f32) {
    const float* p = reinterpret_cast<const float*>(a.w);
    uint32_t w[16];
    if (EVEN || a.cols - c >= 16) {
      __builtin_memcpy(w, p + c, 64);
    } else if (a.cols >= 16) {
      __builtin_memcpy(w, p + (a.cols - 16), 64);
      shift_down(w, 16 - a.cols % 16);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = (i < a.cols) ? f2u(p[i]) : 0u;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = u2f(w[i]);
  } else {
    uint32_t w[8];
    load16<EVEN>(reinterpret_cast<const uint16_t*>(a.w), c, a.cols, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[2 * i] = bf16_lo(w[i]);
      v[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}

// A unit of h; with a residual the sum, written to a.sum where the caller wants it.
// (In place, a row's last unit may read elements that its neighbour has just replaced:
// those that are shifted out.) ONE_OF: of several units of a thread; x is then kept as
// it is until the residual's loads are on their way: the compiler otherwise widens it
// before the branch, so that they wait for it (4608 x 9216 59.3 us, now 56.7).
template <bool EVEN, bool ONE_OF = false>
__device__ __attribute__((always_inline)) inline void load_h(const NormArgs& a, int64_t row, int c, uint32_t (&h)[8]) {
  load16<EVEN>(a.x + row * a.ldx, c, a.cols, h);
  if (a.res) {
    uint32_t r[8];
    load16<EVEN>(a.res + row * a.ldr, c, a.cols, r);
    if constexpr (ONE_OF)
      asm volatile("" : "+v"(h[0]), "+v"(h[1]), "+v"(h[2]), "+v"(h[3]), "+v"(h[4]), "+v"(h[5]), "+v"(h[6]), "+v"(h[7]));
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = pk_bf16(bf16_lo(h[i]) + bf16_lo(r[i]), bf16_hi(h[i]) + bf16_hi(r[i]));
    if (a.sum) store16<EVEN>(a.sum + row * a.lds + c, a.cols - c, h);
  }
}

__device__ __attribute__((always_inline)) inline float squares(const uint32_t (&h)[8], float ss, float scale) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float lo = bf16_lo(h[i]) * scale, hi = bf16_hi(h[i]) * scale;
    ss = __builtin_fmaf(lo, lo, ss);
    ss = __builtin_fmaf(hi, hi, ss);
  }
  return ss;
}

__device__ __attribute__((always_inline)) inline void norm16(const uint32_t (&h)[8], const float (&w)[16], float pre, float rstd,
                                                             float (&y)[16]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[2 * i] = __fmul_rn(__fmul_rn(bf16_lo(h[i]) * pre, rstd), w[2 * i]);
    y[2 * i + 1] = __fmul_rn(__fmul_rn(bf16_hi(h[i]) * pre, rstd), w[2 * i + 1]);
  }
}

__device__ __attribute__((always_inline)) inline uint32_t amax16(const float (&y)[16]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, f2u(y[i]) & 0x7FFFFFFFu);
  return m;
}

// Elements [c, c + 16) of row `row` of y, `cnt` of them in the row, in the output
// format. s: tensor scale; r: its reciprocal (FP8). MX: the lanes of units 2 j and 2 j + 1
// call this together. NVFP4 and MX rows are whole blocks.
template <int FMT, bool EVEN>
__device__ __attribute__((always_inline)) inline void store_y(const NormArgs& a, int64_t row, int c, int cnt, const float (&y)[16],
                                                              float s, float r) {
  if constexpr (FMT == F_BF16) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = pk_bf16(y[2 * i], y[2 * i + 1]);
    store16<EVEN>(reinterpret_cast<uint16_t*>(a.y) + row * a.ldy + c, cnt, w);
  } else if constexpr (FMT == F_FP8 || FMT == F_MXFP8) {
    if constexpr (FMT == F_MXFP8) {
      uint32_t am = amax16(y);
      am = max(am, (uint32_t)__shfl_xor((int)am, 1));
      const uint32_t e = mx_block<false>(am, r);
      if ((c & 31) == 0) a.bscale[row * (a.cols >> 5) + (c >> 5)] = (uint8_t)e;
    }
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t[4] = {__fmul_rn(y[4 * i], r), __fmul_rn(y[4 * i + 1], r), __fmul_rn(y[4 * i + 2], r),
                          __fmul_rn(y[4 * i + 3], r)};
      q[i] = hw_e4m3x4(t);
    }
    uint8_t* o = a.y + row * a.cols + c;
    if (EVEN || cnt >= 16) {
      __builtin_memcpy(o, q, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < cnt) o[i] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
    }
  } else {
    uint32_t am = amax16(y);
    if constexpr (FMT == F_MXFP4) {
      am = max(am, (uint32_t)__shfl_xor((int)am, 1));
      const uint32_t e = mx_block<true>(am, r);
      if ((c & 31) == 0) a.bscale[row * (a.cols >> 5) + (c >> 5)] = (uint8_t)e;
    } else {
      a.bscale[row * (a.cols >> 4) + (c >> 4)] = (uint8_t)nv_block(am, s, __fmul_rn(6.0f, s), r);
    }
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = __fmul_rn(y[i], r);
    const uint32_t q[2] = {hw_e2m1x8(t), hw_e2m1x8(t + 8)};
    __builtin_memcpy(a.y + row * (a.cols >> 1) + (c >> 1), q, 8);
  }
}

// ---------------------------------------------------------------- reductions
// Over the TPR threads of a row: part of a wave, a wave, or the whole workgroup; red:
// words that no thread still reads.
template <int TPR>
__device__ __attribute__((always_inline)) inline float row_sum(float v, float* red) {
#pragma unroll
  for (int off = (TPR < 64 ? TPR : 64) / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v += red[i];
  }
  return v;
}
// The same for the units' sums of 1024 threads with a unit each, in the order that 256
// threads with up to four units each add them in: which of the two takes a row depends
// on the number of rows, its norm must not.
__device__ __attribute__((always_inline)) inline float row_sum_as_256(float v, float (&units)[1024], float* red) {
  const int t = threadIdx.x;
  units[t] = v;
  __syncthreads();
  if (t < 256) {
    v = units[t] + units[t + 256] + units[t + 512] + units[t + 768];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    if ((t & 63) == 0) red[t >> 6] = v;
  }
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}
__device__ __attribute__((always_inline)) inline uint32_t wave_max(uint32_t v) {
  for (int off = 32; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off));
  return v;
}

// Over the whole workgroup.
__device__ __attribute__((always_inline)) inline uint32_t group_max(uint32_t v) {
  __shared__ uint32_t part[16];
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) v = max(v, part[i]);
  return v;
}

// Squares of elements past 2^64 leave fp32, and those below 2^-63 lose digits to its
// subnormal numbers. A row whose sum is no finite number (or none with eps), or so small
// that those count and eps does not hide them, is summed again times 2^-96 or 2^96, an
// exact factor, and eps times its square. Small elements get the factor too. Large
// ones get 2^-4 of it and r the rest (r is then at least 2^-124, a normal number), so
// that elements far below the largest keep their digits.
constexpr float kDown = 1.262177448353618888658765e-29f, kUp = 7.9228162514264337593543950336e28f;  // 2^-96, 2^96
constexpr float kDownPre = 0.0625f, kDownRest = 2.0194839173657902e-28f;                          // 2^-4, 2^-92
// A subnormal square's rounding is at most 2^-150: of all of a row less than 2^-119 (2^31
// elements), 2^-39 of a sum of 2^-80; in their mean 2^-30 of an eps of 2^-120.
constexpr float kSmallSum = 8.2718061255302767e-25f, kSmallEps = 7.5231638452626401e-37f;  // 2^-80, 2^-120

__device__ __attribute__((always_inline)) inline float rstd_of(float ss, int cols, float eps) {
  const float v = __fadd_rn(__fdiv_rn(ss, (float)cols), eps);
  return v > 0.0f || v != v ? __fdiv_rn(1.0f, __fsqrt_rn(v)) : 0.0f;  // (a row of zeros with eps = 0)
}

// What the squares of a row of sum ss are summed again with; 1: they need not be. The
// same in every thread of the row.
__device__ __attribute__((always_inline)) inline float again_by(float ss, float eps) {
  if (!(ss + eps <= 3.40282347e38f)) return kDown;
  return ss < kSmallSum && eps < kSmallEps ? kUp : 1.0f;
}
// The factors of the elements, from the sum ss of the squares times f f.
__device__ __attribute__((always_inline)) inline void factors_again(float ss, int cols, float eps, float f, float& pre, float& rstd) {
  rstd = rstd_of(ss, cols, eps * f * f) * (f < 1.0f ? kDownRest : 1.0f);
  pre = f < 1.0f ? kDownPre : f;
}

__device__ __attribute__((always_inline)) inline float scale_of_max(uint32_t m, float divisor) {
  return m >= 0x7F800000u ? __builtin_nanf("") : __fdiv_rn(u2f(m), divisor);
}

// ---------------------------------------------------------------- rows in registers
// TPR threads share a row, NV units of 16 elements each: unit t + TPR i. TPR <= 64: a
// workgroup has blockDim / TPR rows at a time, else one. One or two units a thread
// measured best at nearly every size (12 shapes from 1 x 1024 to 16384 x 4096, TPR 64 to
// 1024, units of 8 and 16; before the EVEN instances): static FP8 with a residual 4608 x
// 3072 22.7 us with a workgroup per row against 25.3 with a wave, 500 x 3072 5.3 against
// 6.7, 16384 x 4096 84.7 against 91.1. Non-temporal loads or stores lose 5 to 30 %.
//
// Row `row` of thread t: h, and what its elements are multiplied by before the weight.
template <int NV, int TPR, bool EVEN>
__device__ __attribute__((always_inline)) inline void norm_row(const NormArgs& a, int64_t row, int t,
                                                               float (&red)[2][16], int& turn, uint32_t (&h)[NV][8],
                                                               float& pre, float& rstd) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = 16 * (t + TPR * i);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[i][j] = 0u;
    if (c < a.cols) load_h<EVEN, (NV > 1)>(a, row, c, h[i]);
  }
  const auto sum = [&](float f) __attribute__((always_inline)) {
    float ss = squares(h[0], 0.0f, f);
#pragma unroll
    for (int i = 1; i < NV; ++i) ss += squares(h[i], 0.0f, f);
    if constexpr (TPR == 1024 && NV == 1) {
      __shared__ float units[1024];
      ss = row_sum_as_256(ss, units, red[turn]);
    } else {
      ss = row_sum<TPR>(ss, red[turn]);
    }
    turn ^= 1;
    return ss;
  };
  const float all = sum(1.0f);
  pre = 1.0f;
  rstd = rstd_of(all, a.cols, a.eps);
  const float f = again_by(all, a.eps);
  if (f != 1.0f) factors_again(sum(f), a.cols, a.eps, f, pre, rstd);
}

// fn(first column, elements left in the row, the 16 values of y) for the thread's units.
template <int NV, int TPR, bool EVEN, class F>
__device__ __attribute__((always_inline)) inline void each_unit(const NormArgs& a, int t, const uint32_t (&h)[NV][8], float pre,
                                                                float rstd, F fn) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = 16 * (t + TPR * i);
    if (c >= a.cols) continue;
    float w[16], y[16];
    load_weight<EVEN>(a, c, w);
    norm16(h[i], w, pre, rstd, y);
    fn(c, a.cols - c, y);
  }
}

// The largest |y| of a workgroup's rows, to where the launch that codes them reads it:
// one word a workgroup, or (a.regions) one in each of that launch's workgroups' codes.
__device__ __attribute__((always_inline)) inline void leave_max(const NormArgs& a, uint32_t am) {
  am = group_max(am);
  if (a.regions == 0) {
    if (threadIdx.x == 0) a.partial[blockIdx.x] = am;
    return;
  }
  for (int64_t j = threadIdx.x; j < a.regions; j += blockDim.x)
    reinterpret_cast<uint32_t*>(a.y + j * a.region_bytes)[blockIdx.x] = am;
}

template <int FMT, int NV, int TPR, bool EVEN>
__global__ void __launch_bounds__(TPR == 1024 ? 1024 : 256) k_rms_norm(NormArgs a) {
  __shared__ float red[2][16];
  const int t = (int)threadIdx.x % TPR, rpb = (int)blockDim.x / TPR;
  float s = 0.0f, r = 0.0f;
  if (FMT == F_FP8 || FMT == F_NVFP4) {
    s = *a.tscale;
    r = (s > 0.0f) ? __fdiv_rn(1.0f, s) : 0.0f;
  }
  uint32_t am = 0;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * rpb + threadIdx.x / TPR; row < a.rows; row += (int64_t)gridDim.x * rpb) {
    uint32_t h[NV][8];
    float pre, rstd;
    norm_row<NV, TPR, EVEN>(a, row, t, red, turn, h, pre, rstd);
    each_unit<NV, TPR, EVEN>(a, t, h, pre, rstd, [&](int c, int cnt, const float (&y)[16]) __attribute__((always_inline)) {
      if constexpr (FMT == F_AMAX) am = max(am, amax16(y));
      else store_y<FMT, EVEN>(a, row, c, cnt, y, s, r);
    });
  }
  if constexpr (FMT == F_AMAX) leave_max(a, am);
}

// FP8 and NVFP4 with the tensor scale taken from y, where every workgroup has its rows in
// one turn. SLOTS: from the maxima that the launch before left at the start of this
// workgroup's codes (all read before the barrier that any code is written after);
// otherwise the only workgroup's own, which holds every row of the tensor.
template <int FMT, int NV, int TPR, bool SLOTS, bool EVEN>
__global__ void __launch_bounds__(SLOTS && TPR < 1024 ? 256 : 1024) k_rms_norm_scaled(NormArgs a) {
  __shared__ float red[2][16];
  const int t = (int)threadIdx.x % TPR, rpb = (int)blockDim.x / TPR;
  const int64_t row = (int64_t)blockIdx.x * rpb + threadIdx.x / TPR;
  const bool live = row < a.rows;  // (one row a workgroup: always)
  uint32_t h[NV][8], am = 0;
  float pre = 1.0f, rstd = 0.0f;
  int turn = 0;
  if (live) norm_row<NV, TPR, EVEN>(a, row, t, red, turn, h, pre, rstd);
  if constexpr (SLOTS) {
    const uint32_t* slots = reinterpret_cast<const uint32_t*>(a.y + (int64_t)blockIdx.x * a.region_bytes);
    for (int i = (int)threadIdx.x; i < a.slots; i += (int)blockDim.x) am = max(am, slots[i]);
  } else if (live) {
    each_unit<NV, TPR, EVEN>(a, t, h, pre, rstd, [&](int, int, const float (&y)[16]) __attribute__((always_inline)) {
      am = max(am, amax16(y));
    });
  }
  const float s = scale_of_max(group_max(am), FMT == F_FP8 ? 448.0f : 2688.0f);
  const float r = (s > 0.0f) ? __fdiv_rn(1.0f, s) : 0.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.tscale = s;
  if (!live) return;
  each_unit<NV, TPR, EVEN>(a, t, h, pre, rstd, [&](int c, int cnt, const float (&y)[16]) __attribute__((always_inline)) {
    store_y<FMT, EVEN>(a, row, c, cnt, y, s, r);
  });
}

// Rows too long for the registers: a workgroup walks the row twice (three times
// where the squares leave fp32), the second time from the caches where it fits.
template <int FMT, bool EVEN>
__global__ void __launch_bounds__(1024) k_rms_norm_long(NormArgs a) {
  __shared__ float red[2][16];
  float s = 0.0f, r = 0.0f;
  if (FMT == F_FP8 || FMT == F_NVFP4) {
    s = *a.tscale;
    r = (s > 0.0f) ? __fdiv_rn(1.0f, s) : 0.0f;
  }
  uint32_t am = 0;
  NormArgs again = a;  // the second reading: of the stored sum where there is one
  if (a.res && a.sum) {
    again.x = a.sum;
    again.ldx = a.lds;
    again.res = nullptr;
  }
  again.sum = nullptr;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    uint32_t h[8];
    float ss = 0.0f;
    for (int64_t c = 16 * (int64_t)threadIdx.x; c < a.cols; c += 16 * 1024) {
      load_h<EVEN>(a, row, (int)c, h);
      ss = squares(h, ss, 1.0f);
    }
    const float all = row_sum<1024>(ss, red[turn]);
    turn ^= 1;
    float pre = 1.0f, rstd = rstd_of(all, a.cols, a.eps);
    const float f = again_by(all, a.eps);
    if (f != 1.0f) {
      ss = 0.0f;
      for (int64_t c = 16 * (int64_t)threadIdx.x; c < a.cols; c += 16 * 1024) {
        load_h<EVEN>(again, row, (int)c, h);
        ss = squares(h, ss, f);
      }
      factors_again(row_sum<1024>(ss, red[turn]), a.cols, a.eps, f, pre, rstd);
      turn ^= 1;
    }
    for (int64_t c = 16 * (int64_t)threadIdx.x; c < a.cols; c += 16 * 1024) {
      const int cnt = (int)min((int64_t)16, a.cols - c);
      float w[16], y[16];
      load_h<EVEN>(again, row, (int)c, h);
      load_weight<EVEN>(a, (int)c, w);
      norm16(h, w, pre, rstd, y);
      if constexpr (FMT == F_AMAX) am = max(am, amax16(y));
      else store_y<FMT, EVEN>(a, row, (int)c, cnt, y, s, r);
    }
  }
  if constexpr (FMT == F_AMAX) leave_max(a, am);
}

// Workgroups of a launch that leaves a maximum each for k_norm_scale.
constexpr int64_t kNormMaxGroups = 2048;

// The tensor scale from `count` <= kNormMaxGroups maxima (fp32 bits), which may lie in
// `scale` itself. One workgroup, bound by latency: all its loads at once (in a loop,
// dynamic FP8 with a residual 4608 x 3072 takes 0.2 us more of 37, 1024 x 4096 0.1 to 0.6 of 16).
__global__ void __launch_bounds__(256) k_norm_scale(const uint32_t* partial, int count, float* scale, float divisor) {
  uint32_t m = 0;
  uint32_t v[kNormMaxGroups / 256];
#pragma unroll
  for (int i = 0; i < (int)(kNormMaxGroups / 256); ++i) {
    const int at = (int)threadIdx.x + 256 * i;
    v[i] = at < count ? partial[at] : 0;
  }
#pragma unroll
  for (int i = 0; i < (int)(kNormMaxGroups / 256); ++i) m = max(m, v[i]);
  m = group_max(m);
  if (threadIdx.x == 0) *scale = scale_of_max(m, divisor);
}

__global__ void k_norm_empty(float* scale) { *scale = 0.0f; }

// ---------------------------------------------------------------- launchers
// Workgroups of a launch (each thread count stays below 2^32).
constexpr int64_t kNormGroups = int64_t(1) << 20;

// Up to one row a CU of more than 256 units takes as many threads as a workgroup has.
constexpr int64_t kNormFewRows = 256;

struct NormPlan {
  int tpr, nv;     // threads that share a row (0: too long for the registers) and their units
  int64_t rpb;     // rows of a workgroup
  int64_t groups;  // workgroups that have every row in one turn
};
static NormPlan norm_plan(int64_t rows, int64_t cols) {
  const int64_t units = (cols + 15) / 16;
  NormPlan p;
  p.tpr = 0;
  if (units <= 128) {
    for (p.tpr = 8; p.tpr < units; p.tpr *= 2) {}
  } else if (units <= 256 || (units <= 256 * 4 && rows > kNormFewRows)) {
    p.tpr = 256;
  } else if (units <= 1024 * 3) {
    p.tpr = 1024;
  }
  p.nv = p.tpr ? (int)((units + p.tpr - 1) / p.tpr) : 0;
  p.rpb = p.tpr != 0 && p.tpr <= 64 ? 256 / p.tpr : 1;
  p.groups = (rows + p.rpb - 1) / p.rpb;
  return p;
}

// fn(NV, TPR) as constants.
template <class F>
static void with_plan(const NormPlan& p, F fn) {
  const auto call = [&]<int NV, int TPR>() { fn(std::integral_constant<int, NV>(), std::integral_constant<int, TPR>()); };
  switch (p.tpr) {
    case 8: call.template operator()<1, 8>(); break;
    case 16: call.template operator()<1, 16>(); break;
    case 32: call.template operator()<1, 32>(); break;
    case 64: call.template operator()<1, 64>(); break;
    case 128: call.template operator()<1, 128>(); break;
    case 256:
      if (p.nv == 1) call.template operator()<1, 256>();
      else if (p.nv == 2) call.template operator()<2, 256>();
      else if (p.nv == 3) call.template operator()<3, 256>();
      else call.template operator()<4, 256>();
      break;
    default:
      if (p.nv == 1) call.template operator()<1, 1024>();
      else if (p.nv == 2) call.template operator()<2, 1024>();
      else call.template operator()<3, 1024>();
  }
}

// EVEN instances of every format, others of those that take any row length.
template <int FMT, bool EVEN>
static void launch_rows(const NormArgs& a, const NormPlan& p, unsigned groups, hipStream_t st) {
  if (p.tpr == 0) {
    hipLaunchKernelGGL((k_rms_norm_long<FMT, EVEN>), dim3(groups), dim3(1024), 0, st, a);
    return;
  }
  with_plan(p, [&](auto NV, auto TPR) {
    hipLaunchKernelGGL((k_rms_norm<FMT, NV(), TPR(), EVEN>), dim3(groups), dim3((unsigned)(p.rpb * p.tpr)), 0, st, a);
  });
}
template <int FMT>
static void launch_all(const NormArgs& a, const NormPlan& p, int64_t groups_max, hipStream_t st) {
  const unsigned groups = (unsigned)std::min(p.groups, groups_max);
  if constexpr (FMT == F_BF16 || FMT == F_FP8 || FMT == F_AMAX) {
    if (a.cols % 16 != 0) {
      launch_rows<FMT, false>(a, p, groups, st);
      return;
    }
  }
  launch_rows<FMT, true>(a, p, groups, st);
}

template <int FMT, bool SLOTS, bool EVEN>
static void launch_scaled_rows(const NormArgs& a, const NormPlan& p, unsigned groups, unsigned threads, hipStream_t st) {
  with_plan(p, [&](auto NV, auto TPR) {
    hipLaunchKernelGGL((k_rms_norm_scaled<FMT, NV(), TPR(), SLOTS, EVEN>), dim3(groups), dim3(threads), 0, st, a);
  });
}
template <int FMT, bool SLOTS>
static void launch_scaled(const NormArgs& a, const NormPlan& p, unsigned groups, unsigned threads, hipStream_t st) {
  if constexpr (FMT == F_FP8) {
    if (a.cols % 16 != 0) {
      launch_scaled_rows<FMT, SLOTS, false>(a, p, groups, threads, st);
      return;
    }
  }
  launch_scaled_rows<FMT, SLOTS, true>(a, p, groups, threads, st);
}

// Up to so many workgroups the maxima are left in every workgroup's codes: a launch
// less for groups^2 scattered words (dynamic FP8 with a residual 300 x 1024, 75 groups,
// 8.4 us in three launches, 7.2 in two; 128 x 3072, 128, 8.5, 7.6; 1024 x 1024, 256, 9.6, 8.8;
// 300 x 9216, 300, 14.7, 14.0; 500 x 3072, 500, 11.0, 12.1).
constexpr int64_t kNormSlots = 256;

// A tensor scale taken from y.
template <int FMT>
static hipError_t launch_dynamic(NormArgs a, hipStream_t st) {
  const NormPlan p = norm_plan(a.rows, a.cols);
  if (p.tpr != 0 && (p.tpr <= 64 ? a.rows * p.tpr <= 1024 : a.rows == 1)) {
    launch_scaled<FMT, false>(a, p, 1, (unsigned)((a.rows * p.tpr + 63) / 64 * 64), st);
    return hipGetLastError();
  }
  const int64_t row_bytes = FMT == F_FP8 ? (int64_t)a.cols : (int64_t)a.cols / 2;
  NormArgs b = a;  // the last launch: reads the stored sum where there is one
  if (a.res && a.sum) {
    b.x = a.sum;
    b.ldx = a.lds;
    b.res = nullptr;
  }
  b.sum = nullptr;
  // (the last workgroup may have fewer rows, so fewer bytes of codes)
  const int64_t region_bytes = p.rpb * row_bytes, last_bytes = (a.rows - (p.groups - 1) * p.rpb) * row_bytes;
  if (p.tpr != 0 && p.groups <= std::min(kNormSlots, last_bytes / 4) && region_bytes % 4 == 0 &&
      reinterpret_cast<uintptr_t>(a.y) % 4 == 0) {
    a.regions = p.groups;
    a.region_bytes = b.region_bytes = region_bytes;
    b.slots = (int)p.groups;
    launch_all<F_AMAX>(a, p, p.groups, st);
    launch_scaled<FMT, true>(b, p, (unsigned)p.groups, (unsigned)(p.rpb * p.tpr), st);
    return hipGetLastError();
  }
  const uintptr_t base = (reinterpret_cast<uintptr_t>(a.y) + 3) & ~uintptr_t(3);
  const int64_t cap = (a.rows * row_bytes - (int64_t)(base - reinterpret_cast<uintptr_t>(a.y))) / 4;
  int64_t groups = std::min(p.groups, kNormMaxGroups);
  a.partial = reinterpret_cast<uint32_t*>(base);
  if (groups > cap) {  // short rows: one workgroup, its maximum straight into the scale's place
    groups = 1;
    a.partial = reinterpret_cast<uint32_t*>(a.tscale);
  }
  launch_all<F_AMAX>(a, p, groups, st);
  hipLaunchKernelGGL(k_norm_scale, dim3(1), dim3(256), 0, st, a.partial, (int)groups, a.tscale, FMT == F_FP8 ? 448.0f : 2688.0f);
  launch_all<FMT>(b, p, kNormGroups, st);
  return hipGetLastError();
}

hipError_t launch_rms_norm(int fmt, const NormArgs& a, bool static_scale, hipStream_t st) {
  if (a.rows == 0 || a.cols == 0) {
    if (static_scale || !a.tscale) return hipSuccess;
    hipLaunchKernelGGL(k_norm_empty, dim3(1), dim3(1), 0, st, a.tscale);
    return hipGetLastError();
  }
  if (fmt == F_FP8 && !static_scale) return launch_dynamic<F_FP8>(a, st);
  if (fmt == F_NVFP4 && !static_scale) return launch_dynamic<F_NVFP4>(a, st);
  const NormPlan p = norm_plan(a.rows, a.cols);
  if (fmt == F_FP8) launch_all<F_FP8>(a, p, kNormGroups, st);
  else if (fmt == F_NVFP4) launch_all<F_NVFP4>(a, p, kNormGroups, st);
  else if (fmt == F_MXFP4) launch_all<F_MXFP4>(a, p, kNormGroups, st);
  else if (fmt == F_MXFP8) launch_all<F_MXFP8>(a, p, kNormGroups, st);
  else launch_all<F_BF16>(a, p, kNormGroups, st);
  return hipGetLastError();
}

}  // namespace qg
