// Rows in 8 bits: with a scale for each row, as the products of 8-bit integers take them, and with a power of two for every 32
// columns, as checkpoints of activations.  Bound by memory: every row is read once and written once.
#include <algorithm>

#include "moe_act.h"
#include "moe_codes.h"

namespace sptir {
namespace {

struct Rows8 {
  int64_t n_rows;
  int32_t width;
  int32_t lanes, shift;  // of a row: 2^shift from 8 to 64, or 256
  const void* X;  // quantise, pack
  int64_t ldx;
  int8_t* Q;
  int64_t ldq;
  float* scales;       // quantise
  uint8_t* exponents;  // pack, unpack
  int64_t ld_exponents;
  void* Y;  // unpack
  int64_t ldy;
  int32_t least;  // pack: an exponent's least byte ...
  uint32_t top;   // ... and the one with which 64 is past the type's range
};

// The first `many` elements of a 16-byte word of T, zeros behind them
template <typename T>
struct Word {
  static constexpr int kN = 16 / sizeof(T);
  u32x4 w;
  __device__ inline float at(int i) const {
    if constexpr (sizeof(T) == 4) {
      const uint32_t bits = w[i];  // (a bit_cast of an element of a vector takes the first one)
      return __builtin_bit_cast(float, bits);
    } else {
      const uint16_t bits = (uint16_t)(w[i / 2] >> i % 2 * 16);
      return to_float(__builtin_bit_cast(T, bits));
    }
  }
};
template <typename T>
__device__ inline Word<T> read_word(const T* p, int many) {
  Word<T> w;
  if (many >= Word<T>::kN) __builtin_memcpy(&w.w, p, 16);
  else w.w = read_elements(p, max(many, 0));
  return w;
}
// The low bytes of kN numbers
template <int kN>
__device__ inline void write_codes(int8_t* p, int many, const uint32_t (&q)[kN]) {
  uint32_t w[kN / 4];
#pragma unroll
  for (int i = 0; i < kN / 4; ++i) {
    const uint32_t lo = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400), hi = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400);
    w[i] = hi << 16 | lo;
  }
  if (many >= kN) {
    __builtin_memcpy(p, w, kN);
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (i < many) p[i] = (int8_t)q[i];
  }
}

// The largest magnitude, as the bits of a T without their sign: those of infinities and NaN are above all others'.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T>
struct Largest {
  uint32_t m = 0;  // (16 bits: of the even and of the odd elements)
  __device__ inline void take(uint32_t bits) {
    if constexpr (sizeof(T) == 4) m = max(m, bits);
    else m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, bits)));
  }
  __device__ inline void take(const Word<T>& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) take(w.w[i] & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu));
  }
  // as a float32
  __device__ inline float value() const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, m);
    else return to_float(__builtin_bit_cast(T, (uint16_t)max(m & 0xffff, m >> 16)));
  }
};
template <int kTurn>
__device__ inline uint32_t turned_bits(uint32_t v) { return __builtin_amdgcn_update_dpp(0, (int)v, 0x120 + kTurn, 0xf, 0xf, false); }

// Rounding by an addition: 1.5 * 2^23 + a number below 2^22 is rounded to a whole number, to even, whose two's complement has the low bits.
constexpr float kRound = 12582912.f;
constexpr float kSure = 0.5f - 0x1p-15f;  // as near the middle as a guess may be

// The whole number nearest to x / s, the even one of two: a guess, one off at most, and what it leaves, which is exact.  (With u the unit of s's
// last place, x and the guess times s are multiples of u / 2; what is left, up to s / 2, is below 2^24 of them, and where it is more
// its rounding keeps it so.)
__device__ inline int nearest(float x, float s, float inverse) {
  float n = rintf(x * inverse);
  const float left = fmaf(-n, s, x), half = 0.5f * s;
  const bool odd = (int)n & 1;
  if (left > half || (left == half && odd)) n += 1.f;
  if (left < -half || (left == -half && odd)) n -= 1.f;
  return (int)fminf(fmaxf(n, -127.f), 127.f);
}

// A group of lanes per row: the largest magnitude, then the codes, for which the row comes from the caches.  An element's code is x times the
// reciprocal of the scale, rounded: within 2^-16 of the quotient, so the nearest one wherever that is not next to the middle of two; such elements
// are done with care, one at a time.  (Of float32's one in 2^14; of those of 16 bits all that are half of the row's largest, which is next to the
// middle between 63 and 64: somewhere in most words.)  16,384 x 4096 of bf16 with its call 46.6 us, 4.3 TB/s (whole words done with care 50); with rows
// held in registers between the two, whose code was five times as long, 73 us.
template <typename T>
__global__ __launch_bounds__(256) void k_moe_quantise(Rows8 p) {
  constexpr int kN = Word<T>::kN;
  __shared__ uint32_t part[4];
  const int lane = threadIdx.x & (p.lanes - 1);
  const int64_t groups = (int64_t)gridDim.x << (8 - p.shift);
  const int apart = p.lanes * kN;
  for (int64_t r = ((int64_t)blockIdx.x << (8 - p.shift)) + (threadIdx.x >> p.shift); r < p.n_rows; r += groups) {
    const T* x = (const T*)p.X + r * p.ldx;
    Largest<T> most;
#pragma unroll 4
    for (int c = lane * kN; c < p.width; c += apart) most.take(read_word<T>(x + c, p.width - c));
    if (p.lanes >= 16) {
      most.take(turned_bits<8>(most.m));
      most.take(turned_bits<4>(most.m));
      most.take(turned_bits<2>(most.m));
      most.take(turned_bits<1>(most.m));
      for (int d = min(p.lanes, 64) / 2; d >= 16; d >>= 1) most.take((uint32_t)__shfl_xor((int)most.m, d));
    } else {
      for (int d = 4; d; d >>= 1) most.take((uint32_t)__shfl_xor((int)most.m, d));
    }
    if (p.lanes > 64) {
      if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most.m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 4; ++w) most.take(part[w]);
      __syncthreads();
    }
    const float m = most.value();
    const bool finite = m < INFINITY;
    const float s = finite ? m / 127.f : __builtin_nanf("");
    if (lane == 0) p.scales[r] = s;
    // (the reciprocal of a scale near float32's smallest would be infinite; a row of zeros has the scale 0 and the codes 0)
    const bool careful = m < 0x1p-60f || !finite;
    const float up = careful ? 0x1p64f : 1.f, su = s * up, inverse = finite && s > 0.f ? 1.f / su : 0.f;
#pragma unroll 1
    for (int c = lane * kN; c < p.width; c += apart) {
      const Word<T> w = read_word<T>(x + c, p.width - c);
      uint32_t q[kN];
      float near = 0.f;  // how near the middle the nearest to it is
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float v = w.at(i), sum = fmaf(v, inverse, kRound);
        q[i] = __builtin_bit_cast(uint32_t, sum);
        near = fmaxf(near, fabsf(fmaf(v, inverse, kRound - sum)));
      }
      if (!(near < kSure) || careful) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const float v = w.at(i);
          if (__builtin_expect(careful || !(fabsf(fmaf(v, inverse, kRound - __builtin_bit_cast(float, q[i]))) < kSure), 0))
            q[i] = inverse > 0.f ? (uint32_t)nearest(v * up, su, inverse) : 0u;
        }
      }
      write_codes<kN>(p.Q + r * p.ldq + c, p.width - c, q);
    }
  }
}

// A group of lanes per row; 32 / kN neighbours have a block.  Its exponent is the least with largest < 127.5 * 2^e, so that the largest
// code rounds to 127 at most: with largest = f 2^x, 1 <= f < 2, that is x - 6 where f < 255 / 128, otherwise x - 5, which is the
// carry of 2^16 added to the bits.  Bound by memory: 16,384 x 4096 of bf16 40 us, 5.0 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_moe_pack(Rows8 p) {
  constexpr int kN = Word<T>::kN, kLanes = kMoeBlock / kN;
  const int lane = threadIdx.x & (p.lanes - 1);
  const int64_t groups = (int64_t)gridDim.x << (8 - p.shift);
  const int padded = (p.width + kMoeBlock - 1) / kMoeBlock * kMoeBlock;  // (a block's lanes stay together)
  for (int64_t r = ((int64_t)blockIdx.x << (8 - p.shift)) + (threadIdx.x >> p.shift); r < p.n_rows; r += groups) {
    for (int c = lane * kN; c < padded; c += p.lanes * kN) {
      const Word<T> w = read_word<T>((const T*)p.X + r * p.ldx + c, p.width - c);
      Largest<T> most;
      most.take(w);
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) most.take((uint32_t)__shfl_xor((int)most.m, d));
      const uint32_t m = __builtin_bit_cast(uint32_t, most.value());
      const bool finite = m < 0x7f800000u;
      const uint32_t e = finite ? (uint32_t)max((int)((m + 0x10000u) >> 23) - 6, p.least) : 255u;
      const float inverse = __builtin_bit_cast(float, (254u - min(e, 253u)) << 23);
      uint32_t q[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) q[i] = __builtin_bit_cast(uint32_t, fmaf(w.at(i), inverse, kRound));
      if (e >= p.top) {  // (or 255: the codes 0)
#pragma unroll
        for (int i = 0; i < kN; ++i) q[i] = finite ? (uint32_t)(int)fminf(fmaxf(rintf(w.at(i) * inverse), -63.f), 63.f) : 0;
      }
      write_codes<kN>(p.Q + r * p.ldq + c, p.width - c, q);
      if (lane % kLanes == 0) p.exponents[r * p.ld_exponents + c / kMoeBlock] = (uint8_t)e;
    }
  }
}

template <typename T, int kAct>
__device__ inline void act_word(float (&v)[Word<T>::kN]) {
#pragma unroll
  for (int i = 0; i < Word<T>::kN; ++i) v[i] = act_value<kAct, T>(v[i]);
}

// A group of lanes per row, a word of Y each.  Bound by memory: 16,384 x 4096 codes to 2048 of bf16 through swiglu 23 us, 5.9 TB/s,
// since the memory-side cache has part of the codes.
template <typename T>
__global__ __launch_bounds__(256) void k_moe_unpack(Rows8 p, int32_t act) {
  constexpr int kN = Word<T>::kN;
  const bool gated = act == SPTIR_ACT_SWIGLU;
  const int lane = threadIdx.x & (p.lanes - 1), width = gated ? p.width / 2 : p.width;
  const int64_t groups = (int64_t)gridDim.x << (8 - p.shift);
  for (int64_t r = ((int64_t)blockIdx.x << (8 - p.shift)) + (threadIdx.x >> p.shift); r < p.n_rows; r += groups) {
    const int8_t* q = p.Q + r * p.ldq;
    const uint8_t* e = p.exponents + r * p.ld_exponents;
    for (int c = lane * kN; c < width; c += p.lanes * kN) {
      float v[kN], u[kN];
      Kept<kN, true> kept;
      kept.read(q, e, c, width - c);
      if (gated) {
        Kept<kN, false> pair;
        pair.read(q, e, width + c, width - c);
        pair.values(u);
        kept.values(v);
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = act_gated<T>(v[i], u[i]);
      } else {
        kept.values(v);
        if (act == SPTIR_ACT_RELU) act_word<T, SPTIR_ACT_RELU>(v);
        else if (act == SPTIR_ACT_GELU) act_word<T, SPTIR_ACT_GELU>(v);
        else if (act == SPTIR_ACT_SILU) act_word<T, SPTIR_ACT_SILU>(v);
      }
      T o[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) o[i] = from_float<T>(v[i]);
      u32x4 word;
      __builtin_memcpy(&word, o, 16);
      write_word((T*)p.Y + r * p.ldy + c, word, width - c);
    }
  }
}

// lanes of a row of so many 16-byte words, and the grid
dim3 rows8_grid(int64_t words, Rows8* p) {
  p->lanes = 8;
  while (p->lanes < 64 && p->lanes < words) p->lanes *= 2;
  if (words > 256) p->lanes = 256;
  p->shift = 0;
  while (1 << p->shift < p->lanes) ++p->shift;
  const int64_t each = 256 / p->lanes;
  return dim3((unsigned)std::min<int64_t>((p->n_rows + each - 1) / each, 16384));
}

sptir_status_t check_rows8(int32_t type, int64_t n_rows, int32_t width) {
  if (!moe_type_ok(type) || n_rows < 0 || width < 0) return SPTIR_ERR_INVALID_ARG;
  if (n_rows >= (int64_t)INT32_MAX || width > INT32_MAX / 2) return SPTIR_ERR_OVERFLOW;
  return SPTIR_OK;
}

}  // namespace

sptir_status_t moe_unpack(int32_t type, int32_t act, int32_t width, int64_t n_rows, const int8_t* Q, int64_t ldq, const uint8_t* exponents,
                          int64_t ld_exponents, void* Y, int64_t ldy, hipStream_t stream) {
  Rows8 p = {};
  p.n_rows = n_rows;
  p.width = width;
  p.Q = const_cast<int8_t*>(Q); p.ldq = ldq;
  p.exponents = const_cast<uint8_t*>(exponents); p.ld_exponents = ld_exponents;
  p.Y = Y; p.ldy = ldy;
  const int per = 16 / moe_type_bytes(type);
  const dim3 grid = rows8_grid(((act == SPTIR_ACT_SWIGLU ? width / 2 : width) + per - 1) / per, &p);
  moe_with_type(type, [&](auto v) { hipLaunchKernelGGL(k_moe_unpack<decltype(v)>, grid, dim3(256), 0, stream, p, act); });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

}  // namespace sptir

using namespace sptir;

extern "C" sptir_status_t sptir_moe_quantise(int32_t type, int32_t width, int64_t n_rows, const void* X, int64_t ldx, int8_t* Q, int64_t ldq,
                                             float* scales, void* stream) {
  const sptir_status_t st = check_rows8(type, n_rows, width);
  if (st != SPTIR_OK) return st;
  if (ldx < width || ldq < width) return SPTIR_ERR_INVALID_ARG;
  if (n_rows == 0) return SPTIR_OK;
  if (!scales || (width > 0 && (!X || !Q || (const void*)Q == X)) || (const void*)scales == X || (void*)scales == (void*)Q) return SPTIR_ERR_INVALID_ARG;
  Rows8 p = {};
  p.n_rows = n_rows;
  p.width = width;
  p.X = X; p.ldx = ldx;
  p.Q = Q; p.ldq = ldq;
  p.scales = scales;
  const int per = 16 / moe_type_bytes(type);
  const dim3 grid = rows8_grid((width + per - 1) / per, &p);
  moe_with_type(type, [&](auto v) { hipLaunchKernelGGL(k_moe_quantise<decltype(v)>, grid, dim3(256), 0, (hipStream_t)stream, p); });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

extern "C" sptir_status_t sptir_moe_pack(int32_t type, int32_t width, int64_t n_rows, const void* X, int64_t ldx, int8_t* Q, int64_t ldq,
                                         uint8_t* exponents, int64_t ld_exponents, void* stream) {
  const sptir_status_t st = check_rows8(type, n_rows, width);
  if (st != SPTIR_OK) return st;
  if (ldx < width || ldq < width || ld_exponents < moe_blocks(width)) return SPTIR_ERR_INVALID_ARG;
  if (n_rows == 0 || width == 0) return SPTIR_OK;
  if (!X || !Q || !exponents || (const void*)Q == X || (const void*)exponents == X || (void*)exponents == (void*)Q) return SPTIR_ERR_INVALID_ARG;
  Rows8 p = {};
  p.n_rows = n_rows;
  p.width = width;
  p.X = X; p.ldx = ldx;
  p.Q = Q; p.ldq = ldq;
  p.exponents = exponents; p.ld_exponents = ld_exponents;
  // float16 has no smaller unit than 2^-24 and bfloat16's and float32's powers of two begin at 2^-126; 64 * 2^10 and 64 * 2^122 are past their ranges
  p.least = type == SPTIR_F16 ? 127 - 24 : 1;
  p.top = type == SPTIR_F16 ? 127 + 10 : 127 + 122;
  const int per = 16 / moe_type_bytes(type);
  const dim3 grid = rows8_grid((width + per - 1) / per, &p);
  moe_with_type(type, [&](auto v) { hipLaunchKernelGGL(k_moe_pack<decltype(v)>, grid, dim3(256), 0, (hipStream_t)stream, p); });
  SPTIR_HIP(hipGetLastError());
  return SPTIR_OK;
}

extern "C" sptir_status_t sptir_moe_unpack(int32_t type, int32_t activation, int32_t width, int64_t n_rows, const int8_t* Q, int64_t ldq,
                                           const uint8_t* exponents, int64_t ld_exponents, void* Y, int64_t ldy, void* stream) {
  const sptir_status_t st = check_rows8(type, n_rows, width);
  if (st != SPTIR_OK) return st;
  const bool gated = activation == SPTIR_ACT_SWIGLU;
  if (activation < SPTIR_ACT_NONE || activation > SPTIR_ACT_SWIGLU || (gated && width % 2) || ldq < width || ld_exponents < moe_blocks(width) ||
      ldy < (gated ? width / 2 : width))
    return SPTIR_ERR_INVALID_ARG;
  if (n_rows == 0 || width == 0) return SPTIR_OK;
  if (!Y || !Q || !exponents || (const void*)Q == Y || (const void*)exponents == Y) return SPTIR_ERR_INVALID_ARG;
  return moe_unpack(type, activation, width, n_rows, Q, ldq, exponents, ld_exponents, Y, ldy, (hipStream_t)stream);
}
