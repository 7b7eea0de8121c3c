// Shared device code of the microscaled 4-bit (MXFP4) operators: the packed layout's
// operand fragments (include/polyq.h, polyq_mx_bytes; sizes in mx_plan.h), element
// types and the gated block's activations.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mx_plan.h"

namespace polyq {
namespace mx {

constexpr int kNanScale = 255;

typedef int i4v __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Offset of a chunk's codes and of its record's scales inside a tile.
__host__ __device__ inline int64_t chunk_offset(int c) {
  return static_cast<int64_t>(c >> 2) * kRecBytes + kScaleBytes + (c & 3) * kChunkBytes;
}
__host__ __device__ inline int64_t scale_offset(int c) { return static_cast<int64_t>(c >> 2) * kRecBytes; }

// A buffer of `bytes` bytes, at most 2^32 - 1 of them in reach; reads behind it return 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const uint8_t* base, int64_t bytes) {
  const uint32_t reach = bytes > 0xFFFFFFFFll ? 0xFFFFFFFFu : static_cast<uint32_t>(bytes);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), static_cast<short>(0), static_cast<int>(reach),
                                           0x00020000);
}

// 16 bytes per lane from a buffer straight into LDS, lane l's at lds + 16 l.  (The buffer form is counted
// precisely by the compiler's waits; after the global form it waits for every load in flight.)
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t buf, uint8_t* lds, int lane_offset, int offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)lds, 16, lane_offset, offset, 0, 0);
}

// 2^(byte - 127) as the float whose exponent the conversions take; of 255, an infinity, they make NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 0 ? 0x00400000u : byte << 23);
}

// ------------------------------------------------------------------ quantizing a row
// Lane's 8 values of a row from channel k0, as fp32; zero past `k`.  VEC: the row is on 16 bytes and k a multiple
// of a 16-byte vector.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int k0, int k, float* v) {
  if (VEC) {
    typedef T tv __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
      tv r = {};
      if (k0 + h * N < k) r = *reinterpret_cast<const tv*>(row + k0 + h * N);
#pragma unroll
      for (int i = 0; i < N; ++i) v[h * N + i] = static_cast<float>(r[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k0 + i < k ? static_cast<float>(row[k0 + i]) : 0.f;
  }
}
// The codes of those 8 values and, the same in the block's four lanes, its scale byte.
__device__ __forceinline__ uint32_t quantize8(const float* v, uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  const int e = static_cast<int>(top >> 23);
  *byte = static_cast<uint32_t>(max(e - 2, 0));
  const float s = scale_value(*byte);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], s, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], s, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], s, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], s, 3);
  if (e == 255) *byte = kNanScale, code = 0;
  return code;
}
// A record of 16 rows x 512 channels in LDS.  A block of 16 rows is 272 bytes from the next, so that the 16 blocks of
// a row fall into different banks.
struct Record {
  static constexpr int kPitch = kRows * 16 + 16;
  uint8_t codes[16 * kPitch];
  uint8_t scales[kScaleBytes];
  // the 4 bytes of row `row` that hold lane `lane`'s 8 values
  __device__ __forceinline__ uint32_t* at(int row, int lane) {
    return reinterpret_cast<uint32_t*>(&codes[(lane >> 2) * kPitch + row * 16 + (lane & 3) * 4]);
  }
  // the scale byte of that block: chunk lane / 16, its block (lane / 4) % 4
  __device__ __forceinline__ uint8_t* scale(int row, int lane) {
    return &scales[(((lane >> 2) & 3) * kRows + row) * 4 + (lane >> 4)];
  }
  // lane `lane`'s fragment of chunk c
  __device__ __forceinline__ u4v* fragment(int c, int lane) {
    return reinterpret_cast<u4v*>(&codes[(c * 4 + (lane >> 4)) * kPitch + (lane & 15) * 16]);
  }
};

// 16 rows x 128 channels of A (rows of D) by 16 rows x 128 channels of B (columns of D), every
// 32-channel block of a row with its scale in byte `SEL` of that lane's word.  Products
// of two 4-bit values are exact and the sums are kept in fp32.
template <int SEL_A, int SEL_B>
__device__ __forceinline__ f4 mfma_mx(i4v a, i4v b, f4 c, int sa, int sb) {
  const i8v x = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, y = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, SEL_A, sa, SEL_B, sb);
}

// The same for 32 rows x 64 channels of A and B: two row tiles, two of a chunk's four blocks; lane l has
// row l % 32 and block l / 32, and of D column l % 32, rows 8 i + 4 (l / 32) + 0 .. 3 in elements 4 i .. .
// Twice the work an instruction: a loop of nothing but these reaches 6.5 to 7.0 PFLOP/s on random values, of the smaller
// ones 5.2 to 6.0 (on constant ones, which take less power, 8.4 to 9.1 against 6.1 to 6.9).
template <int SEL_A, int SEL_B>
__device__ __forceinline__ f16v mfma_mx32(i4v a, i4v b, f16v c, int sa, int sb) {
  const i8v x = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, y = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, SEL_A, sa, SEL_B, sb);
}

// ------------------------------------------------------------------ element types
struct F32 { typedef float type; };
struct F16 { typedef _Float16 type; };
struct BF16 { typedef __bf16 type; };

inline bool float_type(int t) { return t == POLYQ_MX_F32 || t == POLYQ_MX_F16 || t == POLYQ_MX_BF16; }
inline int type_bytes(int t) { return t == POLYQ_MX_F32 ? 4 : 2; }

// Four consecutive elements; vec: p is aligned to all four.
template <class T>
__device__ __forceinline__ f4 load4(const T* p, bool vec, int valid) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  f4 v = {0.f, 0.f, 0.f, 0.f};
  if (vec && valid >= 4) {
    const t4 r = *reinterpret_cast<const t4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(r[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < valid) v[i] = static_cast<float>(p[i]);
  }
  return v;
}
template <class T>
__device__ __forceinline__ void store4(T* p, f4 v, bool vec, int valid) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  if (vec && valid >= 4) {
    t4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = static_cast<T>(v[i]);
    *reinterpret_cast<t4*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < valid) p[i] = static_cast<T>(v[i]);
  }
}
// Of 16 consecutive 16-bit elements, lanes l and l + 32 hold 0 .. 3 and 4 .. 7 in `a`, 8 .. 11 and 12 .. 15 in `b`
// (what a 32x32 product leaves in two groups of four accumulators).  The halves trade places, so that lane l
// gets the first eight and lane l + 32 the last: one store of 16 bytes a lane in place of two of 8.
template <class T4>
__device__ __forceinline__ u4v pack_halves(T4 a, T4 b) {
  const u2v u = __builtin_bit_cast(u2v, a), v = __builtin_bit_cast(u2v, b);
  const u2v x = __builtin_bit_cast(u2v, __builtin_amdgcn_permlane32_swap(u.x, v.x, false, false));
  const u2v y = __builtin_bit_cast(u2v, __builtin_amdgcn_permlane32_swap(u.y, v.y, false, false));
  return u4v{x.x, y.x, x.y, y.y};
}
// Elements (a at `to`, b eight further on) of one row; `to` is the lane's place in `a`.  All there, rows on 16 bytes.
template <class T>
__device__ __forceinline__ void store_pair(T* to, f4 a, f4 b, int upper) {
  if constexpr (sizeof(T) == 4) {
    store4(to, a, true, 4);
    store4(to + 8, b, true, 4);
  } else {
    typedef T t4 __attribute__((ext_vector_type(4)));
    t4 p, q;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = static_cast<T>(a[i]), q[i] = static_cast<T>(b[i]);
    *reinterpret_cast<u4v*>(to + upper * 4) = pack_halves(p, q);
  }
}
// 32 rows x 64 columns of an output, two 32x32 products side by side whose lane l has row l % 32 and columns 8 r + 4 (l
// / 32) .. + 3 in elements 4 r .. of each, by way of a wave's own 4 or 8 KiB of LDS to rows of `pitch` elements at
// `out`, in pieces of 16 bytes of which 8 or 16 lanes make a row: a store then touches 8 or 4 rows and not 32.
// Only pieces of rows < rows_left and columns < cols_left are written; every piece is all there or not at all, and on
// 16 bytes.  Pieces are swizzled by row so that neighbouring rows fall into different banks.
template <class T>
__device__ __forceinline__ void store_rows(uint8_t* lds, T* out, int64_t pitch, const f16v& a, const f16v& b, int lane,
                                           int rows_left, int cols_left) {
  constexpr int UNITS = 64 * sizeof(T) / 16, PER = 16 / sizeof(T);  // pieces of a row, elements of a piece
  const int row = lane & 31, upper = lane >> 5;
  uint8_t* mine = lds + row * (UNITS * 16);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const f16v& d = t == 0 ? a : b;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f4*>(mine + (((t * 8 + r * 2 + upper) ^ (row & 7)) * 16)) =
            f4{d[4 * r], d[4 * r + 1], d[4 * r + 2], d[4 * r + 3]};
    } else {
      typedef T t4 __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        t4 p, q;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = static_cast<T>(d[4 * r + i]), q[i] = static_cast<T>(d[4 * r + 4 + i]);
        *reinterpret_cast<u4v*>(mine + (((t * 4 + r + upper) ^ (row & 7)) * 16)) = pack_halves(p, q);
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int s = 0; s < UNITS / 2; ++s) {
    const int at = s * (64 / UNITS) + lane / UNITS, unit = lane % UNITS;
    const u4v v = *reinterpret_cast<const u4v*>(lds + at * (UNITS * 16) + (unit ^ (at & 7)) * 16);
    if (at < rows_left && unit * PER < cols_left) *reinterpret_cast<u4v*>(out + at * pitch + unit * PER) = v;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
// The same with the type known at run time.
__device__ __forceinline__ f4 load4(const void* base, int type, int64_t at, bool vec, int valid) {
  if (type == POLYQ_MX_F32) return load4(static_cast<const float*>(base) + at, vec, valid);
  if (type == POLYQ_MX_F16) return load4(static_cast<const _Float16*>(base) + at, vec, valid);
  return load4(static_cast<const __bf16*>(base) + at, vec, valid);
}
__device__ __forceinline__ void store4(void* base, int type, int64_t at, f4 v, bool vec, int valid) {
  if (type == POLYQ_MX_F32) store4(static_cast<float*>(base) + at, v, vec, valid);
  else if (type == POLYQ_MX_F16) store4(static_cast<_Float16*>(base) + at, v, vec, valid);
  else store4(static_cast<__bf16*>(base) + at, v, vec, valid);
}

// bf16 term `term` of `terms` of fp32 values, and what it leaves of them (nothing of one that is not finite).  A term is the
// nearest bf16 value; but one that would be an infinity (from 2^128 - 2^119 on) and the second of three are cut towards
// zero, so that no sum of the first terms lies past the largest float.  One term is within 2^-8 of the value, two are
// within 2^-17, and three are exactly the value, but for bits below 2^-133, the smallest of bf16.
__device__ __forceinline__ bf16x4 next_terms(f4* v, int term, int terms) {
  const bool cut = term > 0 && term + 1 < terms;
  bf16x4 t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = (*v)[i];
    t[i] = static_cast<__bf16>(x);
    if (__builtin_isfinite(x) && (cut || !__builtin_isfinite(static_cast<float>(t[i]))))
      t[i] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(__builtin_bit_cast(uint32_t, x) >> 16));
    (*v)[i] = __builtin_isfinite(x) ? x - static_cast<float>(t[i]) : 0.f;
  }
  return t;
}

// Byte offset of four consecutive elements (row, col ..) of a plane: blocks of 32 rows x 16 columns, a row of
// blocks after the other, rows of 32 bytes in a block.
__device__ __forceinline__ int64_t plane_at(int row, int col, int cols_pad) {
  return (static_cast<int64_t>(row >> 5) * (cols_pad >> 4) + (col >> 4)) * 1024 + (row & 31) * 32 + (col & 15) * 2;
}

// Two transposing LDS reads: lane j of 16 gets column j of the four rows those 16 lanes address with p (8 bytes each,
// four lanes a row), and of the four they address with q.
__device__ __forceinline__ bf16x8 read_transposed(const uint8_t* p, const uint8_t* q) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  union {
    s4 h[2];
    bf16x8 v;
  } u;
  u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(p));
  u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(q));
  return u.v;
}

constexpr int kBlockBytes = 1024;  // 32 x 16 bf16

// A fragment (16 tokens x 128 channels) as four bf16 blocks of 32 channels x 16 tokens, rows of 32 bytes, at
// [channel / 32][tile]: the lanes convert 32 values each into a wave's own 4 KiB of LDS, blocks of 16 tokens x 32
// channels, and read them transposed.
__device__ __forceinline__ void transpose_chunk(uint8_t* lds, i4v codes, uint32_t byte, int lane, uint8_t* out, int chunk,
                                                int tile, int m_tiles, int c_tiles) {
  const float s = scale_value(byte);
  uint8_t* block = lds + (lane >> 4) * kBlockBytes;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t code = static_cast<uint32_t>(codes[w]);
    const u4v v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3))};
    *reinterpret_cast<u4v*>(block + (lane & 15) * 64 + w * 16) = v;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // Lane group h = lane / 16 of a block: channels 16 (h & 1) .. + 15, tokens 8 (h >> 1) .. + 7.
  const int i = lane & 15, half = (lane >> 4) & 1, upper = lane >> 5;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int ct = chunk * 4 + q;
    const uint8_t* p = lds + q * kBlockBytes + (upper * 8 + (i >> 2)) * 64 + half * 32 + (i & 3) * 8;
    const bf16x8 v = read_transposed(p, p + 4 * 64);
    if (ct < c_tiles)
      *reinterpret_cast<bf16x8*>(out + (static_cast<int64_t>(ct) * m_tiles + tile) * kBlockBytes + (half * 16 + i) * 32 + upper * 16) = v;
  }
}

// ------------------------------------------------------------------ activations
// act(g) and, if asked for, act'(g), in fp32:
//   silu       g s,  s = 1 / (1 + exp(-g));        s (1 + g (1 - s))
//   gelu       g P,  P the normal distribution;    P + g exp(-g^2 / 2) / sqrt(2 pi)
//   gelu_tanh  g s,  s = 1 / (1 + exp(-2 z)) = (1 + tanh z) / 2,
//              z = sqrt(2 / pi) (g + 0.044715 g^3);  s + g s (1 - s) 2 z'
// with the hardware's exp2 and reciprocal, each good to a unit of 2^-23: s and P are within
// 2^-20 of themselves for |g| < 3, and as far again as the rounding of the exponent, (1 + g^2)
// 2^-24, carries them in the tails.  With the library's exp and division in their place a gated
// block (silu) of 2000 tokens x 13824 x 5120 took 176 us, and with these 157.
// P(-a) = exp(-a^2 / 2) t p(t), t = 1 / (1 + 0.318 a): p, of degree 9, was fitted to
// exp(z^2) erfc(z) / (2 t) over z = a / sqrt 2 >= 0 (least squares reweighted to an even relative
// error: 3.3e-8).
template <int ACT>
__device__ __forceinline__ float activation(float g, float* slope) {
  const float log2e = 1.44269504088896341f;
  if constexpr (ACT == POLYQ_ACT_GELU) {
    const float a = __builtin_fabsf(g);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.318198051533946f * a);
    float p = -0.02069910056889057f;
    p = p * t + 0.09535936266183853f;
    p = p * t - 0.15031923353672028f;
    p = p * t + 0.07122802734375f;
    p = p * t - 0.011194917373359203f;
    p = p * t + 0.059980735182762146f;
    p = p * t + 0.08762495964765549f;
    p = p * t + 0.11413593590259552f;
    p = p * t + 0.12694157660007477f;
    p = p * t + 0.12694266438484192f;
    const float e = __builtin_amdgcn_exp2f(a * a * (-0.5f * log2e));
    const float q = p * t * e, P = g < 0.f ? q : 1.f - q;
    if (slope) *slope = P + g * (0.39894228040143268f * e);
    return g * P;
  }
  if constexpr (ACT == POLYQ_ACT_GELU_TANH) {
    const float a = 0.79788456080286536f, b = 0.044715f, g2 = g * g;
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.f * log2e * a * g * (1.f + b * g2)));
    // s (1 - s) is 0 where z' overflows the product
    if (slope) *slope = s + (s == 0.f || s == 1.f ? 0.f : g * s * (1.f - s) * 2.f * a * (1.f + 3.f * b * g2));
    return g * s;
  }
  const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-log2e * g));
  if (slope) *slope = s * (1.f + g * (1.f - s));
  return g * s;
}
// The same with the activation known at run time.
__device__ __forceinline__ float activation(int act, float g, float* slope) {
  if (act == POLYQ_ACT_GELU) return activation<POLYQ_ACT_GELU>(g, slope);
  if (act == POLYQ_ACT_GELU_TANH) return activation<POLYQ_ACT_GELU_TANH>(g, slope);
  return activation<POLYQ_ACT_SILU>(g, slope);
}
inline bool valid_act(int act) { return act == POLYQ_ACT_SILU || act == POLYQ_ACT_GELU || act == POLYQ_ACT_GELU_TANH; }

// ------------------------------------------------------------------ host side
inline bool valid_shape(int32_t rows, int32_t k) {
  return rows >= 1 && rows <= POLYQ_MAX_N && k >= 1 && k <= POLYQ_MAX_K;
}
inline polyq_status launched() { return hipGetLastError() == hipSuccess ? POLYQ_OK : POLYQ_ERR_DEVICE; }
inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// x [rows][k] into the packed layout and, if asked for, into transposed blocks (transpose_chunk; rows padded to 64);
// either may be null (arguments checked by the caller).
polyq_status launch_quantize(const void* x, int type, int32_t rows, int32_t k, void* packed, hipStream_t st,
                             void* transposed = nullptr);

// dg and du of the gated block as bf16 planes [terms][2][m_pad][n_pad] in blocks (plane_at; zero behind m and
// n), whose sum over the terms is the fp32 value as near as next_terms brings it.  x is packed.
polyq_status launch_gated_grad(const void* gate, const void* up, const void* x, const void* dh, int dh_type, int32_t m,
                               int32_t n, int32_t k, int act, void* planes, int terms, int32_t m_pad, int32_t n_pad,
                               hipStream_t st);

}  // namespace mx
}  // namespace polyq
