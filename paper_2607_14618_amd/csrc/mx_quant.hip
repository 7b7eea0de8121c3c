// Microscaled 4-bit floating point: quantization into the packed layout, and back, and
// the packing of a checkpoint's codes and scales.
//
// A block of 32 consecutive values of a row shares the scale 2^e, e = floor(log2 max|v|)
// - 2, so that the largest magnitude lies in [4, 8) times 2^e; v / 2^e is rounded to the
// nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, what lies above 6 to 6.
// e is the exponent field of the largest magnitude less 2 (0 at least), and the
// division by a power of two is exact, so nothing rounds but the value itself.  A block
// that holds an infinity or a NaN gets the NaN scale: all of it is NaN.
//
// What bounds it: memory; 2 to 4 bytes are read and 17/32 written per value.  A wave
// takes one record, 16 rows x 512 values: row by row the 64 lanes read 8 values each (1
// or 2 KiB in a row), form the block's maximum over 4 lanes and convert; the codes meet
// in LDS, from where they leave as whole 1 KiB fragments.  A block in LDS is 272 bytes
// apart, so that the 16 blocks of a row fall into different banks.
#include <hip/hip_runtime.h>

#include "mx.h"

namespace polyq {
namespace mx {
namespace {

constexpr int kWaves = 4;
constexpr int kBlockPitch = kRows * 16 + 16;  // bytes of a block of 16 rows in LDS

struct Record {  // one wave's LDS
  uint8_t codes[16 * kBlockPitch];
  uint32_t scales[64];
};

// LDS address of the 4 bytes of row `row` that lane `lane`'s 8 values occupy.
__device__ __forceinline__ int code_slot(int row, int lane) { return (lane >> 2) * kBlockPitch + row * 16 + (lane & 3) * 4; }

// Lane's 8 values of a row (k0 = its first channel), as fp32; zero past `k`.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int k0, int k, float* v) {
  if (VEC) {  // row is 16-byte aligned and k a multiple of the vector
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

template <class T, bool VEC>
__global__ __launch_bounds__(64 * kWaves) void mx_quantize_kernel(const T* __restrict__ x, uint8_t* __restrict__ packed,
                                                                  int rows, int k, int records, int64_t jobs) {
  __shared__ Record lds[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  if (job >= jobs) return;  // waves are independent: no barrier follows
  const int tile = static_cast<int>(job / records), rec = static_cast<int>(job % records);
  Record& r = lds[wave];
  const int k0 = rec * kRec + lane * 8;
  const int valid = min(kRows, rows - tile * kRows);
  constexpr int U = sizeof(T) == 4 ? 4 : 8;  // rows in flight
  uint8_t* sc = reinterpret_cast<uint8_t*>(r.scales);
  for (int i0 = 0; i0 < kRows; i0 += U) {
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
      if (i0 + u < valid) load8<T, VEC>(x + (static_cast<int64_t>(tile) * kRows + i0 + u) * k, k0, k, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, v[u][i]) & 0x7fffffffu);
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
      top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
      const int e = static_cast<int>(top >> 23);
      uint32_t byte = static_cast<uint32_t>(max(e - 2, 0));
      const float s = scale_value(byte);
      uint32_t code = 0;
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[u][0], v[u][1], s, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[u][2], v[u][3], s, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[u][4], v[u][5], s, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[u][6], v[u][7], s, 3);
      if (e == 255) byte = kNanScale, code = 0;
      // rows behind the last and channels behind k: code 0 with scale 1
      const bool none = i0 + u >= valid || rec * kRec + (lane >> 2) * kBlock >= k;
      *reinterpret_cast<uint32_t*>(&r.codes[code_slot(i0 + u, lane)]) = none ? 0u : code;
      if ((lane & 3) == 0) {  // block lane / 4 of the record: chunk lane / 16, its block (lane / 4) % 4
        const int q = (lane >> 2) & 3;
        sc[(q * kRows + i0 + u) * 4 + (lane >> 4)] = static_cast<uint8_t>(none ? 127u : byte);
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  uint8_t* out = packed + tile * tile_bytes(k) + static_cast<int64_t>(rec) * kRecBytes;
  reinterpret_cast<uint32_t*>(out)[lane] = r.scales[lane];
  const int chunks = min(4, chunks_of(k) - rec * 4);
  for (int c = 0; c < chunks; ++c) {
    const u4v w = *reinterpret_cast<const u4v*>(&r.codes[(c * 4 + (lane >> 4)) * kBlockPitch + (lane & 15) * 16]);
    *reinterpret_cast<u4v*>(out + kScaleBytes + c * kChunkBytes + lane * 16) = w;
  }
}

template <class T, bool VEC>
__global__ __launch_bounds__(64 * kWaves) void mx_dequantize_kernel(const uint8_t* __restrict__ packed, T* __restrict__ out,
                                                                    int rows, int k, int records, int64_t jobs) {
  __shared__ Record lds[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  if (job >= jobs) return;
  const int tile = static_cast<int>(job / records), rec = static_cast<int>(job % records);
  Record& r = lds[wave];
  const uint8_t* in = packed + tile * tile_bytes(k) + static_cast<int64_t>(rec) * kRecBytes;
  const int chunks = min(4, chunks_of(k) - rec * 4);
  r.scales[lane] = reinterpret_cast<const uint32_t*>(in)[lane];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (c < chunks) {
      const u4v w = *reinterpret_cast<const u4v*>(in + kScaleBytes + c * kChunkBytes + lane * 16);
      *reinterpret_cast<u4v*>(&r.codes[(c * 4 + (lane >> 4)) * kBlockPitch + (lane & 15) * 16]) = w;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const uint8_t* sc = reinterpret_cast<const uint8_t*>(r.scales);
  const int k0 = rec * kRec + lane * 8, valid = min(kRows, rows - tile * kRows);
  if (k0 >= k) return;  // also the lanes of chunks that are not there
  const int q = (lane >> 2) & 3;
#pragma unroll 4
  for (int i = 0; i < valid; ++i) {
    const uint32_t code = *reinterpret_cast<const uint32_t*>(&r.codes[code_slot(i, lane)]);
    const uint32_t byte = sc[(q * kRows + i) * 4 + (lane >> 4)];
    const float s = scale_value(byte);
    float v[8];
    typedef float f2 __attribute__((ext_vector_type(2)));
    f2 p;
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0), v[0] = p.x, v[1] = p.y;
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1), v[2] = p.x, v[3] = p.y;
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2), v[4] = p.x, v[5] = p.y;
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3), v[6] = p.x, v[7] = p.y;
    T* row = out + (static_cast<int64_t>(tile) * kRows + i) * k;
    if (VEC) {
      typedef T tv __attribute__((ext_vector_type(16 / sizeof(T))));
      constexpr int N = 16 / sizeof(T);
#pragma unroll
      for (int h = 0; h < 8 / N; ++h) {
        tv w;
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = static_cast<T>(v[h * N + j]);
        if (k0 + h * N < k) *reinterpret_cast<tv*>(row + k0 + h * N) = w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k0 + j < k) row[k0 + j] = static_cast<T>(v[j]);
    }
  }
}

// A checkpoint's matrix (two codes a byte, a scale byte per block) into the packed layout
// and back: a thread per row and block, neighbouring threads on neighbouring rows, that
// is on neighbouring 16-byte slices of the packed side.
template <bool PACK, bool VEC>
__global__ __launch_bounds__(256) void mx_repack_kernel(const uint8_t* __restrict__ in, const uint8_t* __restrict__ in_scales,
                                                        uint8_t* __restrict__ out, uint8_t* __restrict__ out_scales,
                                                        int rows, int k, int64_t jobs) {
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (job >= jobs) return;
  const int slots = records_of(k) * 16;  // blocks of whole records
  const int row16 = static_cast<int>(job % kRows), block = static_cast<int>(job / kRows % slots);
  const int tile = static_cast<int>(job / kRows / slots);
  const int chunk = block >> 2, q = block & 3;
  const int64_t row = static_cast<int64_t>(tile) * kRows + row16;
  const int64_t at = tile * tile_bytes(k) + chunk_offset(chunk) + (q * kRows + row16) * 16;
  const int64_t scale_at = tile * tile_bytes(k) + scale_offset(chunk) + (q * kRows + row16) * 4 + (chunk & 3);
  const int row_bytes = (k + 1) / 2, blocks = div_up(k, kBlock);
  const bool there = row < rows && block < blocks;
  const int bytes = min(16, row_bytes - block * 16);  // of this block
  if (PACK) {
    if (block >= chunks_of(k) * 4) {  // past the last chunk only the scale's place exists
      out[scale_at] = 127;
      return;
    }
    u4v w = {0, 0, 0, 0};
    uint8_t s = 127;
    if (there) {
      const uint8_t* src = in + row * row_bytes + block * 16;
      if (VEC && bytes == 16) {
        w = *reinterpret_cast<const u4v*>(src);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i < bytes) w[i / 4] |= static_cast<uint32_t>(src[i]) << (8 * (i & 3));
      }
      if (block * kBlock + bytes * 2 > k) {  // an odd k: the upper half of the last byte is no channel
        const int last = bytes - 1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (last / 4 == i) w[i] &= ~(0xf0u << (8 * (last & 3)));
      }
      s = in_scales[row * blocks + block];
    }
    *reinterpret_cast<u4v*>(out + at) = w;
    out[scale_at] = s;
  } else if (there) {
    const u4v w = *reinterpret_cast<const u4v*>(in + at);
    uint8_t* dst = out + row * row_bytes + block * 16;
    if (VEC && bytes == 16) {
      *reinterpret_cast<u4v*>(dst) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < bytes) dst[i] = static_cast<uint8_t>(w[i / 4] >> (8 * (i & 3)));
    }
    out_scales[row * blocks + block] = in[scale_at];
  }
}

// rows and k as they have to be, the work-groups of a launch over `jobs` within the grid's limit
polyq_status check_jobs(int64_t groups) { return groups > 0x7FFFFFFFll ? POLYQ_ERR_CAPACITY : POLYQ_OK; }

polyq_status launched() { return hipGetLastError() == hipSuccess ? POLYQ_OK : POLYQ_ERR_DEVICE; }

}  // namespace

polyq_status launch_quantize(const void* x, int type, int32_t rows, int32_t k, void* packed, hipStream_t st) {
  const int records = records_of(k);
  const int64_t jobs = static_cast<int64_t>(tiles_of(rows)) * records, groups = (jobs + kWaves - 1) / kWaves;
  if (check_jobs(groups) != POLYQ_OK) return POLYQ_ERR_CAPACITY;
  const bool vec = aligned(x, 16) && static_cast<int64_t>(k) * type_bytes(type) % 16 == 0;
  uint8_t* out = static_cast<uint8_t*>(packed);
  const dim3 grid(static_cast<uint32_t>(groups)), block(64 * kWaves);
#define POLYQ_MX_QUANTIZE(T)                                                                                        \
  if (vec)                                                                                                          \
    mx_quantize_kernel<T, true><<<grid, block, 0, st>>>(static_cast<const T*>(x), out, rows, k, records, jobs);      \
  else                                                                                                              \
    mx_quantize_kernel<T, false><<<grid, block, 0, st>>>(static_cast<const T*>(x), out, rows, k, records, jobs)
  if (type == POLYQ_MX_F32) {
    POLYQ_MX_QUANTIZE(float);
  } else if (type == POLYQ_MX_F16) {
    POLYQ_MX_QUANTIZE(_Float16);
  } else {
    POLYQ_MX_QUANTIZE(__bf16);
  }
#undef POLYQ_MX_QUANTIZE
  return launched();
}

}  // namespace mx
}  // namespace polyq

using namespace polyq;

extern "C" size_t polyq_mx_bytes(int32_t rows, int32_t k) {
  if (!mx::valid_shape(rows, k)) return 0;
  return static_cast<size_t>(mx::tiles_of(rows)) * static_cast<size_t>(mx::tile_bytes(k));
}

extern "C" polyq_status polyq_mx_quantize(const void* x, int32_t type, int32_t rows, int32_t k, void* packed,
                                          void* stream) {
  if (x == nullptr || packed == nullptr || !mx::float_type(type)) return POLYQ_ERR_ARG;
  if (!mx::valid_shape(rows, k)) return POLYQ_ERR_SHAPE;
  if (!mx::aligned(packed, 256) || !mx::aligned(x, mx::type_bytes(type))) return POLYQ_ERR_ARG;
  return mx::launch_quantize(x, type, rows, k, packed, static_cast<hipStream_t>(stream));
}

extern "C" polyq_status polyq_mx_dequantize(const void* packed, int32_t rows, int32_t k, void* out, int32_t type,
                                            void* stream) {
  if (packed == nullptr || out == nullptr || !mx::float_type(type)) return POLYQ_ERR_ARG;
  if (!mx::valid_shape(rows, k)) return POLYQ_ERR_SHAPE;
  if (!mx::aligned(packed, 256) || !mx::aligned(out, mx::type_bytes(type))) return POLYQ_ERR_ARG;
  const int records = mx::records_of(k);
  const int64_t jobs = static_cast<int64_t>(mx::tiles_of(rows)) * records, groups = (jobs + mx::kWaves - 1) / mx::kWaves;
  if (mx::check_jobs(groups) != POLYQ_OK) return POLYQ_ERR_CAPACITY;
  const bool vec = mx::aligned(out, 16) && static_cast<int64_t>(k) * mx::type_bytes(type) % 16 == 0;
  const uint8_t* in = static_cast<const uint8_t*>(packed);
  const dim3 grid(static_cast<uint32_t>(groups)), block(64 * mx::kWaves);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define POLYQ_MX_DEQUANTIZE(T)                                                                                      \
  if (vec)                                                                                                          \
    mx::mx_dequantize_kernel<T, true><<<grid, block, 0, st>>>(in, static_cast<T*>(out), rows, k, records, jobs);     \
  else                                                                                                              \
    mx::mx_dequantize_kernel<T, false><<<grid, block, 0, st>>>(in, static_cast<T*>(out), rows, k, records, jobs)
  if (type == POLYQ_MX_F32) {
    POLYQ_MX_DEQUANTIZE(float);
  } else if (type == POLYQ_MX_F16) {
    POLYQ_MX_DEQUANTIZE(_Float16);
  } else {
    POLYQ_MX_DEQUANTIZE(__bf16);
  }
#undef POLYQ_MX_DEQUANTIZE
  return mx::launched();
}

extern "C" polyq_status polyq_mx_pack(const uint8_t* codes, const uint8_t* scales, int32_t rows, int32_t k,
                                      void* packed, void* stream) {
  if (codes == nullptr || scales == nullptr || packed == nullptr) return POLYQ_ERR_ARG;
  if (!mx::valid_shape(rows, k)) return POLYQ_ERR_SHAPE;
  if (!mx::aligned(packed, 256)) return POLYQ_ERR_ARG;
  const int64_t jobs = static_cast<int64_t>(mx::tiles_of(rows)) * mx::kRows * mx::records_of(k) * 16;
  const int64_t groups = (jobs + 255) / 256;
  if (mx::check_jobs(groups) != POLYQ_OK) return POLYQ_ERR_CAPACITY;
  const bool vec = mx::aligned(codes, 16) && (k + 1) / 2 % 16 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto kernel = vec ? mx::mx_repack_kernel<true, true> : mx::mx_repack_kernel<true, false>;
  kernel<<<dim3(static_cast<uint32_t>(groups)), dim3(256), 0, st>>>(codes, scales, static_cast<uint8_t*>(packed), nullptr,
                                                                    rows, k, jobs);
  return mx::launched();
}

extern "C" polyq_status polyq_mx_unpack(const void* packed, int32_t rows, int32_t k, uint8_t* codes, uint8_t* scales,
                                        void* stream) {
  if (codes == nullptr || scales == nullptr || packed == nullptr) return POLYQ_ERR_ARG;
  if (!mx::valid_shape(rows, k)) return POLYQ_ERR_SHAPE;
  if (!mx::aligned(packed, 256)) return POLYQ_ERR_ARG;
  const int64_t jobs = static_cast<int64_t>(mx::tiles_of(rows)) * mx::kRows * mx::records_of(k) * 16;
  const int64_t groups = (jobs + 255) / 256;
  if (mx::check_jobs(groups) != POLYQ_OK) return POLYQ_ERR_CAPACITY;
  const bool vec = mx::aligned(codes, 16) && (k + 1) / 2 % 16 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto kernel = vec ? mx::mx_repack_kernel<false, true> : mx::mx_repack_kernel<false, false>;
  kernel<<<dim3(static_cast<uint32_t>(groups)), dim3(256), 0, st>>>(static_cast<const uint8_t*>(packed), nullptr, codes,
                                                                    scales, rows, k, jobs);
  return mx::launched();
}
