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
// What bounds it: memory; 2 to 4 bytes are read and 17/32 written per value.  A work-group
// takes one record, 16 rows x 512 values, a wave four of its rows: the 64 lanes read 8
// values each of a row (1 or 2 KiB in a row), form the block's maximum over 4 lanes and
// convert; the codes meet in LDS, from where they leave as whole 1 KiB fragments.
// 4096 x 13824 bf16: 27.5 us (143 MB, 5.2 TB/s), back 22.2 us; 2000 x 13824 15.5, with the transposed blocks in
// place of the packed form 26 (111 MB).  One token 3.1 us.  A wave per record, its 16 rows one
// after the other, took 33, 21 and 5.4.
#include <hip/hip_runtime.h>

#include "mx.h"

namespace polyq {
namespace mx {
namespace {

constexpr int kWaves = 4, kWaveRows = kRows / kWaves;

// packed, or XT and then xt too: the values once more as transposed blocks, for the weights' gradients.
template <class T, bool VEC, bool XT>
__global__ __launch_bounds__(64 * kWaves) void mx_quantize_kernel(const T* __restrict__ x, uint8_t* __restrict__ packed,
                                                                  uint8_t* __restrict__ xt, int rows, int k, int records,
                                                                  int m_tiles) {
  __shared__ Record r;
  __shared__ uint8_t blocks[XT ? kWaves : 1][4 * kBlockBytes];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = static_cast<int>(blockIdx.x / records), rec = static_cast<int>(blockIdx.x % records);
  const int k0 = rec * kRec + lane * 8, row0 = tile * kRows + wave * kWaveRows;
  float v[kWaveRows][8];
#pragma unroll
  for (int u = 0; u < kWaveRows; ++u) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
    if (row0 + u < rows) load8<T, VEC>(x + static_cast<int64_t>(row0 + u) * k, k0, k, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kWaveRows; ++u) {
    uint32_t byte;
    const uint32_t code = quantize8(v[u], &byte);
    // rows behind the last and blocks behind k: code 0 with scale 1
    const bool none = row0 + u >= rows || rec * kRec + (lane >> 2) * kBlock >= k;
    *r.at(wave * kWaveRows + u, lane) = none ? 0u : code;
    if ((lane & 3) == 0) *r.scale(wave * kWaveRows + u, lane) = static_cast<uint8_t>(none ? 127u : byte);
  }
  __syncthreads();
  const bool there = wave < chunks_of(k) - rec * 4;
  const u4v codes = *r.fragment(wave, lane);
  if (!XT || (packed != nullptr && tile * kRows < rows)) {
    uint8_t* out = packed + tile * tile_bytes(k) + static_cast<int64_t>(rec) * kRecBytes;
    if (there) *reinterpret_cast<u4v*>(out + kScaleBytes + wave * kChunkBytes + lane * 16) = codes;
    if (wave == 0) reinterpret_cast<uint32_t*>(out)[lane] = reinterpret_cast<const uint32_t*>(r.scales)[lane];
  }
  if (XT && there)
    transpose_chunk(blocks[XT ? wave : 0], __builtin_bit_cast(i4v, codes), r.scales[lane * 4 + wave], lane, xt, rec * 4 + wave, tile,
                    m_tiles, div_up(k, 32));
}

template <class T, bool VEC>
__global__ __launch_bounds__(64 * kWaves) void mx_dequantize_kernel(const uint8_t* __restrict__ packed, T* __restrict__ out,
                                                                    int rows, int k, int records) {
  __shared__ Record r;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = static_cast<int>(blockIdx.x / records), rec = static_cast<int>(blockIdx.x % records);
  const uint8_t* in = packed + tile * tile_bytes(k) + static_cast<int64_t>(rec) * kRecBytes;
  if (wave < chunks_of(k) - rec * 4) *r.fragment(wave, lane) = *reinterpret_cast<const u4v*>(in + kScaleBytes + wave * kChunkBytes + lane * 16);
  if (wave == 0) reinterpret_cast<uint32_t*>(r.scales)[lane] = reinterpret_cast<const uint32_t*>(in)[lane];
  __syncthreads();
  const int k0 = rec * kRec + lane * 8;
  if (k0 >= k) return;  // also the lanes of chunks that are not there
#pragma unroll
  for (int u = 0; u < kWaveRows; ++u) {
    const int i = wave * kWaveRows + u;
    if (tile * kRows + i >= rows) return;
    const uint32_t code = *r.at(i, lane);
    const float s = scale_value(*r.scale(i, lane));
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
// is on neighbouring 16-byte slices of the packed side.  Bound by memory: 13824 x 5120 into the packed layout 14.7 us
// (75 MB read and written, 5.1 TB/s), back 15.9; rows of a length that is no multiple of 16 bytes, whose bytes move
// one by one, 5120 x 2977: 14.7 and 21.9 us (16 MB).
template <bool PACK, bool VEC>
__device__ __forceinline__ void repack(const uint8_t* __restrict__ in, const uint8_t* __restrict__ in_scales,
                                       uint8_t* __restrict__ out, uint8_t* __restrict__ out_scales, int rows, int k,
                                       int slots, int64_t job) {
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
template <bool PACK, bool VEC>
__global__ __launch_bounds__(256) void mx_repack_kernel(const uint8_t* __restrict__ in, const uint8_t* __restrict__ in_scales,
                                                        uint8_t* __restrict__ out, uint8_t* __restrict__ out_scales,
                                                        int rows, int k, int64_t jobs) {
  const int slots = records_of(k) * 16;  // blocks of whole records
  for (int64_t job = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; job < jobs; job += static_cast<int64_t>(gridDim.x) * 256)
    repack<PACK, VEC>(in, in_scales, out, out_scales, rows, k, slots, job);
}

template <class T>
polyq_status quantize(const T* x, int32_t rows, int32_t k, uint8_t* packed, uint8_t* xt, hipStream_t st) {
  const int records = records_of(k), tiles = xt ? static_cast<int>(align_up(rows, 64) / kRows) : tiles_of(rows);
  const int64_t groups = record_groups(rows, k, xt != nullptr);  // checked by the caller
  const bool vec = aligned(x, 16) && static_cast<int64_t>(k) * sizeof(T) % 16 == 0;
  const auto kernel = xt ? (vec ? mx_quantize_kernel<T, true, true> : mx_quantize_kernel<T, false, true>)
                         : (vec ? mx_quantize_kernel<T, true, false> : mx_quantize_kernel<T, false, false>);
  kernel<<<dim3(static_cast<uint32_t>(groups)), dim3(64 * kWaves), 0, st>>>(x, packed, xt, rows, k, records, tiles);
  return launched();
}

}  // namespace

polyq_status launch_quantize(const void* x, int type, int32_t rows, int32_t k, void* packed, hipStream_t st, void* transposed) {
  uint8_t *out = static_cast<uint8_t*>(packed), *xt = static_cast<uint8_t*>(transposed);
  if (type == POLYQ_MX_F32) return quantize(static_cast<const float*>(x), rows, k, out, xt, st);
  if (type == POLYQ_MX_F16) return quantize(static_cast<const _Float16*>(x), rows, k, out, xt, st);
  return quantize(static_cast<const __bf16*>(x), rows, k, out, xt, st);
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
  if (!mx::launch_fits(mx::record_groups(rows, k, false), 64 * mx::kWaves)) return POLYQ_ERR_CAPACITY;
  return mx::launch_quantize(x, type, rows, k, packed, static_cast<hipStream_t>(stream));
}

extern "C" polyq_status polyq_mx_dequantize(const void* packed, int32_t rows, int32_t k, void* out, int32_t type,
                                            void* stream) {
  if (packed == nullptr || out == nullptr || !mx::float_type(type)) return POLYQ_ERR_ARG;
  if (!mx::valid_shape(rows, k)) return POLYQ_ERR_SHAPE;
  if (!mx::aligned(packed, 256) || !mx::aligned(out, mx::type_bytes(type))) return POLYQ_ERR_ARG;
  const int records = mx::records_of(k);
  const int64_t groups = mx::record_groups(rows, k, false);
  if (!mx::launch_fits(groups, 64 * mx::kWaves)) return POLYQ_ERR_CAPACITY;
  const bool vec = mx::aligned(out, 16) && static_cast<int64_t>(k) * mx::type_bytes(type) % 16 == 0;
  const uint8_t* in = static_cast<const uint8_t*>(packed);
  const dim3 grid(static_cast<uint32_t>(groups)), block(64 * mx::kWaves);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define POLYQ_MX_DEQUANTIZE(T)                                                                                      \
  if (vec)                                                                                                          \
    mx::mx_dequantize_kernel<T, true><<<grid, block, 0, st>>>(in, static_cast<T*>(out), rows, k, records);     \
  else                                                                                                              \
    mx::mx_dequantize_kernel<T, false><<<grid, block, 0, st>>>(in, static_cast<T*>(out), rows, k, records)
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
  const bool vec = mx::aligned(codes, 16) && (k + 1) / 2 % 16 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto kernel = vec ? mx::mx_repack_kernel<true, true> : mx::mx_repack_kernel<true, false>;
  kernel<<<dim3(mx::striding_groups(jobs, 256)), dim3(256), 0, st>>>(codes, scales, static_cast<uint8_t*>(packed), nullptr,
                                                                    rows, k, jobs);
  return mx::launched();
}

extern "C" polyq_status polyq_mx_unpack(const void* packed, int32_t rows, int32_t k, uint8_t* codes, uint8_t* scales,
                                        void* stream) {
  if (codes == nullptr || scales == nullptr || packed == nullptr) return POLYQ_ERR_ARG;
  if (!mx::valid_shape(rows, k)) return POLYQ_ERR_SHAPE;
  if (!mx::aligned(packed, 256)) return POLYQ_ERR_ARG;
  const int64_t jobs = static_cast<int64_t>(mx::tiles_of(rows)) * mx::kRows * mx::records_of(k) * 16;
  const bool vec = mx::aligned(codes, 16) && (k + 1) / 2 % 16 == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto kernel = vec ? mx::mx_repack_kernel<false, true> : mx::mx_repack_kernel<false, false>;
  kernel<<<dim3(mx::striding_groups(jobs, 256)), dim3(256), 0, st>>>(static_cast<const uint8_t*>(packed), nullptr, codes,
                                                                    scales, rows, k, jobs);
  return mx::launched();
}
