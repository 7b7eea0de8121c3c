// Gradients through products of microscaled 4-bit matrices.
//
// Both are products C[p][c] = sum_r A[p][r] B[r][c] whose right operand is a packed
// matrix with the reduction along its ROWS:
//   dx[t][c]  = sum_n d[t][n] W[n][c]     (A = d,    B = W;  gated: dg, G and du, U in one sum)
//   dW[n][c]  = sum_t d[t][n] x^[t][c]    (A = d^T,  B = x^)
// The blocks' scales run along c, so they do not factor out of the sum over r and the 4-bit
// matrix instructions do not apply: B is converted to bf16 (exact: two significant bits
// and a power of two) on its way into LDS and multiplied on the bf16 matrix cores.  A
// comes as planes of bf16 terms whose sum is the value (launch_gated_grad): one term for
// gradients in bf16 (an error of 2^-9 per factor, as large as the result's own rounding),
// two for fp16, three for fp32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace polyq {
namespace mx {
namespace {

constexpr int kStep = 64;  // rows of the reduction per stage

struct GradArgs {
  const __bf16* a;      // planes [terms][a_rows][mats][a_pitch]
  const uint8_t* b[2];  // packed matrices
  void* c[2];           // outputs [p][k]
  float* part;          // splits > 1: [splits][outputs][p][k]
  int64_t plane;        // elements of a plane
  int64_t row;          // elements from one plane row to the next: mats * pitch
  int32_t pitch;        // a_pitch
  int32_t mats;         // matrices: summed over (dx) or one output each (dW)
  int32_t p, k;         // of an output
  int32_t p_pad;        // p of the planes (a multiple of 64)
  int32_t b_rows;       // rows of each packed matrix
  int32_t rsteps;       // stages of one (term, matrix)
  int32_t terms, splits;
  int32_t type, vec;    // of the outputs; rows take vector accesses of four elements
  int32_t p_blocks, c_blocks;
};

// 16-byte unit swizzles: see the kernel.
__device__ __forceinline__ int row_swizzle(int r) { return (r & 3) | ((r >> 1) & 4); }

// WP x WC waves, each TP tiles of 16 p by TC tiles of 16 c.  TRANS: the planes hold A
// transposed (their rows are the reduction).
template <bool TRANS, int WP, int WC, int TP, int TC>
__global__ __launch_bounds__(64 * WP * WC) void mx_grad_kernel(const GradArgs g) {
  constexpr int W = WP * WC, P = WP * TP * 16, C = WC * TC * 16;
  constexpr int A_BYTES = P * kStep * 2, B_BYTES = C * kStep * 2, STAGE = A_BYTES + B_BYTES;
  constexpr int A_LOADS = A_BYTES / 1024 / W;           // 1 KiB pieces of a wave
  constexpr int B_FRAGS = (C / kChunk) * (kStep / kRows);  // packed fragments of a stage
  constexpr int B_LOADS = B_FRAGS / W;
  static_assert(A_LOADS * W * 1024 == A_BYTES && B_LOADS * W == B_FRAGS && C % kChunk == 0, "tile");
  extern __shared__ uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % WP, wc = wave / WP;
  const int total = static_cast<int>(gridDim.x), per = total / 8, rest = total % 8;
  const int xcd = static_cast<int>(blockIdx.x) % 8, turn = static_cast<int>(blockIdx.x) / 8;
  int id = xcd * per + min(xcd, rest) + turn;
  const int pb = id % g.p_blocks;
  id /= g.p_blocks;
  const int cb = id % g.c_blocks;
  const int out = id / g.c_blocks;  // the output matrix (dW)
  const int p0 = pb * P, chunk0 = cb * (C / kChunk);
  const int chunks = chunks_of(g.k), b_tiles = tiles_of(g.b_rows);
  const int64_t tb = tile_bytes(g.k);

  // Stages: terms x (TRANS ? 1 : mats) x rsteps, split evenly.
  const int inner = TRANS ? g.rsteps : g.rsteps * g.mats;
  const int stages = inner * g.terms;
  const int s0 = static_cast<int>(static_cast<int64_t>(stages) * blockIdx.y / g.splits);
  const int s1 = static_cast<int>(static_cast<int64_t>(stages) * (blockIdx.y + 1) / g.splits);

  auto fetch_a = [&](int s, int half) {
    const int term = s / inner, r = s % inner;
    const int mat = TRANS ? out : r / g.rsteps, r0 = (TRANS ? r : r % g.rsteps) * kStep;
    const __bf16* base = g.a + term * g.plane + static_cast<int64_t>(mat) * g.pitch;
#pragma unroll
    for (int i = 0; i < A_LOADS; ++i) {
      const int piece = (i * W + wave) * 64 + lane;  // 16-byte piece of the stage, in LDS order
      const __bf16* src;
      if (TRANS) {  // rows of P elements: pieces swizzled in pairs (32 bytes, a tile of 16 p)
        const int r16 = piece / (P / 8), slot = piece % (P / 8);
        const int pc = ((slot >> 1) ^ row_swizzle(r16)) * 2 + (slot & 1);
        src = base + static_cast<int64_t>(r0 + r16) * g.row + min(p0 + pc * 8, g.p_pad - 8);
      } else {  // rows of 64 elements = 8 pieces
        const int row = piece >> 3, pc = (piece & 7) ^ (row & 7);
        src = base + static_cast<int64_t>(min(p0 + row, g.p_pad - 1)) * g.row + r0 + pc * 8;
      }
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                       (__attribute__((address_space(3))) void*)(lds + half * STAGE + (i * W + wave) * 1024),
                                       16, 0, 0);
    }
  };
  i4v codes[B_LOADS];
  uint32_t bytes[B_LOADS];
  auto fetch_b = [&](int s) {
    const int r = s % inner;
    const int mat = TRANS ? 0 : r / g.rsteps, t0 = (TRANS ? r : r % g.rsteps) * (kStep / kRows);
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) {
      const int f = i * W + wave, tile = t0 + f % (kStep / kRows), c = min(chunk0 + f / (kStep / kRows), chunks - 1);
      const uint8_t* src = g.b[mat] + min(tile, b_tiles - 1) * tb;
      codes[i] = *reinterpret_cast<const i4v*>(src + chunk_offset(c) + lane * 16);
      bytes[i] = src[scale_offset(c) + lane * 4 + (c & 3)];
      if (tile >= b_tiles) codes[i] = i4v{0, 0, 0, 0}, bytes[i] = 127;  // rows behind the last: zeros
    }
  };
  auto store_b = [&](int half) {
    uint8_t* base = lds + half * STAGE + A_BYTES;
#pragma unroll
    for (int i = 0; i < B_LOADS; ++i) {
      const int f = i * W + wave, r = (f % (kStep / kRows)) * kRows + (lane & 15);
      const int unit = (f / (kStep / kRows)) * 8 + (lane >> 4) * 2;  // 32-byte units of 16 columns
      const float s = scale_value(bytes[i]);
      const bool nan = bytes[i] == kNanScale;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t v[8];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t code = static_cast<uint32_t>(codes[i][h * 2 + w]);
          v[w * 4 + 0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0));
          v[w * 4 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1));
          v[w * 4 + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2));
          v[w * 4 + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3));
        }
        if (nan) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = 0x7fc07fc0u;
        }
        uint8_t* dst = base + r * (C * 2) + ((unit + h) ^ row_swizzle(r)) * 32;
        *reinterpret_cast<u4v*>(dst) = u4v{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<u4v*>(dst + 16) = u4v{v[4], v[5], v[6], v[7]};
      }
    }
  };
  // Fragment of a 64-row tile in LDS with the reduction along its rows: 8 rows (32 s + 8 (lane /
  // 16) ..) of column lane % 16 of unit `unit`.  A transposing read hands lane j of 16
  // lanes column j of the four rows whose 32 bytes those lanes address.
  auto frag_rows = [&](const uint8_t* base, int pitch, int s, int unit) -> bf16x8 {
    const int i = lane & 15, r = s * 32 + (lane >> 4) * 8 + (i >> 2);
    typedef short s4 __attribute__((ext_vector_type(4)));
    union {
      s4 h[2];
      bf16x8 v;
    } u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = r + 4 * h;
      const uint8_t* p = base + row * pitch + (unit ^ row_swizzle(row)) * 32 + (i & 3) * 8;
      u.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(p));
    }
    return u.v;
  };
  f4 acc[TP][TC];
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](int half) {
    const uint8_t* la = lds + half * STAGE;
    const uint8_t* lb = la + A_BYTES;
#pragma unroll
    for (int s = 0; s < kStep / 32; ++s) {
      bf16x8 fa[TP], fb[TC];
#pragma unroll
      for (int j = 0; j < TC; ++j) fb[j] = frag_rows(lb, C * 2, s, wc * TC + j);
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        if (TRANS) {
          fa[i] = frag_rows(la, P * 2, s, wp * TP + i);
        } else {
          const int row = (wp * TP + i) * 16 + (lane & 15), pc = (s * 4 + (lane >> 4)) ^ (row & 7);
          fa[i] = *reinterpret_cast<const bf16x8*>(la + row * (kStep * 2) + pc * 16);
        }
      }
#pragma unroll
      for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int j = 0; j < TC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  };
  if (s0 < s1) {
    fetch_a(s0, 0);
    fetch_b(s0);
    store_b(0);
    if (s0 + 1 < s1) fetch_b(s0 + 1);
  }
  for (int s = s0; s < s1; ++s) {
    const int half = (s - s0) & 1;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + 1 < s1) {
      store_b(half ^ 1);
      fetch_a(s + 1, half ^ 1);
      if (s + 2 < s1) fetch_b(s + 2);
    }
    multiply(half);
  }
#pragma unroll
  for (int i = 0; i < TP; ++i) {
    const int row = p0 + (wp * TP + i) * 16 + (lane & 15);
    if (row >= g.p) continue;
#pragma unroll
    for (int j = 0; j < TC; ++j) {
      const int col = cb * C + (wc * TC + j) * 16 + (lane >> 4) * 4;
      if (col >= g.k) continue;
      const int64_t at = static_cast<int64_t>(row) * g.k + col;
      if (g.splits > 1) {
        const int outs = TRANS ? g.mats : 1;
        float* part = g.part + (static_cast<int64_t>(blockIdx.y) * outs + out) * g.p * g.k;
        store4(part + at, acc[i][j], g.k % 4 == 0, g.k - col);
      } else {
        store4(g.c[out], g.type, at, acc[i][j], g.vec, g.k - col);
      }
    }
  }
}

// Adds the splits' sums in order.
__global__ __launch_bounds__(256) void mx_grad_sum_kernel(const GradArgs g) {
  const int64_t n = static_cast<int64_t>(g.p) * g.k;
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  const int valid = static_cast<int>(min(static_cast<int64_t>(4), n - at));
  const int outs = gridDim.y, out = blockIdx.y;
  const bool vec = n % 4 == 0;
  f4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < g.splits; ++s) v += load4(g.part + (static_cast<int64_t>(s) * outs + out) * n + at, vec, valid);
  store4(g.c[out], g.type, at, v, g.vec, valid);
}

// d [m][n] into planes of bf16 terms [terms][m_pad][n_pad], zero in the padding: four elements a thread.
__global__ __launch_bounds__(256) void mx_planes_kernel(const void* __restrict__ d, int type, int m, int n, int vec,
                                                        __bf16* __restrict__ planes, int terms, int m_pad, int n_pad) {
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= static_cast<int64_t>(m_pad) * n_pad) return;
  const int row = static_cast<int>(at / n_pad), col = static_cast<int>(at % n_pad);
  f4 v = {0.f, 0.f, 0.f, 0.f};
  if (row < m && col < n) v = load4(d, type, static_cast<int64_t>(row) * n + col, vec, n - col);
  for (int t = 0; t < terms; ++t) {
    const bf16x4 b = next_terms(&v);
    *reinterpret_cast<bf16x4*>(planes + static_cast<int64_t>(t) * m_pad * n_pad + at) = b;
  }
}

polyq_status launched() { return hipGetLastError() == hipSuccess ? POLYQ_OK : POLYQ_ERR_DEVICE; }

inline int64_t pad64(int64_t v) { return align_up(v, 64); }

// One gradient product's tile and splits.
struct Shape {
  bool big;
  int p_blocks, c_blocks, splits;
};
Shape grad_shape(int p, int k, int outs, int stages) {
  Shape s;
  const int64_t big = static_cast<int64_t>(div_up(p, 256)) * div_up(k, 256) * outs;
  s.big = big >= 200;
  const int tile = s.big ? 256 : 128;
  s.p_blocks = div_up(p, tile), s.c_blocks = div_up(k, tile);
  const int64_t groups = static_cast<int64_t>(s.p_blocks) * s.c_blocks * outs;
  // Split the reduction where the output's tiles leave most of the GPU idle: at least 8 stages each.
  s.splits = 1;
  while (groups * s.splits * 2 <= 512 && stages / (s.splits * 2) >= 8 && s.splits < 32) s.splits *= 2;
  return s;
}

template <bool TRANS, int WP, int WC, int TP, int TC>
polyq_status run_tile(const GradArgs& g, int outs, hipStream_t st) {
  const size_t lds = 2 * static_cast<size_t>(WP * TP * 16 + WC * TC * 16) * kStep * 2;
  const auto kernel = mx_grad_kernel<TRANS, WP, WC, TP, TC>;
  if (lds > 65536 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(lds)) != hipSuccess)
    return POLYQ_ERR_DEVICE;
  const int64_t groups = static_cast<int64_t>(g.p_blocks) * g.c_blocks * outs;
  if (groups > 0x7FFFFFFFll) return POLYQ_ERR_CAPACITY;
  kernel<<<dim3(static_cast<uint32_t>(groups), g.splits), dim3(64 * WP * WC), lds, st>>>(g);
  return launched();
}

template <bool TRANS>
polyq_status run_grad(GradArgs g, int outs, void* part, hipStream_t st) {
  const int stages = g.terms * g.rsteps * (TRANS ? 1 : g.mats);
  const Shape s = grad_shape(g.p, g.k, outs, stages);
  g.splits = s.splits, g.p_blocks = s.p_blocks, g.c_blocks = s.c_blocks;
  g.part = static_cast<float*>(part);
  const polyq_status r = s.big ? run_tile<TRANS, 2, 4, 8, 4>(g, outs, st) : run_tile<TRANS, 2, 2, 4, 4>(g, outs, st);
  if (r != POLYQ_OK || s.splits == 1) return r;
  const int64_t blocks = (static_cast<int64_t>(g.p) * g.k + 1023) / 1024;
  mx_grad_sum_kernel<<<dim3(static_cast<uint32_t>(blocks), outs), dim3(256), 0, st>>>(g);
  return launched();
}

// Workspace of a backward call, in order: packed x, planes, partial sums (of dx, then of the weights' gradients:
// one room, the launches are ordered).
struct GradPlan {
  int terms;
  int32_t m_pad, n_pad;
  size_t x_bytes, plane_bytes, part_bytes, total;
};
GradPlan grad_plan(int32_t m, int32_t n, int32_t k, int mats, int x_type, int grad_type, bool dx, bool dw) {
  GradPlan p;
  p.terms = grad_type == POLYQ_MX_BF16 ? 1 : grad_type == POLYQ_MX_F16 ? 2 : 3;
  p.m_pad = static_cast<int32_t>(pad64(m)), p.n_pad = static_cast<int32_t>(pad64(n));
  p.x_bytes = x_type == POLYQ_MX_PACKED ? 0 : align_up(static_cast<int64_t>(polyq_mx_bytes(m, k)), 256);
  p.plane_bytes = static_cast<size_t>(p.terms) * p.m_pad * mats * p.n_pad * 2;
  p.part_bytes = 0;
  if (dx) {
    const Shape s = grad_shape(m, k, 1, p.terms * mats * (p.n_pad / kStep));
    if (s.splits > 1) p.part_bytes = std::max(p.part_bytes, static_cast<size_t>(s.splits) * m * k * 4);
  }
  if (dw) {
    const Shape s = grad_shape(n, k, mats, p.terms * (p.m_pad / kStep));
    if (s.splits > 1) p.part_bytes = std::max(p.part_bytes, static_cast<size_t>(s.splits) * mats * n * k * 4);
  }
  p.total = p.x_bytes + p.plane_bytes + p.part_bytes;
  return p;
}

struct Request {
  const void *d, *x;
  int32_t d_type, x_type, m;
  const void* w[2];
  int32_t mats, n, k, act;  // act < 0: the linear layer
  void *dx, *dw[2];
  int32_t grad_type;
};

polyq_status backward(const Request& q, void* ws, size_t ws_bytes, hipStream_t st) {
  if (q.d == nullptr || q.w[0] == nullptr || q.w[1] == nullptr) return POLYQ_ERR_ARG;
  const bool dw = q.dw[0] != nullptr;
  if (dw != (q.dw[q.mats - 1] != nullptr) || (q.dx == nullptr && !dw)) return POLYQ_ERR_ARG;
  const bool need_x = dw || q.act >= 0;
  if (!float_type(q.d_type) || !float_type(q.grad_type)) return POLYQ_ERR_ARG;
  if (need_x && (q.x == nullptr || !(float_type(q.x_type) || q.x_type == POLYQ_MX_PACKED))) return POLYQ_ERR_ARG;
  if (q.m < 1) return POLYQ_ERR_ARG;
  if (!valid_shape(q.m, q.k) || !valid_shape(q.n, q.k)) return POLYQ_ERR_SHAPE;
  if (!aligned(q.w[0], 256) || !aligned(q.w[1], 256) || !aligned(q.d, type_bytes(q.d_type))) return POLYQ_ERR_ARG;
  if (need_x && !aligned(q.x, q.x_type == POLYQ_MX_PACKED ? 256 : type_bytes(q.x_type))) return POLYQ_ERR_ARG;
  const int size = type_bytes(q.grad_type);
  if (!aligned(q.dx, size) || !aligned(q.dw[0], size) || !aligned(q.dw[1], size)) return POLYQ_ERR_ARG;
  GradPlan p = grad_plan(q.m, q.n, q.k, q.mats, need_x ? q.x_type : POLYQ_MX_PACKED, q.grad_type, q.dx != nullptr, dw);
  if (ws == nullptr || ws_bytes < p.total) return POLYQ_ERR_CAPACITY;
  if (!aligned(ws, 256)) return POLYQ_ERR_ARG;
  uint8_t* at = static_cast<uint8_t*>(ws);
  const void* x = q.x;
  if (p.x_bytes > 0) {
    const polyq_status s = launch_quantize(q.x, q.x_type, q.m, q.k, at, st);
    if (s != POLYQ_OK) return s;
    x = at;
  }
  void* planes = at + p.x_bytes;
  void* part = at + p.x_bytes + p.plane_bytes;
  if (q.act >= 0) {
    const polyq_status s = launch_gated_grad(q.w[0], q.w[1], x, q.d, q.d_type, q.m, q.n, q.k, q.act, planes, p.terms,
                                             p.m_pad, p.n_pad, st);
    if (s != POLYQ_OK) return s;
  } else {
    const int64_t blocks = (static_cast<int64_t>(p.m_pad) * p.n_pad / 4 + 255) / 256;
    if (blocks > 0x7FFFFFFFll) return POLYQ_ERR_CAPACITY;
    const int vec = q.n % 4 == 0 && aligned(q.d, 4 * type_bytes(q.d_type));
    mx_planes_kernel<<<dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, st>>>(
        q.d, q.d_type, q.m, q.n, vec, static_cast<__bf16*>(planes), p.terms, p.m_pad, p.n_pad);
    const polyq_status s = launched();
    if (s != POLYQ_OK) return s;
  }
  GradArgs g{};
  g.a = static_cast<const __bf16*>(planes);
  g.mats = q.mats, g.pitch = p.n_pad, g.row = static_cast<int64_t>(q.mats) * p.n_pad, g.plane = g.row * p.m_pad;
  g.k = q.k, g.terms = p.terms, g.type = q.grad_type;
  if (q.dx != nullptr) {
    g.b[0] = static_cast<const uint8_t*>(q.w[0]), g.b[1] = static_cast<const uint8_t*>(q.w[1]);
    g.c[0] = q.dx, g.p = q.m, g.p_pad = p.m_pad, g.b_rows = q.n, g.rsteps = p.n_pad / kStep;
    g.vec = q.k % 4 == 0 && aligned(q.dx, 4 * size);
    const polyq_status s = run_grad<false>(g, 1, part, st);
    if (s != POLYQ_OK) return s;
  }
  if (dw) {
    g.b[0] = g.b[1] = static_cast<const uint8_t*>(x);
    g.c[0] = q.dw[0], g.c[1] = q.dw[1], g.p = q.n, g.p_pad = p.n_pad, g.b_rows = q.m, g.rsteps = p.m_pad / kStep;
    g.vec = q.k % 4 == 0 && aligned(q.dw[0], 4 * size) && aligned(q.dw[1], 4 * size);
    return run_grad<true>(g, q.mats, part, st);
  }
  return POLYQ_OK;
}

size_t backward_bytes(int32_t m, int32_t n, int32_t k, int mats, int x_type, int grad_type, int dx, int dw) {
  if (!valid_shape(m, k) || !valid_shape(n, k) || !float_type(grad_type)) return 0;
  if (!float_type(x_type) && x_type != POLYQ_MX_PACKED) return 0;
  return grad_plan(m, n, k, mats, x_type, grad_type, dx != 0, dw != 0).total;
}

}  // namespace
}  // namespace mx
}  // namespace polyq

using namespace polyq;

extern "C" size_t polyq_mx_linear_backward_workspace_bytes(int32_t m, int32_t n, int32_t k, int32_t x_type,
                                                           int32_t grad_type, int32_t dx, int32_t dw) {
  return mx::backward_bytes(m, n, k, 1, dw ? x_type : POLYQ_MX_PACKED, grad_type, dx, dw);
}

extern "C" polyq_status polyq_mx_linear_backward(const void* dy, int32_t dy_type, const void* x, int32_t x_type, int32_t m,
                                                 const void* w, int32_t n, int32_t k, void* dx, void* dw,
                                                 int32_t grad_type, void* workspace, size_t workspace_bytes, void* stream) {
  const mx::Request q{dy, x, dy_type, x_type, m, {w, w}, 1, n, k, -1, dx, {dw, nullptr}, grad_type};
  return mx::backward(q, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" size_t polyq_mx_gated_backward_workspace_bytes(int32_t m, int32_t n, int32_t k, int32_t x_type,
                                                          int32_t grad_type, int32_t dx, int32_t dw) {
  return mx::backward_bytes(m, n, k, 2, x_type, grad_type, dx, dw);
}

extern "C" polyq_status polyq_mx_gated_backward(const void* dh, int32_t dh_type, const void* x, int32_t x_type, int32_t m,
                                                const void* gate, const void* up, int32_t n, int32_t k, int32_t act,
                                                void* dx, void* dgate, void* dup, int32_t grad_type, void* workspace,
                                                size_t workspace_bytes, void* stream) {
  if (!mx::valid_act(act)) return POLYQ_ERR_ARG;
  const mx::Request q{dh, x, dh_type, x_type, m, {gate, up}, 2, n, k, act, dx, {dgate, dup}, grad_type};
  return mx::backward(q, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}
