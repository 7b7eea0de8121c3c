// Products of microscaled 4-bit matrices: the linear layer y = x^ W^T and the gated block
// h = act(x^ G^T) * (x^ U^T), x^ the quantized activations; and the gated block's
// g, u once more in its backward pass, where dg and du leave instead of h.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mx.h"

namespace polyq {
namespace mx {
namespace {

enum Mode { kLinear = 0, kGated = 1, kGatedGrad = 2 };

struct Args {
  const uint8_t* w[2];  // packed weights (gate, up in the gated modes)
  const uint8_t* x;     // packed activations
  void* y;              // [m][n] of y_type; kGatedGrad: the planes
  const void* dh;       // kGatedGrad: [m][n] of dh_type
  int32_t m, n, k;
  int32_t y_type, dh_type, act;
  int32_t y_vec, dh_vec;      // rows of y / dh take vector accesses of four elements
  int32_t terms, m_pad, n_pad;  // kGatedGrad: planes bf16 [terms][m_pad][2][n_pad]
  int32_t token_blocks;
};

// Four consecutive outputs (rows n0 .. n0 + 3 of the weights) of one token.
template <int MODE>
__device__ __forceinline__ void finish(const Args& a, int token, int n0, f4 v, f4 u) {
  if (MODE == kGatedGrad) {
    // du = dh act(g), dg = dh u act'(g) as sums of bf16 terms; zero in the padding
    if (token >= a.m_pad || n0 >= a.n_pad) return;
    f4 dg = {0.f, 0.f, 0.f, 0.f}, du = {0.f, 0.f, 0.f, 0.f};
    if (token < a.m && n0 < a.n) {
      const int valid = a.n - n0;
      const f4 d = load4(a.dh, a.dh_type, static_cast<int64_t>(token) * a.n + n0, a.dh_vec, valid);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= valid) break;
        float slope;
        const float act = activation(a.act, v[i], &slope);
        dg[i] = d[i] * u[i] * slope;
        du[i] = d[i] * act;
      }
    }
    __bf16* out = static_cast<__bf16*>(a.y) + static_cast<int64_t>(token) * 2 * a.n_pad + n0;
    const int64_t plane = static_cast<int64_t>(a.m_pad) * 2 * a.n_pad;
    for (int t = 0; t < a.terms; ++t) {
      const bf16x4 g4 = next_terms(&dg), u4 = next_terms(&du);
      *reinterpret_cast<bf16x4*>(out + t * plane) = g4;
      *reinterpret_cast<bf16x4*>(out + t * plane + a.n_pad) = u4;
    }
  } else {
    if (token >= a.m || n0 >= a.n) return;
    if (MODE == kGated) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = activation(a.act, v[i], nullptr) * u[i];
    }
    store4(a.y, a.y_type, static_cast<int64_t>(token) * a.n + n0, v, a.y_vec, a.n - n0);
  }
}

// ---------------------------------------------------------------- few tokens
// A work-group of W waves takes TN row tiles (in the gated modes TN / 2 of each matrix) by
// TM token tiles; its waves split K and their sums meet in LDS.
template <int MODE, int TN, int TM, int W>
__global__ __launch_bounds__(64 * W) void mx_stream_kernel(const Args a) {
  __shared__ f4 sums[W][TN * TM][64];
  constexpr int NM = MODE == kLinear ? 1 : 2, PT = TN / NM;  // matrices, row tiles of each
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int chunks = chunks_of(a.k), row_tiles = tiles_of(a.n), token_tiles = tiles_of(a.m);
  const int64_t tb = tile_bytes(a.k);
  const int tile0 = static_cast<int>(blockIdx.x) * PT, tok0 = static_cast<int>(blockIdx.y) * TM;
  const int c0 = static_cast<int>(static_cast<int64_t>(chunks) * wave / W);
  const int c1 = static_cast<int>(static_cast<int64_t>(chunks) * (wave + 1) / W);
  const uint8_t* wp[TN];
  const uint8_t* xp[TM];
#pragma unroll
  for (int i = 0; i < TN; ++i) wp[i] = a.w[i / PT] + min(tile0 + i % PT, row_tiles - 1) * tb;
#pragma unroll
  for (int j = 0; j < TM; ++j) xp[j] = a.x + min(tok0 + j, token_tiles - 1) * tb;
  f4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

  constexpr int U = TN * TM <= 4 ? 4 : 2;
  auto step = [&](int c, auto count) {
    constexpr int N = decltype(count)::value;
    i4v ca[N][TN], cb[N][TM];
    uint32_t sa[N][TN], sb[N][TM];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int64_t at = chunk_offset(c + u) + lane * 16, sat = scale_offset(c + u) + lane * 4;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        ca[u][i] = *reinterpret_cast<const i4v*>(wp[i] + at);
        sa[u][i] = *reinterpret_cast<const uint32_t*>(wp[i] + sat);
      }
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        cb[u][j] = *reinterpret_cast<const i4v*>(xp[j] + at);
        sb[u][j] = *reinterpret_cast<const uint32_t*>(xp[j] + sat);
      }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int sh = 8 * ((c + u) & 3);
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
          acc[i][j] = mfma_mx<0, 0>(ca[u][i], cb[u][j], acc[i][j], static_cast<int>(sa[u][i] >> sh),
                                    static_cast<int>(sb[u][j] >> sh));
    }
  };
  int c = c0;
  for (; c + U <= c1; c += U) step(c, std::integral_constant<int, U>());
  for (; c < c1; ++c) step(c, std::integral_constant<int, 1>());

#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) sums[wave][i * TM + j][lane] = acc[i][j];
  __syncthreads();
  for (int item = threadIdx.x; item < PT * TM * 64; item += 64 * W) {
    const int l = item & 63, ij = item >> 6, i = ij / TM, j = ij % TM;
    f4 v[NM];
#pragma unroll
    for (int h = 0; h < NM; ++h) {
      v[h] = sums[0][(h * PT + i) * TM + j][l];
#pragma unroll
      for (int w = 1; w < W; ++w) v[h] += sums[w][(h * PT + i) * TM + j][l];
    }
    finish<MODE>(a, (tok0 + j) * kRows + (l & 15), (tile0 + i) * kRows + (l >> 4) * 4, v[0], v[NM - 1]);
  }
}

// ---------------------------------------------------------------- many tokens
// WN x WM waves, each TN row tiles (the gated modes: TN / 2 of each matrix) by TM token
// tiles.  K is walked KC chunks at a time: the fragments of both operands go from
// memory straight into one half of a ring in LDS while the other half is multiplied.
template <int MODE, int WN, int WM, int TN, int TM, int KC>
__global__ __launch_bounds__(64 * WN * WM) void mx_gemm_kernel(const Args a) {
  constexpr int W = WN * WM, RT = WN * TN, CT = WM * TM, SLOTS = RT + CT;
  constexpr int NM = MODE == kLinear ? 1 : 2, PT = TN / NM;
  constexpr int STAGE = SLOTS * KC * kChunkBytes;
  constexpr int LOADS = SLOTS * KC / W;
  static_assert(SLOTS * KC % W == 0 && 4 % KC == 0, "tile");
  extern __shared__ uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WN, wm = wave / WN;
  // Work-groups b, b + 8, ... share an XCD and its L2: each XCD takes a run of consecutive tiles,
  // token blocks fastest, so that a weight panel is read by one XCD.
  const int total = static_cast<int>(gridDim.x), per = total / 8, rest = total % 8;
  const int xcd = static_cast<int>(blockIdx.x) % 8, turn = static_cast<int>(blockIdx.x) / 8;
  const int id = xcd * per + min(xcd, rest) + turn;
  const int rb = id / a.token_blocks, tbk = id % a.token_blocks;
  const int chunks = chunks_of(a.k), records = records_of(a.k);
  const int row_tiles = tiles_of(a.n), token_tiles = tiles_of(a.m);
  const int64_t tb = tile_bytes(a.k);
  // Slot s of a stage: row tile s of the work-group (s = wn TN + i), then its token tiles.
  auto slot_ptr = [&](int s) -> const uint8_t* {
    if (s < RT) {
      const int sw = s / TN, i = s % TN;
      return a.w[i / PT] + min((rb * WN + sw) * PT + i % PT, row_tiles - 1) * tb;
    }
    return a.x + min(tbk * CT + s - RT, token_tiles - 1) * tb;
  };
  const uint8_t* src[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) src[i] = slot_ptr((i * W + wave) / KC);
  auto fetch = [&](int c, int half) {  // chunks c .. c + KC - 1 (the last one again past the end)
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = i * W + wave;
      const int64_t at = chunk_offset(min(c + piece % KC, chunks - 1));
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(src[i] + at + lane * 16),
          (__attribute__((address_space(3))) void*)(lds + half * STAGE + piece * kChunkBytes), 16, 0, 0);
    }
  };
  const uint8_t* sa_ptr[TN];
  const uint8_t* sb_ptr[TM];
#pragma unroll
  for (int i = 0; i < TN; ++i) sa_ptr[i] = slot_ptr(wn * TN + i) + lane * 4;
#pragma unroll
  for (int j = 0; j < TM; ++j) sb_ptr[j] = slot_ptr(RT + wm * TM + j) + lane * 4;
  int sa[TN], sb[TM], na[TN], nb[TM];
  auto scales = [&](int rec) {
    const int64_t at = static_cast<int64_t>(min(rec, records - 1)) * kRecBytes;
#pragma unroll
    for (int i = 0; i < TN; ++i) na[i] = *reinterpret_cast<const int*>(sa_ptr[i] + at);
#pragma unroll
    for (int j = 0; j < TM; ++j) nb[j] = *reinterpret_cast<const int*>(sb_ptr[j] + at);
  };
  f4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

  auto multiply = [&](int half, int kc, auto sel) {
    constexpr int SEL = decltype(sel)::value;
    const uint8_t* base = lds + half * STAGE + kc * kChunkBytes + lane * 16;
    i4v ca[TN], cb[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) cb[j] = *reinterpret_cast<const i4v*>(base + (RT + wm * TM + j) * KC * kChunkBytes);
#pragma unroll
    for (int i = 0; i < TN; ++i) ca[i] = *reinterpret_cast<const i4v*>(base + (wn * TN + i) * KC * kChunkBytes);
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = mfma_mx<SEL, SEL>(ca[i], cb[j], acc[i][j], sa[i], sb[j]);
  };
  scales(0);
  fetch(0, 0);
  constexpr int STEPS = 4 / KC;
  auto stage = [&](int rec, auto step) {
    constexpr int S = decltype(step)::value;
    const int c = rec * 4 + S * KC;
    if (S > 0 && c >= chunks) return;  // the last record may be shorter
    const int half = (rec * STEPS + S) & 1;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (S == 0) {
#pragma unroll
      for (int i = 0; i < TN; ++i) sa[i] = na[i];
#pragma unroll
      for (int j = 0; j < TM; ++j) sb[j] = nb[j];
      scales(rec + 1);
    }
    if (c + KC < chunks) fetch(c + KC, half ^ 1);
    multiply(half, 0, std::integral_constant<int, S * KC>());
    if (KC > 1 && c + 1 < chunks) multiply(half, 1, std::integral_constant<int, (S * KC + 1) & 3>());
  };
  for (int rec = 0; rec < records; ++rec) {
    stage(rec, std::integral_constant<int, 0>());
    if (STEPS > 1) stage(rec, std::integral_constant<int, 1 % STEPS>());
    if (STEPS > 2) stage(rec, std::integral_constant<int, 2 % STEPS>());
    if (STEPS > 2) stage(rec, std::integral_constant<int, 3 % STEPS>());
  }

#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int token = (tbk * CT + wm * TM + j) * kRows + (lane & 15);
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int n0 = ((rb * WN + wn) * PT + i) * kRows + (lane >> 4) * 4;
      finish<MODE>(a, token, n0, acc[i][j], acc[NM == 2 ? PT + i : i][j]);
    }
  }
}

// ---------------------------------------------------------------- launches
polyq_status launched() { return hipGetLastError() == hipSuccess ? POLYQ_OK : POLYQ_ERR_DEVICE; }

template <int MODE, int TN, int TM, int W>
polyq_status run_stream(const Args& a, hipStream_t st) {
  const int pt = TN / (MODE == kLinear ? 1 : 2);
  const dim3 grid(div_up(tiles_of(a.n), pt), div_up(tiles_of(a.m), TM));
  mx_stream_kernel<MODE, TN, TM, W><<<grid, dim3(64 * W), 0, st>>>(a);
  return launched();
}

template <int MODE, int WN, int WM, int TN, int TM, int KC>
polyq_status run_gemm(Args a, hipStream_t st) {
  const int pt = WN * TN / (MODE == kLinear ? 1 : 2);
  a.token_blocks = div_up(MODE == kGatedGrad ? a.m_pad / kRows : tiles_of(a.m), WM * TM);
  const int64_t groups = static_cast<int64_t>(div_up(MODE == kGatedGrad ? a.n_pad / kRows : tiles_of(a.n), pt)) * a.token_blocks;
  if (groups > 0x7FFFFFFFll) return POLYQ_ERR_CAPACITY;
  const size_t lds = 2 * static_cast<size_t>(WN * TN + WM * TM) * KC * kChunkBytes;
  const auto kernel = mx_gemm_kernel<MODE, WN, WM, TN, TM, KC>;
  if (lds > 65536 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(lds)) != hipSuccess)
    return POLYQ_ERR_DEVICE;
  kernel<<<dim3(static_cast<uint32_t>(groups)), dim3(64 * WN * WM), lds, st>>>(a);
  return launched();
}

template <int MODE>
polyq_status run(const Args& a, hipStream_t st) {
  if (MODE != kGatedGrad && a.m <= 16) return run_stream<MODE, MODE == kLinear ? 1 : 2, 1, 8>(a, st);
  const int64_t tiles = static_cast<int64_t>(tiles_of(a.n)) * (MODE == kLinear ? 1 : 2) * tiles_of(a.m);
  if (tiles >= 256 * 256) return run_gemm<MODE, 2, 4, 8, 4, 2>(a, st);
  return run_gemm<MODE, 2, 2, 4, 4, 2>(a, st);
}

}  // namespace

polyq_status launch_gated_grad(const void* gate, const void* up, const void* x, const void* dh, int dh_type, int32_t m,
                               int32_t n, int32_t k, int act, void* planes, int terms, int32_t m_pad, int32_t n_pad,
                               hipStream_t st) {
  Args a{};
  a.w[0] = static_cast<const uint8_t*>(gate), a.w[1] = static_cast<const uint8_t*>(up);
  a.x = static_cast<const uint8_t*>(x);
  a.y = planes, a.dh = dh, a.dh_type = dh_type;
  a.m = m, a.n = n, a.k = k, a.act = act;
  a.terms = terms, a.m_pad = m_pad, a.n_pad = n_pad;
  a.dh_vec = n % 4 == 0 && aligned(dh, 4 * type_bytes(dh_type));
  return run<kGatedGrad>(a, st);
}

namespace {

// The activations' packed form: as given, or quantized into the workspace.
polyq_status packed_input(const void* x, int x_type, int32_t m, int32_t k, void* ws, size_t ws_bytes, const uint8_t** out,
                          hipStream_t st) {
  if (x_type == POLYQ_MX_PACKED) {
    *out = static_cast<const uint8_t*>(x);
    return POLYQ_OK;
  }
  *out = static_cast<const uint8_t*>(ws);
  return launch_quantize(x, x_type, m, k, ws, st);
}

polyq_status product(const void* x, int x_type, int32_t m, const void* w0, const void* w1, int32_t n, int32_t k, int act,
                     void* y, int y_type, void* ws, size_t ws_bytes, hipStream_t st) {
  if (x == nullptr || w0 == nullptr || w1 == nullptr || y == nullptr) return POLYQ_ERR_ARG;
  if (!(float_type(x_type) || x_type == POLYQ_MX_PACKED) || !float_type(y_type)) return POLYQ_ERR_ARG;
  if (m < 1) return POLYQ_ERR_ARG;
  if (!valid_shape(m, k) || !valid_shape(n, k)) return POLYQ_ERR_SHAPE;
  if (!aligned(w0, 256) || !aligned(w1, 256) || !aligned(y, type_bytes(y_type))) return POLYQ_ERR_ARG;
  if (!aligned(x, x_type == POLYQ_MX_PACKED ? 256 : type_bytes(x_type))) return POLYQ_ERR_ARG;
  const size_t need = polyq_mx_workspace_bytes(m, k, x_type);
  if (need > 0 && (ws == nullptr || ws_bytes < need)) return POLYQ_ERR_CAPACITY;
  if (need > 0 && !aligned(ws, 256)) return POLYQ_ERR_ARG;
  Args a{};
  a.w[0] = static_cast<const uint8_t*>(w0), a.w[1] = static_cast<const uint8_t*>(w1);
  a.y = y, a.y_type = y_type, a.act = act;
  a.m = m, a.n = n, a.k = k;
  a.y_vec = n % 4 == 0 && aligned(y, 4 * type_bytes(y_type));
  const polyq_status s = packed_input(x, x_type, m, k, ws, ws_bytes, &a.x, st);
  if (s != POLYQ_OK) return s;
  return act < 0 ? run<kLinear>(a, st) : run<kGated>(a, st);
}

}  // namespace
}  // namespace mx
}  // namespace polyq

using namespace polyq;

extern "C" size_t polyq_mx_workspace_bytes(int32_t m, int32_t k, int32_t x_type) {
  return mx::float_type(x_type) ? polyq_mx_bytes(m, k) : 0;
}

extern "C" polyq_status polyq_mx_linear(const void* x, int32_t x_type, int32_t m, const void* w, int32_t n, int32_t k,
                                        void* y, int32_t y_type, void* workspace, size_t workspace_bytes, void* stream) {
  return mx::product(x, x_type, m, w, w, n, k, -1, y, y_type, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" polyq_status polyq_mx_gated(const void* x, int32_t x_type, int32_t m, const void* gate, const void* up,
                                       int32_t n, int32_t k, int32_t act, void* h, int32_t h_type, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  if (!mx::valid_act(act)) return POLYQ_ERR_ARG;
  return mx::product(x, x_type, m, gate, up, n, k, act, h, h_type, workspace, workspace_bytes,
                     static_cast<hipStream_t>(stream));
}
