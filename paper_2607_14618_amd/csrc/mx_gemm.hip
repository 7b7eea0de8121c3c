// Products of microscaled 4-bit matrices: the linear layer y = x^ W^T and the gated block
// h = act(x^ G^T) * (x^ U^T), x^ the quantized activations; and the gated block's
// g, u once more in its backward pass, where dg and du leave instead of h.
//
// x^ and the weights are multiplied in their 4 bits: a lane's 16 bytes and scale byte of the packed layout are what it
// hands to a scaled matrix instruction, so nothing is unpacked.  Three kernels: up to 16 tokens read every weight once and
// are bound by that (mx_stream_kernel), some tokens by latency (mx_split_kernel), many by the matrix cores
// (mx_gemm_kernel); choose() in mx_plan.h says which.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mx.h"

namespace polyq {
namespace mx {
namespace {

enum Mode { kLinear = 0, kGated = 1, kGatedGrad = 2 };

struct Args {
  const uint8_t* w[2];  // packed weights (gate, up in the gated modes)
  const void* x;        // packed activations, or for few tokens [m][k] of x_type
  int32_t x_type, x_vec;  // rows of x take 16-byte accesses
  void* y;              // [m][n] of y_type; kGatedGrad: the planes
  const void* dh;       // kGatedGrad: [m][n] of dh_type
  int32_t m, n, k;
  int32_t y_type, dh_type, act;
  int32_t y_vec, dh_vec;      // rows of y / dh take vector accesses of four elements
  int32_t y_vec16;            // rows of y take 16-byte accesses
  int32_t terms, m_pad, n_pad;  // kGatedGrad: planes [terms][2][m_pad][n_pad]
  int32_t token_blocks;
};

// The activation as a compile-time number where a thread has many values (a branch for each of them took 5 of 153
// us of a gated block of 2000 tokens, 12 of 189 of its gradients); kAnyAct: whatever Args::act says.
constexpr int kAnyAct = -1;
template <int ACT>
__device__ __forceinline__ float activate(int act, float g, float* slope) {
  if constexpr (ACT == kAnyAct) return activation(act, g, slope);
  else return activation<ACT>(g, slope);
}

// dg = dh u act'(g), du = dh act(g) of four rows of the weights and one token.  Where dh u alone is past the largest
// float, the slope, which may be next to nothing, comes first.
template <int ACT>
__device__ __forceinline__ void gated_grad(int act, f4 d, f4 g, f4 u, f4* dg, f4* du) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float slope;
    const float a = activate<ACT>(act, g[i], &slope);
    const float product = d[i] * u[i];
    (*dg)[i] = __builtin_isfinite(product) ? product * slope : u[i] * slope * d[i];
    (*du)[i] = d[i] * a;
  }
}
template <int ACT>
__device__ __forceinline__ f4 gated(int act, f4 g, f4 u) {
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i] = activate<ACT>(act, g[i], nullptr) * u[i];
  return g;
}

// Four consecutive outputs (rows n0 .. n0 + 3 of the weights) of one token, which may lie behind the last.
template <int MODE, class T>
__device__ __forceinline__ void finish(const Args& a, int token, int n0, f4 v, f4 u) {
  if (MODE == kGatedGrad) {
    // zeros in the padding
    if (token >= a.m_pad || n0 >= a.n_pad) return;
    f4 dg = {0.f, 0.f, 0.f, 0.f}, du = {0.f, 0.f, 0.f, 0.f};
    if (token < a.m && n0 < a.n) {
      const int valid = a.n - n0;
      const f4 d = load4(static_cast<const T*>(a.dh) + static_cast<int64_t>(token) * a.n + n0, a.dh_vec, valid);
      gated_grad<kAnyAct>(a.act, d, v, u, &dg, &du);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= valid) dg[i] = du[i] = 0.f;
    }
    const int64_t plane = static_cast<int64_t>(a.m_pad) * a.n_pad * 2;
    uint8_t* out = static_cast<uint8_t*>(a.y) + plane_at(token, n0, a.n_pad);
    for (int t = 0; t < a.terms; ++t) {
      *reinterpret_cast<bf16x4*>(out + 2 * t * plane) = next_terms(&dg, t, a.terms);
      *reinterpret_cast<bf16x4*>(out + (2 * t + 1) * plane) = next_terms(&du, t, a.terms);
    }
  } else {
    if (token >= a.m || n0 >= a.n) return;
    if (MODE == kGated) v = gated<kAnyAct>(a.act, v, u);
    store4(static_cast<T*>(a.y) + static_cast<int64_t>(token) * a.n + n0, v, a.y_vec, a.n - n0);
  }
}

// Two groups of four (n0 and n0 + 8; lanes l + 32 four further on), all there, rows on vectors.
template <int MODE, class T, int ACT>
__device__ __forceinline__ void finish_pair(const Args& a, int token, int n0, int upper, f4 v, f4 u, f4 v8, f4 u8) {
  const int64_t at = static_cast<int64_t>(token) * a.n + n0;
  if (MODE == kGatedGrad) {
    const T* dh = static_cast<const T*>(a.dh) + at;
    f4 dg, du, dg8, du8;
    gated_grad<ACT>(a.act, load4(dh, true, 4), v, u, &dg, &du);
    gated_grad<ACT>(a.act, load4(dh + 8, true, 4), v8, u8, &dg8, &du8);
    const int64_t plane = static_cast<int64_t>(a.m_pad) * a.n_pad * 2;
    uint8_t* out = static_cast<uint8_t*>(a.y) + plane_at(token, n0 - 4 * upper, a.n_pad) + upper * 16;
    for (int t = 0; t < a.terms; ++t) {
      const bf16x4 g0 = next_terms(&dg, t, a.terms), g1 = next_terms(&dg8, t, a.terms);
      const bf16x4 u0 = next_terms(&du, t, a.terms), u1 = next_terms(&du8, t, a.terms);
      *reinterpret_cast<u4v*>(out + 2 * t * plane) = pack_halves(g0, g1);
      *reinterpret_cast<u4v*>(out + (2 * t + 1) * plane) = pack_halves(u0, u1);
    }
  } else {
    if (MODE == kGated) v = gated<ACT>(a.act, v, u), v8 = gated<ACT>(a.act, v8, u8);
    store_pair(static_cast<T*>(a.y) + at, v, v8, upper);
  }
}

// f(type of y or dh).
template <int MODE, class F>
__device__ __forceinline__ void with_type(const Args& a, F f) {
  const int type = MODE == kGatedGrad ? a.dh_type : a.y_type;
  if (type == POLYQ_MX_BF16) f(BF16());
  else if (type == POLYQ_MX_F16) f(F16());
  else f(F32());
}

// ---------------------------------------------------------------- few tokens
// A work-group of W waves takes TN row tiles (in the gated modes TN / 2 of each matrix) by one
// token tile; its waves split K and their sums meet in LDS.  T: the activations' type, which
// every wave then quantizes for its own part of K in its own LDS (one launch instead of
// two); or `Packed`.
// What bounds it: memory.  Gate and up of 13824 x 5120, one token: 75 MB in 13 to 15 us (5.0 to 5.7 TB/s), of 25600 x 5120, 16
// tokens: 139 MB in 28 us (5.0 TB/s); 5120 x 5120, one token: 5.6 us, of which a launch is 2.  Eight waves share K so that a
// few hundred work-groups have all weights in flight: with 4 waves 14.1 us in place of 15.3 and 29.3 in place of 28.4 (there
// is one launch shape for both, and it is the one for several tokens), with 16 20.2 and 31.9; two row tiles of each matrix a work-group 16.2 and 33.8.
struct Packed {};
template <int MODE, class T, bool VEC, int TN, int W>
__global__ __launch_bounds__(64 * W) void mx_stream_kernel(const Args a) {
  constexpr bool RAW = !std::is_same<T, Packed>::value;
  constexpr int NM = MODE == kLinear ? 1 : 2, PT = TN / NM;  // matrices, row tiles of each
  union Shared {
    f4 sums[W][TN][64];
    Record x[RAW ? W : 1];
  };
  __shared__ Shared lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int chunks = chunks_of(a.k), row_tiles = tiles_of(a.n);
  const int64_t tb = tile_bytes(a.k);
  const int tile0 = static_cast<int>(blockIdx.x) * PT;
  const int c0 = static_cast<int>(static_cast<int64_t>(chunks) * wave / W);
  const int c1 = static_cast<int>(static_cast<int64_t>(chunks) * (wave + 1) / W);
  const uint8_t* wp[TN];
#pragma unroll
  for (int i = 0; i < TN; ++i) wp[i] = a.w[i / PT] + min(tile0 + i % PT, row_tiles - 1) * tb;
  f4 acc[TN];
#pragma unroll
  for (int i = 0; i < TN; ++i) acc[i] = f4{0.f, 0.f, 0.f, 0.f};
  Record& rec = lds.x[RAW ? wave : 0];
  if (RAW) {  // tokens behind the last: code 0, scale 1
    for (int i = lane; i < static_cast<int>(sizeof(rec.codes) / 16); i += 64) reinterpret_cast<u4v*>(rec.codes)[i] = u4v{0, 0, 0, 0};
    reinterpret_cast<uint32_t*>(rec.scales)[lane] = 0x7f7f7f7fu;
  }

  auto step = [&](int c, auto count) {
    constexpr int N = decltype(count)::value;
    i4v ca[N][TN], cb[N];
    uint32_t sa[N][TN], sb[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int64_t at = chunk_offset(c + u) + lane * 16, sat = scale_offset(c + u) + lane * 4;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        ca[u][i] = *reinterpret_cast<const i4v*>(wp[i] + at);
        sa[u][i] = *reinterpret_cast<const uint32_t*>(wp[i] + sat);
      }
      if constexpr (!RAW) {
        cb[u] = *reinterpret_cast<const i4v*>(static_cast<const uint8_t*>(a.x) + at);
        sb[u] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.x) + sat);
      }
    }
    if constexpr (RAW) {  // channels 128 c .. of all tokens, as a record of which N chunks are read
      const int k0 = c * kChunk + lane * 8;
      const T* x = static_cast<const T*>(a.x);
      auto put = [&](int t, const float* v) {
        uint32_t byte;
        const uint32_t code = quantize8(v, &byte);
        *rec.at(t, lane) = code;
        if ((lane & 3) == 0) *rec.scale(t, lane) = static_cast<uint8_t>(byte);
      };
      for (int t = 0; t < a.m; t += 2) {  // two tokens' loads at a time
        float v[2][8];
        load8<T, VEC>(x + static_cast<int64_t>(t) * a.k, k0, a.k, v[0]);
        load8<T, VEC>(x + static_cast<int64_t>(min(t + 1, a.m - 1)) * a.k, k0, a.k, v[1]);
        put(t, v[0]);
        if (t + 1 < a.m) put(t + 1, v[1]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const uint32_t word = reinterpret_cast<const uint32_t*>(rec.scales)[lane];
#pragma unroll
      for (int u = 0; u < N; ++u) {
        cb[u] = __builtin_bit_cast(i4v, *rec.fragment(u, lane));
        sb[u] = word >> (8 * u) << (8 * ((c + u) & 3));
      }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int sh = 8 * ((c + u) & 3);
#pragma unroll
      for (int i = 0; i < TN; ++i)
        acc[i] = mfma_mx<0, 0>(ca[u][i], cb[u], acc[i], static_cast<int>(sa[u][i] >> sh), static_cast<int>(sb[u] >> sh));
    }
  };
  constexpr int U = 4;
  int c = c0;
  for (; c + U <= c1; c += U) step(c, std::integral_constant<int, U>());
  if (c1 - c == 3) step(c, std::integral_constant<int, 3>());
  else if (c1 - c == 2) step(c, std::integral_constant<int, 2>());
  else if (c1 - c == 1) step(c, std::integral_constant<int, 1>());

  if (RAW) __syncthreads();  // the sums take the records' place
#pragma unroll
  for (int i = 0; i < TN; ++i) lds.sums[wave][i][lane] = acc[i];
  __syncthreads();
  for (int item = threadIdx.x; item < PT * 64; item += 64 * W) {
    const int l = item & 63, i = item >> 6;
    f4 v[NM];
#pragma unroll
    for (int h = 0; h < NM; ++h) {
      v[h] = lds.sums[0][h * PT + i][l];
#pragma unroll
      for (int w = 1; w < W; ++w) v[h] += lds.sums[w][h * PT + i][l];
    }
    const int token = l & 15, n0 = (tile0 + i) * kRows + (l >> 4) * 4;
    with_type<MODE>(a, [&](auto t) { finish<MODE, typename decltype(t)::type>(a, token, n0, v[0], v[NM - 1]); });
  }
}

// ---------------------------------------------------------------- some tokens
// A work-group of W waves takes 32 rows (of each matrix) by TM x 32 tokens, its waves split K, and
// their sums meet in LDS: many work-groups where the outputs are few.  Both operands
// come straight from memory, the tokens from L2.  77 tokens, 1357 x 2976: 4.7 us, where the tiled kernel below walks all of
// K in one work-group and takes 9.7.
template <int MODE, int TM, int W>
__global__ __launch_bounds__(64 * W, 2) void mx_split_kernel(const Args a) {
  constexpr int NM = MODE == kLinear ? 1 : 2;
  extern __shared__ f4 sums[];  // [W][NM][TM][4][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int second = (lane >> 4) & 1, at16 = (lane >> 5) * 256 + (lane & 15) * 16, at4 = at16 >> 2;
  const int rb = static_cast<int>(blockIdx.x) / a.token_blocks, tbk = static_cast<int>(blockIdx.x) % a.token_blocks;
  const int chunks = chunks_of(a.k), row_tiles = tiles_of(a.n), token_tiles = tiles_of(a.m);
  const int64_t tb = tile_bytes(a.k);
  const int c0 = static_cast<int>(static_cast<int64_t>(chunks) * wave / W);
  const int c1 = static_cast<int>(static_cast<int64_t>(chunks) * (wave + 1) / W);
  const uint8_t *wp[NM], *xp[TM];
#pragma unroll
  for (int i = 0; i < NM; ++i) wp[i] = a.w[i] + min(rb * 2 + second, row_tiles - 1) * tb;
#pragma unroll
  for (int j = 0; j < TM; ++j)
    xp[j] = static_cast<const uint8_t*>(a.x) + min((tbk * TM + j) * 2 + second, token_tiles - 1) * tb;
  f16v acc[NM][TM];
#pragma unroll
  for (int i = 0; i < NM; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  auto step = [&](int c, auto count) {
    constexpr int N = decltype(count)::value;
    i4v ca[N][NM][2], cb[N][TM][2];
    uint32_t sa[N][NM][2], sb[N][TM][2];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int64_t at = chunk_offset(c + u) + at16, sat = scale_offset(c + u) + at4;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < NM; ++i) {
          ca[u][i][h] = *reinterpret_cast<const i4v*>(wp[i] + at + h * 512);
          sa[u][i][h] = *reinterpret_cast<const uint32_t*>(wp[i] + sat + h * 128);
        }
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          cb[u][j][h] = *reinterpret_cast<const i4v*>(xp[j] + at + h * 512);
          sb[u][j][h] = *reinterpret_cast<const uint32_t*>(xp[j] + sat + h * 128);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int sh = 8 * ((c + u) & 3);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
          for (int i = 0; i < NM; ++i)
            acc[i][j] = mfma_mx32<0, 0>(ca[u][i][h], cb[u][j][h], acc[i][j], static_cast<int>(sa[u][i][h] >> sh),
                                        static_cast<int>(sb[u][j][h] >> sh));
    }
  };
  int c = c0;
  for (; c + 2 <= c1; c += 2) step(c, std::integral_constant<int, 2>());
  if (c < c1) step(c, std::integral_constant<int, 1>());
#pragma unroll
  for (int i = 0; i < NM; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        sums[(((wave * NM + i) * TM + j) * 4 + r) * 64 + lane] =
            f4{acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]};
  __syncthreads();
  with_type<MODE>(a, [&](auto t) {
    for (int item = threadIdx.x; item < TM * 256; item += 64 * W) {
      f4 v[NM];
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        v[i] = sums[i * TM * 256 + item];
#pragma unroll
        for (int w = 1; w < W; ++w) v[i] += sums[(w * NM + i) * TM * 256 + item];
      }
      const int l = item & 63, r = (item >> 6) & 3, j = item >> 8;
      finish<MODE, typename decltype(t)::type>(a, (tbk * TM + j) * 32 + (l & 31), rb * 32 + r * 8 + (l >> 5) * 4, v[0], v[NM - 1]);
    }
  });
}

// ---------------------------------------------------------------- many tokens
// WN x WM waves, each TN x 32 rows (the gated modes: TN / 2 x 32 of each matrix) by TM x 32
// tokens.  K is walked a record (4 chunks) at a time.  The tokens' fragments go from
// memory straight into one half of a ring in LDS while the other half is multiplied; the
// weights' fragments are what their wave alone multiplies and go into its registers, AHEAD
// chunks ahead.  Through LDS both operands of such a tile would ask for 94 of its 128 bytes a
// clock; so it is 64 there and 48 of 64 from the caches.  Fragments are read half a chunk ahead
// of their products, in the order written (the scheduler would sink them to their uses).
// What bounds it: the matrix cores and what their power leaves.  On random values a loop of nothing but these
// instructions reaches 6.5 to 7.0 PFLOP/s (clocks fall to 2.0 GHz), gate/up of 2000 tokens x 13824 x 5120 3.9 (146 us:
// products alone 88, in which 1728 work-groups in rounds of 512 leave a sixth idle, loads of weights 20, of scales 10 and
// tokens 14, stores 10), the down projection 3.4 (82 us).  Measured on the way for the former: 16x16x128 instructions and both operands in LDS 228 us, weights in
// registers 205, 32x32x64 instructions and buffer loads into LDS (after the global form the compiler waits for all loads)
// 176, activations by hardware exp2 and reciprocal 157, 16-byte stores 153, one branch for all activations 146.  One wave per SIMD with twice the tile: 247.
template <int MODE, int WN, int WM, int TN, int TM, int AHEAD>
__global__ __launch_bounds__(64 * WN * WM, 2) void mx_gemm_kernel(const Args a) {
  constexpr int W = WN * WM, CT = WM * TM;
  constexpr int NM = MODE == kLinear ? 1 : 2, PT = TN / NM;
  constexpr int STAGE = CT * 8 * kChunkBytes, LOADS = CT * 8 / W;
  static_assert(CT * 8 % W == 0, "tile");
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
  // Of a pair of row tiles, lanes 16 .. 31 and 48 .. 63 take the second (the first again where there is none).
  const int second = (lane >> 4) & 1, at16 = (lane >> 5) * 256 + (lane & 15) * 16, at4 = at16 >> 2;
  // Buffers that begin at the work-group's first tiles; a lane's offsets of its tiles inside them.
  const int row0 = min(rb * WN * PT * 2, row_tiles - 1), tok0 = min(tbk * CT * 2, token_tiles - 1);
  const __amdgpu_buffer_rsrc_t wbuf0 = make_rsrc(a.w[0] + row0 * tb, (row_tiles - row0) * tb);
  const __amdgpu_buffer_rsrc_t wbuf1 = make_rsrc(a.w[NM - 1] + row0 * tb, (row_tiles - row0) * tb);
  const __amdgpu_buffer_rsrc_t xbuf = make_rsrc(static_cast<const uint8_t*>(a.x) + tok0 * tb, (token_tiles - tok0) * tb);
  const uint32_t tb32 = static_cast<uint32_t>(tb);
  uint32_t wo[PT], xo[TM];
#pragma unroll
  for (int i = 0; i < PT; ++i) wo[i] = (min(((rb * WN + wn) * PT + i) * 2 + second, row_tiles - 1) - row0) * tb32;
#pragma unroll
  for (int j = 0; j < TM; ++j) xo[j] = (min((tbk * CT + wm * TM + j) * 2 + second, token_tiles - 1) - tok0) * tb32;
  auto chunk_at = [&](int c) { return static_cast<uint32_t>(chunk_offset(min(c, chunks - 1))); };  // the last again past the end
  auto fetch = [&](int rec, int half) {  // the tokens' codes of a record
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = i * W + wave;
      const uint32_t tile = (min(tbk * CT * 2 + piece / 4, token_tiles - 1) - tok0) * tb32;
      load_to_lds(xbuf, lds + half * STAGE + piece * kChunkBytes, lane * 16, tile + chunk_at(rec * 4 + piece % 4));
    }
  };
  // Scales of the record at hand and of the next one.
  int sa[TN][2], sb[TM][2], na[TN][2], nb[TM][2];
  auto scales = [&](int rec) {
    const uint32_t at = static_cast<uint32_t>(min(rec, records - 1)) * kRecBytes;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < TN; ++i)
        na[i][h] = static_cast<int>(__builtin_amdgcn_raw_buffer_load_b32(i < PT ? wbuf0 : wbuf1, wo[i % PT] + at4 + h * 128, at, 0));
#pragma unroll
      for (int j = 0; j < TM; ++j)
        nb[j][h] = static_cast<int>(__builtin_amdgcn_raw_buffer_load_b32(xbuf, xo[j] + at4 + h * 128, at, 0));
    }
  };
  auto take_scales = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < TN; ++i) sa[i][h] = na[i][h];
#pragma unroll
      for (int j = 0; j < TM; ++j) sb[j][h] = nb[j][h];
    }
  };
  i4v ca[AHEAD][TN][2], cb[2][TM];
  auto weights = [&](int c, int to) {
    const uint32_t at = chunk_at(c);
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        ca[to][i][h] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(i < PT ? wbuf0 : wbuf1, wo[i % PT] + at16 + h * 512, at, 0));
    asm volatile("" ::: "memory");  // keeps the order of the loads: the waits below count them
  };
  auto tokens = [&](int half, int c, int h) {  // half chunk 2 c + h of a record, to cb[h]
    const uint8_t* base = lds + half * STAGE + (wm * TM * 8 + second * 4 + c) * kChunkBytes + at16 + h * 512;
#pragma unroll
    for (int j = 0; j < TM; ++j) cb[h][j] = *reinterpret_cast<const i4v*>(base + j * 8 * kChunkBytes);
  };
  f16v acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  auto multiply = [&](auto which, auto half_chunk) {
    constexpr int C = decltype(which)::value, H = decltype(half_chunk)::value;
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int i = 0; i < TN; ++i) acc[i][j] = mfma_mx32<C, C>(ca[C % AHEAD][i][H], cb[H][j], acc[i][j], sa[i][H], sb[j][H]);
  };
  // One chunk: two halves, the second's and then the next chunk's token fragments read ahead of the products.
  auto chunk = [&](int rec, int ring, auto which) {
    constexpr int C = decltype(which)::value;
    tokens(ring, C, 1);
    __builtin_amdgcn_sched_barrier(0);  // as written: the scheduler would move the reads to their uses
    multiply(which, std::integral_constant<int, 0>());
    __builtin_amdgcn_sched_barrier(0);
    if (C < 3) {
      tokens(ring, C + 1, 0);
    } else {
      // The next record's tokens have arrived: their loads are older than the 2 TN latest, and than the last
      // chunk's weights that the products above have waited for.  All waves are past their reads of this record.
      constexpr int SINCE = 2 * TN * (AHEAD - 1);
      __builtin_amdgcn_s_waitcnt(0x0070 | (SINCE & 15) | (SINCE >> 4 << 14));  // vmcnt(SINCE) lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      tokens(ring ^ 1, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    multiply(which, std::integral_constant<int, 1>());
    __builtin_amdgcn_sched_barrier(0);
    weights(rec * 4 + C + AHEAD, C % AHEAD);
    __builtin_amdgcn_sched_barrier(0);
  };
  fetch(0, 0);
  scales(0);
  asm volatile("" ::: "memory");
#pragma unroll
  for (int c = 0; c < AHEAD; ++c) weights(c, c);
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  tokens(0, 0, 0);
  const int whole = chunks / 4;
  for (int rec = 0; rec < whole; ++rec) {
    take_scales();
    if (rec + 1 < records) fetch(rec + 1, (rec + 1) & 1);
    scales(rec + 1);
    asm volatile("" ::: "memory");
    chunk(rec, rec & 1, std::integral_constant<int, 0>());
    chunk(rec, rec & 1, std::integral_constant<int, 1>());
    chunk(rec, rec & 1, std::integral_constant<int, 2>());
    chunk(rec, rec & 1, std::integral_constant<int, 3>());
  }
  if (whole < records) {  // one to three chunks more
    take_scales();
    chunk(whole, whole & 1, std::integral_constant<int, 0>());
    if (chunks - whole * 4 > 1) chunk(whole, whole & 1, std::integral_constant<int, 1>());
    if (chunks - whole * 4 > 2) chunk(whole, whole & 1, std::integral_constant<int, 2>());
  }

  auto out = [&](auto t, auto act, auto whole) {
    typedef typename decltype(t)::type T;
    constexpr int ACT = decltype(act)::value;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int token = (tbk * CT + wm * TM + j) * 32 + (lane & 31);
#pragma unroll
      for (int i = 0; i < PT; ++i)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const int n0 = ((rb * WN + wn) * PT + i) * 32 + r * 8 + (lane >> 5) * 4;
          const f16v &x = acc[i][j], &y = acc[NM == 2 ? PT + i : i][j];
          const f4 v = {x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]};
          const f4 u = {y[4 * r], y[4 * r + 1], y[4 * r + 2], y[4 * r + 3]};
          const f4 v8 = {x[4 * r + 4], x[4 * r + 5], x[4 * r + 6], x[4 * r + 7]};
          const f4 u8 = {y[4 * r + 4], y[4 * r + 5], y[4 * r + 6], y[4 * r + 7]};
          if (decltype(whole)::value) {
            finish_pair<MODE, T, ACT>(a, token, n0, lane >> 5, v, u, v8, u8);
          } else {
            finish<MODE, T>(a, token, n0, v, u);
            finish<MODE, T>(a, token, n0 + 8, v8, u8);
          }
        }
    }
  };
  const bool all = (rb + 1) * (WN * PT * 32) <= a.n && (tbk + 1) * (CT * 32) <= a.m && (MODE == kGatedGrad ? a.dh_vec : a.y_vec16);
  with_type<MODE>(a, [&](auto t) {
    if (!all) out(t, std::integral_constant<int, kAnyAct>(), std::false_type());
    else if constexpr (MODE == kLinear) out(t, std::integral_constant<int, kAnyAct>(), std::true_type());
    else if (a.act == POLYQ_ACT_SILU) out(t, std::integral_constant<int, POLYQ_ACT_SILU>(), std::true_type());
    else if (a.act == POLYQ_ACT_GELU) out(t, std::integral_constant<int, POLYQ_ACT_GELU>(), std::true_type());
    else out(t, std::integral_constant<int, POLYQ_ACT_GELU_TANH>(), std::true_type());
  });
}

// ---------------------------------------------------------------- launches
template <int MODE, class T, bool VEC>
polyq_status run_stream(const Args& a, hipStream_t st) {
  constexpr int TN = MODE == kLinear ? 1 : 2, W = 8;
  mx_stream_kernel<MODE, T, VEC, TN, W><<<dim3(tiles_of(a.n)), dim3(64 * W), 0, st>>>(a);
  return launched();
}
template <int MODE, class T>
polyq_status run_raw(const Args& a, hipStream_t st) {
  return a.x_vec ? run_stream<MODE, T, true>(a, st) : run_stream<MODE, T, false>(a, st);
}

template <int MODE, int TM, int W>
polyq_status run_split(Args a, int64_t groups, hipStream_t st) {
  a.token_blocks = div_up(MODE == kGatedGrad ? a.m_pad : a.m, TM * 32);
  const size_t lds = static_cast<size_t>(W) * (MODE == kLinear ? 1 : 2) * TM * 4096;
  mx_split_kernel<MODE, TM, W><<<dim3(static_cast<uint32_t>(groups)), dim3(64 * W), lds, st>>>(a);
  return launched();
}

template <int MODE, int WN, int WM, int TN, int TM, int AHEAD>
polyq_status run_gemm(Args a, int64_t groups, hipStream_t st) {
  static_assert(WN * TN * 32 == 256, "product_launch");
  a.token_blocks = div_up(MODE == kGatedGrad ? a.m_pad : a.m, WM * TM * 32);
  const size_t lds = 16 * static_cast<size_t>(WM * TM) * kChunkBytes;
  const auto kernel = mx_gemm_kernel<MODE, WN, WM, TN, TM, AHEAD>;
  kernel<<<dim3(static_cast<uint32_t>(groups)), dim3(64 * WN * WM), lds, st>>>(a);
  return launched();
}

template <int MODE>
polyq_status run(const Args& a, hipStream_t st) {
  if constexpr (MODE != kGatedGrad) {
    if (a.x_type == POLYQ_MX_F32) return run_raw<MODE, float>(a, st);
    if (a.x_type == POLYQ_MX_F16) return run_raw<MODE, _Float16>(a, st);
    if (a.x_type == POLYQ_MX_BF16) return run_raw<MODE, __bf16>(a, st);
    if (a.m <= 16) return run_stream<MODE, Packed, true>(a, st);
  }
  constexpr int mats = MODE == kLinear ? 1 : 2;
  const Choice c = choose(a.m, a.n, a.k, mats);
  const int64_t groups = product_launch(c, MODE == kGatedGrad ? a.m_pad : a.m, MODE == kGatedGrad ? a.n_pad : a.n, mats).groups;
  if (c.split) return c.tm == 1 ? run_split<MODE, 1, 8>(a, groups, st) : run_split<MODE, 2, mats == 1 ? 8 : 4>(a, groups, st);
  if (c.tm == 1) return run_gemm<MODE, 4, 1, 2, 1, 4>(a, groups, st);
  if (c.tm == 2) return run_gemm<MODE, 4, 1, 2, 2, 4>(a, groups, st);
  if (c.tm == 3) return run_gemm<MODE, 4, 1, 2, 3, 2>(a, groups, st);
  return run_gemm<MODE, 4, 1, 2, 4, 2>(a, groups, st);
}

}  // namespace

polyq_status launch_gated_grad(const void* gate, const void* up, const void* x, const void* dh, int dh_type, int32_t m,
                               int32_t n, int32_t k, int act, void* planes, int terms, int32_t m_pad, int32_t n_pad,
                               hipStream_t st) {
  Args a{};
  a.w[0] = static_cast<const uint8_t*>(gate), a.w[1] = static_cast<const uint8_t*>(up);
  a.x = x, a.x_type = POLYQ_MX_PACKED;
  a.y = planes, a.dh = dh, a.dh_type = dh_type;
  a.m = m, a.n = n, a.k = k, a.act = act;
  a.terms = terms, a.m_pad = m_pad, a.n_pad = n_pad;
  a.dh_vec = n % 4 == 0 && aligned(dh, 4 * type_bytes(dh_type));
  return run<kGatedGrad>(a, st);
}

namespace {

// Up to this many tokens every work-group quantizes the activations itself; more are quantized once, in a launch before.
// Itself / once, us for 1, 2, 3, 4 and 8 tokens: linear 5120 x 5120 5.9 6.4 7.4 8.1 11.3 / 8.1 8.3 8.4 8.5 8.6, of 5120 x
// 13824 12.5 12.4 14.5 15.6 22.1 / 16.9 15.8 15.9 16.2 16.2; gated 13824 x 5120 18.3 18.6 21.3 22.5 28.9 / 20.6 20.3
// 20.4 20.8 21.0, of 25600 x 5120 30.4 29.5 35.0 36.1 47.0 / 33.8 30.7 31.1 31.5 32.0.
constexpr int raw_tokens(bool gated) { return gated ? 2 : 4; }
size_t product_bytes(int32_t m, int32_t k, int x_type, bool gated) {
  return float_type(x_type) && m > raw_tokens(gated) ? polyq_mx_bytes(m, k) : 0;
}

polyq_status product(const void* x, int x_type, int32_t m, const void* w0, const void* w1, int32_t n, int32_t k, int act,
                     void* y, int y_type, void* ws, size_t ws_bytes, hipStream_t st) {
  if (x == nullptr || w0 == nullptr || w1 == nullptr || y == nullptr) return POLYQ_ERR_ARG;
  if (!(float_type(x_type) || x_type == POLYQ_MX_PACKED) || !float_type(y_type)) return POLYQ_ERR_ARG;
  if (m < 1) return POLYQ_ERR_ARG;
  if (!valid_shape(m, k) || !valid_shape(n, k)) return POLYQ_ERR_SHAPE;
  if (!aligned(w0, 256) || !aligned(w1, 256) || !aligned(y, type_bytes(y_type))) return POLYQ_ERR_ARG;
  if (!aligned(x, x_type == POLYQ_MX_PACKED ? 256 : type_bytes(x_type))) return POLYQ_ERR_ARG;
  const size_t need = product_bytes(m, k, x_type, act >= 0);
  if (need > 0 && (ws == nullptr || ws_bytes < need)) return POLYQ_ERR_CAPACITY;
  if (need > 0 && !aligned(ws, 256)) return POLYQ_ERR_ARG;
  if (need > 0 && !launch_fits(record_groups(m, k, false), 256)) return POLYQ_ERR_CAPACITY;
  if (m > 16 && !product_fits(m, n, k, act < 0 ? 1 : 2, m, n)) return POLYQ_ERR_CAPACITY;
  Args a{};
  a.w[0] = static_cast<const uint8_t*>(w0), a.w[1] = static_cast<const uint8_t*>(w1);
  a.y = y, a.y_type = y_type, a.act = act;
  a.m = m, a.n = n, a.k = k;
  a.y_vec = n % 4 == 0 && aligned(y, 4 * type_bytes(y_type));
  a.y_vec16 = n * type_bytes(y_type) % 16 == 0 && aligned(y, 16);
  a.x = x, a.x_type = x_type;
  a.x_vec = x_type != POLYQ_MX_PACKED && aligned(x, 16) && static_cast<int64_t>(k) * type_bytes(x_type) % 16 == 0;
  if (need > 0) {
    const polyq_status s = launch_quantize(x, x_type, m, k, ws, st);
    if (s != POLYQ_OK) return s;
    a.x = ws, a.x_type = POLYQ_MX_PACKED;
  }
  return act < 0 ? run<kLinear>(a, st) : run<kGated>(a, st);
}

}  // namespace
}  // namespace mx
}  // namespace polyq

using namespace polyq;

extern "C" size_t polyq_mx_linear_workspace_bytes(int32_t m, int32_t k, int32_t x_type) {
  return mx::product_bytes(m, k, x_type, false);
}
extern "C" size_t polyq_mx_gated_workspace_bytes(int32_t m, int32_t k, int32_t x_type) {
  return mx::product_bytes(m, k, x_type, true);
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
