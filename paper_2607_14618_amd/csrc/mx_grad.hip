// Gradients through products of microscaled 4-bit matrices.
//
//   dx[t][c]  = sum_n d[t][n] W[n][c]     (gated: dg, G and du, U in one sum)
//   dW[n][c]  = sum_t d[t][n] x^[t][c]
// The blocks' scales run along c, so they do not factor out of the sums and the 4-bit
// matrix instructions do not apply: W and x^ are converted to bf16 (exact: two
// significant bits and a power of two, below 2^128) and multiplied on the bf16 matrix cores.  d
// comes as planes of bf16 terms whose sum is the value (launch_gated_grad): one term for
// gradients in bf16 (an error of at most 2^-8 per factor, as large as the result's own rounding),
// two for fp16 (2^-17), three for fp32 (next_terms says how exact).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace polyq {
namespace mx {
namespace {

// A gradient product of either kind is D[l][s] = sum_r L[r][l] S[s][r]:
//   dx   l = c, s = t, r = n:  L = W, converted;           S = d
//   dW   l = n, s = c, r = t:  L = d;                      S = x^ transposed, converted once
// L passes through LDS in blocks of 32 r x 16 l (1 KiB, rows of 32 bytes) and is read transposed; in blocks of odd l
// tiles rows 4 .. 7 change places with 0 .. 3 (and 12 .. 15 with 8 .. 11), so that a fragment's two
// tiles are read from different banks, and dx's converted rows 8 .. 15 have their 16-byte halves
// exchanged, so that they are written to other banks than 0 .. 7;
// S is stored in memory as blocks of 32 s x 16 r, which are the operand fragments of a
// wave, and goes from there into registers a stage ahead.
// A stage is 64 r: four steps of products, each wave reading the next step's L ahead of them and converting the next
// stage's W between them; one barrier a stage.
// What bounds it: the matrix cores (2.0 PFLOP/s of nothing but these instructions on random values) at the share that whole
// tiles leave of a round: 2000 tokens, 5120 x 13824: dx 256 us (1106 TFLOP/s; 432 tiles on 256 compute units), dW 265 (1068;
// 1080 tiles); gated 13824 x 5120: dx 485 + 23 for the sum of 3 splits (1167), dW 495 (1144).  A library product of the same
// bf16 shapes reaches 950 to 1250.  Tried: 128 x 128 a wave, one wave per SIMD (312, 318 us for the first two); 128 x 256 and 256
// x 128 by four waves, two work-groups a compute unit (290, 290); work-groups that walk several outputs with the next one's
// loads under way (280, 290); L of dW by loads straight into LDS, for which the compiler waits before every transposing
// read (282, 316).
struct GradArgs {
  const uint8_t* d;     // planes [terms][mats][p_tiles][n_tiles] of blocks of 32 tokens x 16 n
  const uint8_t* xt;    // dW: [c_tiles][m_tiles] blocks of 32 c x 16 tokens
  const uint8_t* w[2];  // dx: the packed weights
  void* out[2];         // dx [m][k]; dW [n][k] each
  float* part;          // splits > 1: [splits][outputs][rows][k]
  int64_t plane;        // bytes of the planes of one term and matrix
  int32_t mats, terms, splits;
  int32_t m, n, k;
  int32_t m_pad, n_pad; // multiples of 64
  int32_t rows;         // of an output: m or n
  int32_t rsteps;       // stages of one term (and matrix)
  int32_t l_blocks, s_blocks;
  int32_t type, vec;    // of the outputs; rows take vector accesses of four elements
  int32_t vec16;        // k is a multiple of 16 and the outputs are on 16 bytes
};

// WL x WS waves, each TL x 32 l by TS x 32 s.  TERMS: planes of d that a stage of dx multiplies the one W by; more
// terms than that are further stages.
template <bool DW, int WL, int WS, int TL, int TS, int TERMS>
__global__ __launch_bounds__(64 * WL * WS, 2) void mx_grad_kernel(const GradArgs g) {
  constexpr int W = WL * WS, L = WL * TL * 32, S = WS * TS * 32;
  constexpr int STAGE = L * kStep * 2;
  constexpr int BLOCKS = STAGE / kBlockBytes / W;                 // dW: blocks a wave carries into LDS per stage
  constexpr int FRAGS = (L / kChunk) * (kStep / kRows) / W;       // dx: packed fragments a wave converts per stage
  static_assert(BLOCKS * W * kBlockBytes == STAGE && FRAGS * W * kChunk * kRows == L * kStep && L % kChunk == 0, "tile");
  extern __shared__ uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wl = wave % WL, ws = wave / WL;
  const int total = static_cast<int>(gridDim.x), per = total / 8, rest = total % 8;
  const int xcd = static_cast<int>(blockIdx.x) % 8, turn = static_cast<int>(blockIdx.x) / 8;
  int id = xcd * per + min(xcd, rest) + turn;
  const int sb = id % g.s_blocks;
  id /= g.s_blocks;
  const int lb = id % g.l_blocks, mat_out = id / g.l_blocks;  // the output matrix (dW)
  const int64_t tb = tile_bytes(g.k);

  // Stages: terms x (DW ? 1 : mats) x rsteps, split evenly.
  const int stages = g.terms / TERMS * g.rsteps * (DW ? 1 : g.mats);
  const int first = static_cast<int>(static_cast<int64_t>(stages) * blockIdx.y / g.splits);
  const int last = static_cast<int>(static_cast<int64_t>(stages) * (blockIdx.y + 1) / g.splits);

  // A stage's place: plane (term and, for dx, matrix) and r step; past the end the last one's.
  struct Place {
    int stage, plane, r;
  };
  auto advance = [&](Place p) {
    const bool more = p.stage + 1 < last, wrap = p.r + 1 == g.rsteps;
    return Place{p.stage + 1, p.plane + (more && wrap ? 1 : 0), !more ? p.r : wrap ? 0 : p.r + 1};
  };
  // S: fragments of the work-group's s tiles; r in tiles of 16.
  const int s_tiles = DW ? div_up(g.k, 32) : g.m_pad / 32;
  const int64_t s_tile = static_cast<int64_t>(DW ? g.m_pad : g.n_pad) / 16 * kBlockBytes;
  const int s0 = min(sb * (S / 32), s_tiles - 1);
  uint32_t so[TS];
#pragma unroll
  for (int i = 0; i < TS; ++i)
    so[i] = static_cast<uint32_t>(min(sb * (S / 32) + ws * TS + i, s_tiles - 1) - s0) * static_cast<uint32_t>(s_tile) +
            (lane & 31) * 32 + (lane >> 5) * 16;
  i4v sf[4][TERMS][TS];
  auto load_s = [&](const Place& p, auto which) {  // the fragments of step J of a stage
    constexpr int J = decltype(which)::value;
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      const uint8_t* base = (DW ? g.xt : g.d + (p.plane + t * g.mats) * g.plane) + s0 * s_tile;
      const __amdgpu_buffer_rsrc_t buf = make_rsrc(base, (s_tiles - s0) * s_tile);
#pragma unroll
      for (int i = 0; i < TS; ++i)
        sf[J][t][i] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(buf, so[i], (p.r * 4 + J) * kBlockBytes, 0));
    }
  };

  // L of dW: whole blocks by way of registers.
  const int n_tiles = g.n_pad / 16, n0 = min(lb * (L / 16), n_tiles - 1);
  i4v blocks[BLOCKS];
  auto fetch_blocks = [&](const Place& p) {
    const uint8_t* base = g.d + (p.plane * g.mats + mat_out) * g.plane + (static_cast<int64_t>(p.r) * 2 * n_tiles + n0) * kBlockBytes;
    const __amdgpu_buffer_rsrc_t buf = make_rsrc(base, (static_cast<int64_t>(2) * n_tiles - n0) * kBlockBytes);
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      const int block = i * W + wave, rt = block / (L / 16), lt = min(lb * (L / 16) + block % (L / 16), n_tiles - 1) - n0;
      blocks[i] = __builtin_bit_cast(i4v, __builtin_amdgcn_raw_buffer_load_b128(buf, lane * 16, (rt * n_tiles + lt) * kBlockBytes, 0));
    }
  };
  auto store_blocks = [&](int half) {
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
      *reinterpret_cast<i4v*>(lds + half * STAGE + (i * W + wave) * kBlockBytes + ((lane * 16) ^ ((wave & 1) * 128))) = blocks[i];
  };
  // L of dx: packed fragments (16 r x 128 l) into registers, and from there as bf16 into LDS.
  const int chunks = chunks_of(g.k), b_tiles = tiles_of(g.n);
  i4v codes[FRAGS];
  uint32_t words[FRAGS];  // the scales of the fragment's record
  const uint8_t *w0 = g.w[0], *w1 = g.w[1];
  int tile0 = 0;  // the first row tile of the stage in `codes`
  auto fetch_codes = [&](const Place& p) {
    const uint8_t* w = g.mats > 1 && (p.plane & 1) ? w1 : w0;
    tile0 = p.r * (kStep / kRows);
#pragma unroll
    for (int i = 0; i < FRAGS; ++i) {
      const int f = i * W + wave, tile = min(tile0 + f % (kStep / kRows), b_tiles - 1);
      const int c = min(lb * (L / kChunk) + f / (kStep / kRows), chunks - 1);
      const uint8_t* src = w + tile * tb;
      codes[i] = *reinterpret_cast<const i4v*>(src + chunk_offset(c) + lane * 16);
      words[i] = *reinterpret_cast<const uint32_t*>(src + scale_offset(c) + lane * 4);
    }
  };
  auto convert = [&](int half, auto which) {  // half H of each fragment's 32 channels per lane
    constexpr int H = decltype(which)::value;
#pragma unroll
    for (int i = 0; i < FRAGS; ++i) {
      const int f = i * W + wave, rt = f % (kStep / kRows);
      const bool there = tile0 + rt < b_tiles;  // rows behind the last tile are zeros
      const int c = min(lb * (L / kChunk) + f / (kStep / kRows), chunks - 1);
      const float s = scale_value(there ? (words[i] >> (8 * (c & 3))) & 255u : 127u);
      uint32_t v[8];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t code = there ? static_cast<uint32_t>(codes[i][H * 2 + w]) : 0u;
        v[w * 4 + 0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0));
        v[w * 4 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1));
        v[w * 4 + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2));
        v[w * 4 + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3));
      }
      const int lt = f / (kStep / kRows) * 8 + (lane >> 4) * 2 + H;
      uint8_t* dst = lds + half * STAGE + ((rt >> 1) * (L / 16) + lt) * kBlockBytes + ((rt & 1) * 16 + ((lane & 15) ^ (H * 4))) * 32;
      const int first = ((lane >> 3) & 1) * 16;
      *reinterpret_cast<u4v*>(dst + first) = u4v{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<u4v*>(dst + (first ^ 16)) = u4v{v[4], v[5], v[6], v[7]};
    }
  };
  // Fragment of 32 l x 16 r: a transposing read hands lane j of 16 lanes column j of the four rows whose 32
  // bytes those lanes address; lane groups 1 and 3 have l 16 .. 31, groups 2 and 3 r 8 .. 15.
  const int odd = (lane >> 4) & 1;
  const int l_lane = odd * kBlockBytes + ((lane >> 5) * 8 + ((lane & 15) >> 2)) * 32 + (((lane & 3) * 8) ^ (DW ? 0 : (lane >> 5) * 16));
  const int l_first = l_lane + odd * 128, l_second = l_lane + (odd ^ 1) * 128;
  bf16x8 lf[2][TL];
  auto read_l = [&](int half, int step, int to) {
    const uint8_t* base = lds + half * STAGE + ((step >> 1) * (L / 16) + wl * TL * 2) * kBlockBytes + (step & 1) * 512;
#pragma unroll
    for (int i = 0; i < TL; ++i) lf[to][i] = read_transposed(base + l_first + i * 2 * kBlockBytes, base + l_second + i * 2 * kBlockBytes);
  };

  f16v acc[TL][TS];
#pragma unroll
  for (int i = 0; i < TL; ++i)
#pragma unroll
    for (int j = 0; j < TS; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  auto multiply = [&](auto which) {  // rows of D: the output's columns c
    constexpr int J = decltype(which)::value;
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int j = 0; j < TS; ++j) {
        const bf16x8 sv = __builtin_bit_cast(bf16x8, sf[J][t][j]);
#pragma unroll
        for (int i = 0; i < TL; ++i)
          acc[i][j] = DW ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(sv, lf[J & 1][i], acc[i][j], 0, 0, 0)
                         : __builtin_amdgcn_mfma_f32_32x32x16_bf16(lf[J & 1][i], sv, acc[i][j], 0, 0, 0);
      }
  };
  typedef std::integral_constant<int, 0> I0;
  typedef std::integral_constant<int, 1> I1;
  typedef std::integral_constant<int, 2> I2;
  typedef std::integral_constant<int, 3> I3;
  auto fence = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // A product occupies the matrix unit for 32 clocks; the vector work of the next stage goes in between.
  auto mix = [&]() {
#pragma unroll
    for (int i = 0; i < TL * TS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(DW ? 0x200 : 0x002, DW ? 1 : 6 * FRAGS, 0);
    }
  };
  Place next = {first, first / g.rsteps, first % g.rsteps};
  auto fetch_l = [&](const Place& p) { DW ? fetch_blocks(p) : fetch_codes(p); };
  if (first < last) {
    fetch_l(next);
    load_s(next, I0());
    load_s(next, I1());
    load_s(next, I2());
    load_s(next, I3());
    if (DW) {
      store_blocks(0);
    } else {
      convert(0, I0());
      convert(0, I1());
    }
    next = advance(next);
    fetch_l(next);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    fence();
    read_l(0, 0, 0);
  }
  for (int stage = first; stage < last; ++stage) {  // `next`: the stage after this one
    const int half = (stage - first) & 1;
    // The other half is free: every wave read the last of it before the barrier below.
    read_l(half, 1, 1);
    fence();
    multiply(I0());
    fence();
    load_s(next, I0());
    read_l(half, 2, 0);
    fence();
    multiply(I1());
    if (!DW) {
      convert(half ^ 1, I0());
      mix();
    }
    fence();
    load_s(next, I1());
    read_l(half, 3, 1);
    fence();
    multiply(I2());
    if (DW) store_blocks(half ^ 1);
    else convert(half ^ 1, I1());
    mix();
    fence();
    load_s(next, I2());
    const Place after = advance(next);
    fetch_l(after);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the next stage's L is in LDS, this one's is read
    __builtin_amdgcn_s_barrier();
    fence();
    read_l(half ^ 1, 0, 0);
    fence();
    multiply(I3());
    fence();
    load_s(next, I3());
    next = after;
  }
  const bool vec = g.splits > 1 ? g.k % 4 == 0 : g.vec, vec16 = g.splits > 1 ? g.k % 16 == 0 : g.vec16;
  auto out = [&](auto t) {
    typedef typename decltype(t)::type T;
    T* base = static_cast<T*>(g.splits > 1 ? static_cast<void*>(g.part + (static_cast<int64_t>(blockIdx.y) * (DW ? g.mats : 1) + mat_out) *
                                                                              g.rows * g.k)
                                           : (mat_out ? g.out[1] : g.out[0]));
    if (vec16) {  // pairs of tiles side by side, by way of LDS
      uint8_t* room = lds + wave * 8192;
#pragma unroll
      for (int o = 0; o < (DW ? TL : TS); ++o)
#pragma unroll
        for (int c = 0; c < (DW ? TS : TL); c += 2) {
          const int row = (DW ? (lb * WL + wl) * TL + o : (sb * WS + ws) * TS + o) * 32;
          const int col = (DW ? (sb * WS + ws) * TS + c : (lb * WL + wl) * TL + c) * 32;
          store_rows(room, base + static_cast<int64_t>(row) * g.k + col, g.k, DW ? acc[o][c] : acc[c][o],
                     DW ? acc[o][c + 1] : acc[c + 1][o], lane, g.rows - row, g.k - col);
        }
      return;
    }
#pragma unroll
    for (int i = 0; i < TL; ++i)
#pragma unroll
      for (int j = 0; j < TS; ++j) {
        const int lt = (lb * WL + wl) * TL + i, st = (sb * WS + ws) * TS + j;
        const int row = (DW ? lt : st) * 32 + (lane & 31), col = (DW ? st : lt) * 32 + (lane >> 5) * 4;
        if (row >= g.rows) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (col + r * 8 < g.k)
            store4(base + static_cast<int64_t>(row) * g.k + col + r * 8,
                   f4{acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]}, vec, g.k - col - r * 8);
      }
  };
  __syncthreads();  // every wave has read the last of its L
  if (g.splits > 1 || g.type == POLYQ_MX_F32) out(F32());
  else if (g.type == POLYQ_MX_F16) out(F16());
  else out(BF16());
}

// x^ [m][k], packed, as bf16 blocks of 32 channels x 16 tokens, [c_tiles][m_pad / 16], zero behind m and k: a wave takes
// a chunk of a tile.  (Activations that come in their own type leave the quantization in both forms.)
__global__ __launch_bounds__(256) void mx_transpose_kernel(const uint8_t* __restrict__ packed, uint8_t* __restrict__ out, int m,
                                                           int k, int m_tiles, int c_tiles, int64_t jobs) {
  __shared__ uint8_t lds[4][4 * kBlockBytes];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (job >= jobs) return;  // waves are independent: no barrier follows
  const int chunks = chunks_of(k), tile = static_cast<int>(job / chunks), chunk = static_cast<int>(job % chunks);
  i4v codes = {0, 0, 0, 0};
  uint32_t byte = 127;
  if (tile * kRows < m) {
    const uint8_t* src = packed + tile * tile_bytes(k);
    codes = *reinterpret_cast<const i4v*>(src + chunk_offset(chunk) + lane * 16);
    byte = src[scale_offset(chunk) + lane * 4 + (chunk & 3)];
  }
  transpose_chunk(lds[wave], codes, byte, lane, out, chunk, tile, m_tiles, c_tiles);
}

// Adds the splits' sums in order.
__global__ __launch_bounds__(256) void mx_grad_sum_kernel(const GradArgs g) {
  const int64_t n = static_cast<int64_t>(g.rows) * g.k;
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  const int valid = static_cast<int>(min(static_cast<int64_t>(4), n - at));
  const int outs = gridDim.y, out = blockIdx.y;
  const bool vec = n % 4 == 0;
  f4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < g.splits; ++s) v += load4(g.part + (static_cast<int64_t>(s) * outs + out) * n + at, vec, valid);
  store4(out ? g.out[1] : g.out[0], g.type, at, v, g.vec, valid);
}

// d [m][n] into the planes, zero in the padding: four elements a thread at a time.
__global__ __launch_bounds__(256) void mx_planes_kernel(const void* __restrict__ d, int type, int m, int n, int vec,
                                                        uint8_t* __restrict__ planes, int terms, int m_pad, int n_pad) {
  const int64_t quads = static_cast<int64_t>(m_pad) * n_pad / 4;
  for (int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; id < quads; id += static_cast<int64_t>(gridDim.x) * 256) {
    const int row = static_cast<int>(id / (n_pad / 4)), col = static_cast<int>(id % (n_pad / 4)) * 4;
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if (row < m && col < n) v = load4(d, type, static_cast<int64_t>(row) * n + col, vec, n - col);
    for (int t = 0; t < terms; ++t)
      *reinterpret_cast<bf16x4*>(planes + t * (static_cast<int64_t>(m_pad) * n_pad * 2) + plane_at(row, col, n_pad)) =
          next_terms(&v, t, terms);
  }
}

inline int64_t pad64(int64_t v) { return align_up(v, 64); }

template <bool DW, int WL, int WS, int TL, int TS, int TERMS>
polyq_status run_tile(const GradArgs& g, int outs, hipStream_t st) {
  const size_t lds = 2 * static_cast<size_t>(WL * TL * 32) * kStep * 2;
  const auto kernel = mx_grad_kernel<DW, WL, WS, TL, TS, TERMS>;
  const int64_t groups = static_cast<int64_t>(g.l_blocks) * g.s_blocks * outs;
  kernel<<<dim3(static_cast<uint32_t>(groups), g.splits), dim3(64 * WL * WS), lds, st>>>(g);
  return launched();
}

template <bool DW>
polyq_status run_grad(GradArgs g, const Shape& h, void* part, hipStream_t st) {
  const int outs = DW ? g.mats : 1;
  g.splits = h.splits, g.l_blocks = h.l_blocks, g.s_blocks = h.s_blocks;
  g.part = static_cast<float*>(part);
  polyq_status r;
  if (h.s == 256) r = run_tile<DW, 2, 4, 4, 2, 1>(g, outs, st);
  else if constexpr (DW) r = run_tile<true, 4, 1, 2, 2, 1>(g, outs, st);
  else if (h.l == 256)
    r = g.terms == 1   ? run_tile<false, 4, 1, 2, 2, 1>(g, 1, st)
        : g.terms == 2 ? run_tile<false, 4, 1, 2, 2, 2>(g, 1, st)
                       : run_tile<false, 4, 1, 2, 2, 3>(g, 1, st);
  else
    r = g.terms == 1   ? run_tile<false, 2, 2, 2, 1, 1>(g, 1, st)
        : g.terms == 2 ? run_tile<false, 2, 2, 2, 1, 2>(g, 1, st)
                       : run_tile<false, 2, 2, 2, 1, 3>(g, 1, st);
  if (r != POLYQ_OK || h.splits == 1) return r;
  const int64_t blocks = (static_cast<int64_t>(g.rows) * g.k + 1023) / 1024;
  mx_grad_sum_kernel<<<dim3(static_cast<uint32_t>(blocks), outs), dim3(256), 0, st>>>(g);
  return launched();
}

// Workspace of a backward call, in order: packed x, planes, transposed x, partial sums (of dx, then of the weights' gradients:
// one room, the launches are ordered).
struct GradPlan {
  int terms;
  int32_t m_pad, n_pad;
  Shape dx, dw;
  size_t x_bytes, plane_bytes, xt_bytes, part_bytes, total;
  bool fits;  // every launch
};
GradPlan grad_plan(int32_t m, int32_t n, int32_t k, int mats, int x_type, int grad_type, bool dx, bool dw) {
  // the packed x is what g and u are computed from; the linear layer's gradients need the transposed one alone
  GradPlan p{};
  p.terms = grad_type == POLYQ_MX_BF16 ? 1 : grad_type == POLYQ_MX_F16 ? 2 : 3;
  p.m_pad = static_cast<int32_t>(pad64(m)), p.n_pad = static_cast<int32_t>(pad64(n));
  p.x_bytes = x_type == POLYQ_MX_PACKED || mats == 1 ? 0 : align_up(static_cast<int64_t>(polyq_mx_bytes(m, k)), 256);
  p.plane_bytes = static_cast<size_t>(p.terms) * p.m_pad * mats * p.n_pad * 2;
  p.xt_bytes = dw ? static_cast<size_t>(div_up(k, 32)) * (p.m_pad / 16) * kBlockBytes : 0;
  p.fits = (x_type == POLYQ_MX_PACKED || launch_fits(record_groups(m, k, dw), 256)) &&
           (mats == 1 || product_fits(m, n, k, mats, p.m_pad, p.n_pad));
  if (dx) {
    p.dx = grad_shape(false, k, m, 1, mats * (p.n_pad / kStep), p.terms);
    p.fits = p.fits && shape_fits(p.dx, 1, m, k);
    if (p.dx.splits > 1) p.part_bytes = std::max(p.part_bytes, static_cast<size_t>(p.dx.splits) * m * k * 4);
  }
  if (dw) {
    p.dw = grad_shape(true, n, k, mats, p.m_pad / kStep, p.terms);
    p.fits = p.fits && shape_fits(p.dw, mats, n, k) && (x_type != POLYQ_MX_PACKED || launch_fits(transpose_groups(p.m_pad, k), 256));
    if (p.dw.splits > 1) p.part_bytes = std::max(p.part_bytes, static_cast<size_t>(p.dw.splits) * mats * n * k * 4);
  }
  p.total = p.x_bytes + p.plane_bytes + p.xt_bytes + p.part_bytes;
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
  if (q.m > kMaxRows || q.n > kMaxRows) return POLYQ_ERR_CAPACITY;
  if (!aligned(q.w[0], 256) || !aligned(q.w[1], 256) || !aligned(q.d, type_bytes(q.d_type))) return POLYQ_ERR_ARG;
  if (need_x && !aligned(q.x, q.x_type == POLYQ_MX_PACKED ? 256 : type_bytes(q.x_type))) return POLYQ_ERR_ARG;
  const int size = type_bytes(q.grad_type);
  if (!aligned(q.dx, size) || !aligned(q.dw[0], size) || !aligned(q.dw[1], size)) return POLYQ_ERR_ARG;
  const GradPlan p = grad_plan(q.m, q.n, q.k, q.mats, need_x ? q.x_type : POLYQ_MX_PACKED, q.grad_type, q.dx != nullptr, dw);
  if (!p.fits || ws == nullptr || ws_bytes < p.total) return POLYQ_ERR_CAPACITY;
  if (!aligned(ws, 256)) return POLYQ_ERR_ARG;
  uint8_t* at = static_cast<uint8_t*>(ws);
  const void* x = q.x;
  void* planes = at + p.x_bytes;
  uint8_t* xt = at + p.x_bytes + p.plane_bytes;
  if (need_x && q.x_type != POLYQ_MX_PACKED) {
    const polyq_status s = launch_quantize(q.x, q.x_type, q.m, q.k, p.x_bytes > 0 ? at : nullptr, st, dw ? xt : nullptr);
    if (s != POLYQ_OK) return s;
    x = at;
  }
  void* part = xt + p.xt_bytes;
  if (q.act >= 0) {
    const polyq_status s = launch_gated_grad(q.w[0], q.w[1], x, q.d, q.d_type, q.m, q.n, q.k, q.act, planes, p.terms,
                                             p.m_pad, p.n_pad, st);
    if (s != POLYQ_OK) return s;
  } else {
    const uint32_t blocks = striding_groups(static_cast<int64_t>(p.m_pad) * p.n_pad / 4, 256);
    const int vec = q.n % 4 == 0 && aligned(q.d, 4 * type_bytes(q.d_type));
    mx_planes_kernel<<<dim3(blocks), dim3(256), 0, st>>>(
        q.d, q.d_type, q.m, q.n, vec, static_cast<uint8_t*>(planes), p.terms, p.m_pad, p.n_pad);
    const polyq_status s = launched();
    if (s != POLYQ_OK) return s;
  }
  GradArgs g{};
  g.d = static_cast<const uint8_t*>(planes), g.xt = xt;
  g.w[0] = static_cast<const uint8_t*>(q.w[0]), g.w[1] = static_cast<const uint8_t*>(q.w[1]);
  g.plane = static_cast<int64_t>(p.m_pad) * p.n_pad * 2;
  g.mats = q.mats, g.terms = p.terms, g.type = q.grad_type;
  g.m = q.m, g.n = q.n, g.k = q.k, g.m_pad = p.m_pad, g.n_pad = p.n_pad;
  if (q.dx != nullptr) {
    g.out[0] = q.dx, g.rows = q.m, g.rsteps = p.n_pad / kStep;
    g.vec = q.k % 4 == 0 && aligned(q.dx, 4 * size), g.vec16 = q.k % 16 == 0 && aligned(q.dx, 16);
    const polyq_status s = run_grad<false>(g, p.dx, part, st);
    if (s != POLYQ_OK) return s;
  }
  if (dw) {
    if (q.x_type == POLYQ_MX_PACKED) {
      const int m_tiles = p.m_pad / 16, c_tiles = div_up(q.k, 32);
      const int64_t jobs = static_cast<int64_t>(m_tiles) * chunks_of(q.k);
      mx_transpose_kernel<<<dim3(static_cast<uint32_t>(transpose_groups(p.m_pad, q.k))), dim3(256), 0, st>>>(static_cast<const uint8_t*>(x), xt, q.m, q.k,
                                                                                    m_tiles, c_tiles, jobs);
      const polyq_status s = launched();
      if (s != POLYQ_OK) return s;
    }
    g.out[0] = q.dw[0], g.out[1] = q.dw[1], g.rows = q.n, g.rsteps = p.m_pad / kStep;
    g.vec = q.k % 4 == 0 && aligned(q.dw[0], 4 * size) && aligned(q.dw[1], 4 * size);
    g.vec16 = q.k % 16 == 0 && aligned(q.dw[0], 16) && aligned(q.dw[1], 16);
    return run_grad<true>(g, p.dw, part, st);
  }
  return POLYQ_OK;
}

size_t backward_bytes(int32_t m, int32_t n, int32_t k, int mats, int x_type, int grad_type, int dx, int dw) {
  if (!valid_shape(m, k) || !valid_shape(n, k) || !float_type(grad_type)) return 0;
  if (!float_type(x_type) && x_type != POLYQ_MX_PACKED) return 0;
  if (m > kMaxRows || n > kMaxRows) return 0;
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
