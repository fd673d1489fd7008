// k_head.hip -- the loss of a model's last stage: softmax cross entropy of
// x w^T over a large vocabulary, and its gradients, without the logits.
//
//   z = x w^T,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_{i,t_i}
//   d_iv = g_i (exp(z_iv - lse_i) - [v = t_i]),  dx = d w,  dw = d^T x
//
// Tokens without a target are left out before anything is computed: the first
// kernel lists the others, and every later one works on that list, whose
// length stays on the device (tiles past it end at once).
//
// The loss needs one product.  Its epilogue reduces each token's logits, a
// piece of 64 or 128 vocabulary entries at a time, to their maximum and the
// sum of their exponentials; a small kernel joins the pieces.  With gradients
// the epilogue also leaves exp(z - piece's maximum), 16 bits each, so that the
// logits are computed once (6 n v h operations, not 8); another pass turns
// them, now that lse is known, into the softmax minus the target, once by
// tokens and once by vocabulary entries, the operands of the two gradient
// products.  That matrix exists for a chunk of tokens only.
//
// All three products have the matrix units' operands contiguous in the summed
// index, so w and x are transposed on the way (and padded where rows do not
// start at 16 bytes).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "tc_gemm.hpp"
#include "tc_internal.hpp"

namespace tc {

namespace {

// ------------------------------------------------------------------- types
// T: dtype of x and w.  V8: the matrix units' operand.  PLANES: 2 for
// binary32, which goes in as two binary16 planes after a scaling that puts the
// largest magnitude at 2^14 (22 bits of every element down to 2^-28 of it; the
// absolute error of smaller ones is 2^-39 of it).
template <typename T> struct Type;
template <> struct Type<bf16_t> { using V8 = bhalf8; static constexpr int PLANES = 1; };
template <> struct Type<f16_t> { using V8 = half8; static constexpr int PLANES = 1; };
template <> struct Type<float> { using V8 = half8; static constexpr int PLANES = 2; };

// The softmax entries go into the gradient products in bfloat16 as they are,
// in binary16 times 2^14: their range there is 2^-28 to 1 with 11 bits, and
// 2^-38 at the least.
template <typename T> constexpr float P_SCALE = std::is_same_v<T, bf16_t> ? 1.0f : 16384.0f;

// How a softmax numerator (0 .. 1) is held between the two passes over it.
// 16-bit types: in 16 bits, none for a sign.  bfloat16 needs the range of
// binary32 rather than the bits: 7 exponent bits are all that a number up to 1
// uses, 9 mantissa bits follow them.  binary16 needs the bits: 5 exponent bits
// (2^-30, and evenly down to 2^-41) and 11 mantissa bits.
template <typename T> struct Numerator {
  using R = uint16_t;
  static constexpr int SHIFT = std::is_same_v<T, bf16_t> ? 14 : 12;
  static constexpr float SCALE = std::is_same_v<T, bf16_t> ? 1.0f : 0x1p-96f;
  static __device__ __forceinline__ uint16_t down(float p) {
    return (uint16_t)((__float_as_uint(p * SCALE) + (1u << (SHIFT - 1))) >> SHIFT);
  }
  static __device__ __forceinline__ float up(uint16_t u, float f) {
    return __uint_as_float((uint32_t)u << SHIFT) * (f * (1.0f / SCALE));
  }
};
template <> struct Numerator<float> {
  using R = float;
  static __device__ __forceinline__ float down(float p) { return p; }
  static __device__ __forceinline__ float up(float p, float f) { return p * f; }
};

template <typename V8, int J> struct Cfg;
// 256 x 256, one workgroup of 8 wavefronts per compute unit; for fewer tokens
// 256 x 128 and 256 x 64, two of 4 wavefronts
template <typename V8> struct Cfg<V8, 256> : Gemm<V8, 4, 2, 2, 4, 4> { static constexpr uint32_t PER_CU = 1; };
template <typename V8> struct Cfg<V8, 128> : Gemm<V8, 4, 2, 2, 2, 3> { static constexpr uint32_t PER_CU = 2; };
template <typename V8> struct Cfg<V8, 64> : Gemm<V8, 2, 2, 4, 1, 4> { static constexpr uint32_t PER_CU = 2; };
uint32_t tile_tokens(uint64_t rows) { return rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }

// what the first kernels find out about the inputs, on the device
struct Info {
  uint32_t count;        // tokens with a target
  uint32_t top_g, top_x, top_w;   // patterns of the largest |weight|, |x|, |w|
};

// tokens with a target in the chunk that starts at the list's place c0
__device__ __forceinline__ uint32_t chunk_tokens(const HeadArgs& a, uint32_t c0) {
  const uint32_t n = ((const Info*)a.info)->count;
  return min(n > c0 ? n - c0 : 0u, (uint32_t)a.chunk);
}

// exponent that scales a binary32 operand: the largest magnitude becomes 2^14 .. 2^15
__device__ __forceinline__ int plane_exp(uint32_t top) { return top == 0 ? 0 : 14 - ((int)(top >> 23) - 127); }

constexpr float LOG2E = 1.44269504f;

template <typename T>
__device__ __forceinline__ uint16_t narrow(float v) {
  if constexpr (std::is_same_v<T, bf16_t>) return Elem<bf16_t>::down(v);
  else return Elem<f16_t>::down(v);
}

// ------------------------------------------------- tokens that have a target
constexpr int RNT = 1024;

__global__ __launch_bounds__(RNT) void k_head_rows(const HeadArgs a) {
  __shared__ uint32_t part[RNT / WAVE], base;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  Info* const info = (Info*)a.info;
  if (threadIdx.x == 0) base = 0;
  uint32_t top = 0;
  for (uint64_t i0 = 0; i0 < a.n; i0 += RNT) {
    const uint64_t i = i0 + threadIdx.x;
    bool keep = false;
    if (i < a.n) {
      const int64_t t = a.target[i];
      keep = t != a.ignore;
      if (keep && (t < 0 || (uint64_t)t >= a.v)) {
        raise_error(KERR_BAD_INDEX);
        keep = false;
      }
      if (!keep) a.loss[i] = a.lse[i] = 0.0f;
      else if (a.weight) top = max(top, __float_as_uint(a.weight[i]) & 0x7FFFFFFFu);
    }
    const uint64_t ones = __ballot(keep);
    __syncthreads();
    if (lane == 0) part[wave] = (uint32_t)__popcll(ones);
    __syncthreads();
    uint32_t at = base;
    for (uint32_t k = 0; k < wave; ++k) at += part[k];
    if (keep) a.rows[at + (uint32_t)__popcll(ones & ((1ull << lane) - 1))] = (uint32_t)i;
    __syncthreads();
    if (threadIdx.x == RNT - 1) base = at + (uint32_t)__popcll(ones);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  __syncthreads();
  if (lane == 0) part[wave] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (uint32_t k = 0; k < RNT / WAVE; ++k) top = max(top, part[k]);
    info->count = base;
    info->top_g = a.weight ? top : 0x3F800000u;
    info->top_x = info->top_w = 0;
  }
}

// gradients of tokens without a target are zero
template <typename T>
__global__ __launch_bounds__(256) void k_head_zero(const HeadArgs a) {
  using R = typename Elem<T>::raw;
  const int64_t t = a.target[blockIdx.x];
  if (t != a.ignore && t >= 0 && (uint64_t)t < a.v) return;
  R* d = (R*)a.dx + (uint64_t)blockIdx.x * a.h;
  for (uint32_t k = threadIdx.x; k < a.h; k += 256) d[k] = R{};
}

// largest magnitude of x's listed rows, or of w (a maximum: any order gives it)
__global__ __launch_bounds__(256) void k_head_top(const HeadArgs a, bool of_w) {
  __shared__ uint32_t part[4];
  Info* const info = (Info*)a.info;
  const uint64_t rows = of_w ? a.v : info->count;
  uint32_t top = 0;
  for (uint64_t r = blockIdx.x * 4u + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4u) {
    const float* p = of_w ? (const float*)a.w + r * a.ldw : (const float*)a.x + a.rows[r] * a.ldx;
#pragma unroll 8
    for (uint32_t k = threadIdx.x & 63u; k < a.h; k += 64) top = max(top, __float_as_uint(p[k]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) atomicMax(of_w ? &info->top_w : &info->top_x, max(max(part[0], part[1]), max(part[2], part[3])));
}

// ------------------------------------------------------ operands laid out
// 64 x 64 pieces of x (the chunk's listed rows) or w into blocks, by rows and
// transposed, zeros around them; binary32 as two planes.
template <typename T, bool OF_W>
__global__ __launch_bounds__(256) void k_head_pack(const HeadArgs a, uint32_t c0, char* rows_out, char* cols_out) {
  using R = typename Elem<T>::raw;
  constexpr int PL = Type<T>::PLANES;
  __shared__ __attribute__((aligned(16))) uint16_t tile[PL][64][72];
  const Info info = *(const Info*)a.info;
  const uint32_t r0 = blockIdx.y * 64u, k0 = blockIdx.x * 64u;
  uint32_t rows = (uint32_t)a.v;
  if (!OF_W) {
    rows = chunk_tokens(a, c0);
    if (r0 >= rows) return;
  }
  const int e = PL == 2 ? plane_exp(OF_W ? info.top_w : info.top_x) : 0;
  const uint32_t kk = threadIdx.x & 63u;
#pragma unroll 4
  for (uint32_t q = 0; q < 16; ++q) {
    const uint32_t r = r0 + q * 4u + (threadIdx.x >> 6), k = k0 + kk;
    R v{};
    if (r < rows && k < a.h) {
      const uint64_t row = OF_W ? r : a.rows[c0 + r];
      v = ((const R*)(OF_W ? a.w : a.x))[row * (OF_W ? a.ldw : a.ldx) + k];
    }
    if constexpr (PL == 2) {
      const float s = __builtin_ldexpf(v, e);
      const uint16_t hi = Elem<f16_t>::down(s);
      tile[0][r - r0][kk] = hi;
      tile[1][r - r0][kk] = Elem<f16_t>::down(s - Elem<f16_t>::up(hi));
    } else {
      tile[0][r - r0][kk] = v;
    }
  }
  __syncthreads();
  const uint64_t rb = OF_W ? a.v_blocks : a.c_blocks, kb = OF_W ? a.k_dx : (uint32_t)(a.chunk / KSTAGE);
#pragma unroll
  for (int p = 0; p < PL; ++p)
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      // piece `u`: of block u / 64, at its place u % 64
      const uint32_t u = q * 256u + threadIdx.x, blk = u >> 6, row = (u >> 2) & 15u, piece = (u & 3u) ^ turn(row);
      const uint32_t m = (blk >> 1) * 16u + row, n = (blk & 1u) * 32u + piece * 8u;    // m along rows, n along k
      if (rows_out && k0 + (blk & 1u) * 32u < a.k_logits * KSTAGE) {
        char* o = rows_out + p * (OF_W ? a.wr_plane : a.xr_plane);
        *reinterpret_cast<u32x4*>(o + (((k0 >> 5) + (blk & 1u)) * rb + (r0 >> 4) + (blk >> 1)) * 1024u + (u & 63u) * 16u) =
            *reinterpret_cast<const u32x4*>(&tile[p][m][n]);
      }
      if (cols_out && (r0 >> 5) + (blk & 1u) < kb) {
        char* o = cols_out + p * (OF_W ? a.wc_plane : a.xc_plane);
        uint16_t v[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) v[z] = tile[p][n + z][m];
        u32x4 w;
        __builtin_memcpy(&w, v, 16);
        *reinterpret_cast<u32x4*>(o + (((r0 >> 5) + (blk & 1u)) * (uint64_t)a.h_blocks + (k0 >> 4) + (blk >> 1)) * 1024u + (u & 63u) * 16u) = w;
      }
    }
}

// ---------------------------------------------------------------- the logits
// Tile order: 8 token tiles wide, so that the workgroups that run together on
// a die share rows of both operands.
struct Tile { uint32_t i, j; };
__device__ __forceinline__ Tile tile_of(uint32_t t, uint32_t ni, uint32_t nj) {
  const uint32_t group = t / (8u * ni), rem = t - group * 8u * ni, width = min(8u, nj - group * 8u);
  return {rem / width, group * 8u + rem % width};
}

// pt: softmax numerators relative to their piece's maximum, in blocks as dx's
// product takes them (binary32: blocks of 2 KB, pieces where they are)
template <typename T, int J, bool GRAD, bool DIRECT>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, J>::NT), 2) void k_head_logits(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, J>;
  constexpr int PL = Type<T>::PLANES;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const Info info = *(const Info*)a.info;
  const uint32_t left = chunk_tokens(a, c0);
  const uint32_t ni = ((uint32_t)a.v + G::TI - 1) / G::TI, nj = (left + G::TJ - 1) / G::TJ;
  // (only as many tiles as there are tokens for; the grid holds the most there can be)
  const uint32_t t = die_tile(blockIdx.x, gridDim.x);
  if (t >= ni * nj) return;
  const Tile tile = tile_of(t, ni, nj);
  const uint32_t i0 = tile.i * G::TI, j0 = tile.j * G::TJ;
  const Blocks B{a.xr, a.c_blocks, a.xr_plane};
  f32x16 acc[G::WI][G::WJ];
  const uint32_t per = a.k_logits, count = (PL == 2 ? 3 : 1) * per;
  if constexpr (DIRECT) {
    const Rows A{(const char*)a.w, a.ldw * 2, (uint32_t)a.v, nullptr};
    G::template run<1>(A, i0, B, j0, per, 0, count, lds, acc);
  } else {
    const Blocks A{a.wr, a.v_blocks, a.wr_plane};
    G::template run<PL == 2 ? 3 : 1>(A, i0, B, j0, per, 0, count, lds, acc);
  }

  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
  const uint32_t iw = i0 + (wave % G::NWI) * (G::WI * 32), jw = j0 + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u);
  if (iw >= a.v) return;
  const uint32_t piece = iw / (G::WI * 32);
  const float scale = Type<T>::PLANES == 2 ? __builtin_ldexpf(1.0f, -plane_exp(info.top_w) - plane_exp(info.top_x)) : 1.0f;
#pragma unroll
  for (int y = 0; y < G::WJ; ++y) {
    const uint32_t j = jw + y * 32;
    float top = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < G::WI; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (Type<T>::PLANES == 2) acc[x][y][r] *= scale;
        if (iw + x * 32 + h * 16 + r >= a.v) acc[x][y][r] = -__builtin_inff();
        top = fmaxf(top, acc[x][y][r]);
      }
    top = fmaxf(top, __shfl_xor(top, 32));
    // the logit of the token's target, where this piece holds it
    const uint32_t goal = j < left ? (uint32_t)a.target[a.rows[c0 + j]] - iw : ~0u;
    if (__ballot(goal < G::WI * 32u)) {
#pragma unroll
      for (int x = 0; x < G::WI; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (goal == x * 32 + h * 16 + r) a.zt[j] = acc[x][y][r];
    }
    float sum = 0.0f;
#pragma unroll
    for (int x = 0; x < G::WI; ++x) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f((acc[x][y][r] - top) * LOG2E);
        acc[x][y][r] = p;
        sum += p;
      }
      if (GRAD && j < left) {
        const uint32_t kb = (iw >> 5) + x;
        if (kb < a.k_dx) {
          using R = typename Numerator<T>::R;
          R v[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) v[r] = Numerator<T>::down(acc[x][y][r]);
          constexpr uint32_t PIECE = 8 * sizeof(R);
          char* o = a.pt + ((uint64_t)kb * a.c_blocks + (j >> 4)) * (64u * PIECE) + (j & 15u) * 4u * PIECE;
          if constexpr (PL == 2) {
            __builtin_memcpy(o + h * 2 * PIECE, v, 2 * PIECE);
          } else {
            __builtin_memcpy(o + ((2u * h) ^ turn(j)) * PIECE, v, PIECE);
            __builtin_memcpy(o + ((2u * h + 1u) ^ turn(j)) * PIECE, v + 8, PIECE);
          }
        }
      }
    }
    sum += __shfl_xor(sum, 32);
    if (h == 0 && j < left) a.stats[(uint64_t)piece * a.chunk + j] = make_float2(top, sum);
  }
}

// ------------------------------------------------- pieces joined, the losses
constexpr int SNT = 1024;

__global__ __launch_bounds__(SNT) void k_head_loss(const HeadArgs a, uint32_t c0, uint32_t pieces) {
  __shared__ float2 part[SNT / 64][64];
  const uint32_t left = chunk_tokens(a, c0);
  const uint32_t r = threadIdx.x & 63u, q = threadIdx.x >> 6, j = blockIdx.x * 64u + r;
  if (blockIdx.x * 64u >= left) return;
  float m = -__builtin_inff(), s = 0.0f;
  if (j < left) {
#pragma unroll 4
    for (uint32_t p = q; p < pieces; p += SNT / 64) {
      const float2 v = a.stats[(uint64_t)p * a.chunk + j];
      const float top = fmaxf(m, v.x);
      // (a piece whose logits are all -inf adds nothing)
      if (top > -__builtin_inff()) s = s * __expf(m - top) + v.y * __expf(v.x - top);
      m = top;
    }
  }
  part[q][r] = make_float2(m, s);
  __syncthreads();
  if (q == 0 && j < left) {
    float top = m;
    for (int k = 1; k < SNT / 64; ++k) top = fmaxf(top, part[k][r].x);
    float sum = 0.0f;
    for (int k = 0; k < SNT / 64; ++k) sum += part[k][r].y * __expf(part[k][r].x - top);
    const float lse = top + logf(sum);
    const uint32_t i = a.rows[c0 + j];
    a.lse[i] = lse;
    a.loss[i] = lse - a.zt[j];
    a.row_lse[j] = lse;
  }
}

// --------------------------------------------- softmax minus target, twice
// 64 tokens x 128 vocabulary entries.  By tokens (dx's operand): the entry
// without the token's weight, which dx gets at its end.  By vocabulary entries
// (dw's operand): times the weight (in binary16 as a share of the largest).
template <typename T>
__global__ __launch_bounds__(256) void k_head_softmax(const HeadArgs a, uint32_t c0, uint32_t piece_bits) {
  constexpr int PL = Type<T>::PLANES;
  using R = typename Numerator<T>::R;
  constexpr uint32_t PIECE = 8 * sizeof(R);
  __shared__ __attribute__((aligned(16))) uint16_t tile[PL][128][72];
  __shared__ float lse[64], wt[64];
  __shared__ uint32_t goal[64];
  const Info info = *(const Info*)a.info;
  const uint32_t left = chunk_tokens(a, c0);
  const uint32_t j0 = blockIdx.y * 64u, i0 = blockIdx.x * 128u;
  if (j0 >= left) return;
  if (threadIdx.x < 64) {
    const uint32_t j = j0 + threadIdx.x;
    lse[threadIdx.x] = 0.0f;
    wt[threadIdx.x] = 0.0f;
    goal[threadIdx.x] = ~0u;
    if (j < left) {
      const uint32_t i = a.rows[c0 + j];
      lse[threadIdx.x] = a.row_lse[j];
      const float g = a.weight ? a.weight[i] : 1.0f, top = __uint_as_float(info.top_g);
      wt[threadIdx.x] = std::is_same_v<T, bf16_t> ? g : top > 0.0f ? g / top : 0.0f;
      goal[threadIdx.x] = (uint32_t)a.target[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t q = 0; q < 2; ++q) {
    // two pieces of one token: 32 such pairs in each of 16 blocks
    const uint32_t u = q * 256u + threadIdx.x, blk = u >> 5, half = u & 1u;
    const uint32_t r = (blk & 3u) * 16u + ((u >> 1) & 15u), c = (blk >> 2) * 32u + half * 16u, j = j0 + r, i = i0 + c;
    float p[16] = {};
    const bool in = j < left && (i >> 5) < a.k_dx;
    const uint64_t block = (uint64_t)(i >> 5) * a.c_blocks + (j >> 4);
    const uint32_t first = PL == 2 ? 0u : turn(j);
    if (in) {
      const float f = __expf(a.stats[(uint64_t)(i >> piece_bits) * a.chunk + j].x - lse[r]);
      const char* s = a.pt + block * (64u * PIECE) + (j & 15u) * 4u * PIECE;
      R v[16];
      __builtin_memcpy(v, s + ((2u * half) ^ first) * PIECE, PIECE);
      __builtin_memcpy(v + 8, s + ((2u * half + 1u) ^ first) * PIECE, PIECE);
#pragma unroll
      for (int z = 0; z < 16; ++z) p[z] = Numerator<T>::up(v[z], f);
#pragma unroll
      for (int z = 0; z < 16; ++z)
        if (i + z == goal[r]) p[z] -= 1.0f;
    }
    uint16_t v[PL][16];
#pragma unroll
    for (int z = 0; z < 16; ++z) {
      const float s = p[z] * P_SCALE<T>, t = s * wt[r];
      v[0][z] = narrow<T>(s);
      const uint16_t hi = narrow<T>(t);
      tile[0][c + z][r] = hi;
      if constexpr (PL == 2) {
        v[1][z] = narrow<T>(s - Elem<f16_t>::up(v[0][z]));
        tile[1][c + z][r] = narrow<T>(t - Elem<f16_t>::up(hi));
      }
    }
    if (in)
#pragma unroll
      for (int l = 0; l < PL; ++l) {
        char* o = a.pr + l * a.pr_plane + block * 1024u + (j & 15u) * 64u;
        __builtin_memcpy(o + ((2u * half) ^ turn(j)) * 16u, v[l], 16);
        __builtin_memcpy(o + ((2u * half + 1u) ^ turn(j)) * 16u, v[l] + 8, 16);
      }
  }
  __syncthreads();
#pragma unroll
  for (int l = 0; l < PL; ++l)
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) {
      // one piece of 8 tokens: 64 in each of 16 blocks
      const uint32_t u = q * 256u + threadIdx.x, blk = u >> 6, row = (u >> 2) & 15u, piece = (u & 3u) ^ turn(row);
      const uint32_t c = (blk >> 1) * 16u + row, r = (blk & 1u) * 32u + piece * 8u;
      if (i0 + c >= a.v) continue;
      *reinterpret_cast<u32x4*>(a.pc + l * a.pc_plane + (((j0 >> 5) + (blk & 1u)) * (uint64_t)a.v_blocks + (i0 >> 4) + (blk >> 1)) * 1024u +
                                (u & 63u) * 16u) = *reinterpret_cast<const u32x4*>(&tile[l][c][r]);
    }
}

// ------------------------------------------------------------- the gradients
// dx of the chunk's tokens: sums over `splits` parts of the vocabulary
template <typename T, int J>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, J>::NT), 2) void k_head_dx(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, J>;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const uint32_t left = chunk_tokens(a, c0);
  const uint32_t ni = (a.h + G::TI - 1) / G::TI, nj = (left + G::TJ - 1) / G::TJ;
  const uint32_t t = die_tile(blockIdx.x, gridDim.x);
  if (t >= ni * nj * a.splits) return;
  // a part's tiles together: they share its rows of w and of the softmax
  const uint32_t split = t / (ni * nj);
  const Tile tile = tile_of(t - split * ni * nj, ni, nj);
  const uint32_t i0 = tile.i * G::TI, j0 = tile.j * G::TJ;
  const uint32_t all = (Type<T>::PLANES == 2 ? 3 : 1) * a.k_dx;
  const uint32_t s0 = (uint32_t)((uint64_t)all * split / a.splits), s1 = (uint32_t)((uint64_t)all * (split + 1) / a.splits);
  const Blocks A{a.wc, a.h_blocks, a.wc_plane}, B{a.pr, a.c_blocks, a.pr_plane};
  f32x16 acc[G::WI][G::WJ];
  G::template run<Type<T>::PLANES == 2 ? 3 : 1>(A, i0, B, j0, a.k_dx, s0, s1 - s0, lds, acc);
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
  const uint32_t iw = i0 + (wave % G::NWI) * (G::WI * 32) + h * 16, jw = j0 + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u);
#pragma unroll
  for (int y = 0; y < G::WJ; ++y)
#pragma unroll
    for (int x = 0; x < G::WI; ++x) {
      const uint32_t i = iw + x * 32, j = jw + y * 32;
      if (i >= a.hq || j >= left) continue;
      float4* o = reinterpret_cast<float4*>(a.dx_part + ((uint64_t)split * a.chunk + j) * a.hq + i);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        o[q] = make_float4(acc[x][y][q * 4], acc[x][y][q * 4 + 1], acc[x][y][q * 4 + 2], acc[x][y][q * 4 + 3]);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_head_dx_sum(const HeadArgs a, uint32_t c0) {
  using R = typename Elem<T>::raw;
  const Info info = *(const Info*)a.info;
  const uint32_t j = blockIdx.x;
  if (c0 + j >= info.count) return;
  const uint32_t i = a.rows[c0 + j];
  float f = (a.weight ? a.weight[i] : 1.0f) / P_SCALE<T>;
  if (Type<T>::PLANES == 2) f = __builtin_ldexpf(f, -plane_exp(info.top_w));
  R* o = (R*)a.dx + (uint64_t)i * a.h;
  for (uint32_t k = threadIdx.x; k < a.h; k += 256) {
    float s = 0.0f;
    for (uint32_t q = 0; q < a.splits; ++q) s += a.dx_part[((uint64_t)q * a.chunk + j) * a.hq + k];
    o[k] = Elem<T>::down(s * f);
  }
}

// dw: a tile of vocabulary entries by hidden positions, summed over the
// chunk's tokens.  One chunk: rounded to its dtype here.  More: binary32 sums
// from chunk to chunk, rounded by k_head_dw_round after the last.
template <typename T>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, 256>::NT), 2) void k_head_dw(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, 256>;
  using R = typename Elem<T>::raw;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const Info info = *(const Info*)a.info;
  const uint32_t left = chunk_tokens(a, c0);
  if (c0 > 0 && left == 0) return;
  const uint32_t ni = (a.h + G::TI - 1) / G::TI, nj = ((uint32_t)a.v + G::TJ - 1) / G::TJ;
  const uint32_t t = die_tile(blockIdx.x, gridDim.x);
  if (t >= ni * nj) return;
  const uint32_t i0 = t % ni * G::TI, j0 = t / ni * G::TJ;
  const uint32_t per = (left + KSTAGE - 1) / KSTAGE;
  const Blocks A{a.xc, a.h_blocks, a.xc_plane}, B{a.pc, a.v_blocks, a.pc_plane};
  f32x16 acc[G::WI][G::WJ];
  G::template run<Type<T>::PLANES == 2 ? 3 : 1>(A, i0, B, j0, per, 0, (Type<T>::PLANES == 2 ? 3 : 1) * per, lds, acc);
  float f = 1.0f / P_SCALE<T>;
  if (!std::is_same_v<T, bf16_t>) f *= __uint_as_float(info.top_g);
  if (Type<T>::PLANES == 2) f = __builtin_ldexpf(f, -plane_exp(info.top_x));
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
  const uint32_t iw = i0 + (wave % G::NWI) * (G::WI * 32) + h * 16, jw = j0 + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u);
#pragma unroll
  for (int y = 0; y < G::WJ; ++y)
#pragma unroll
    for (int x = 0; x < G::WI; ++x) {
      const uint32_t i = iw + x * 32, j = jw + y * 32;
      if (i >= a.h || j >= a.v) continue;
      if (a.dw_sum) {
        float* o = a.dw_sum + (uint64_t)j * a.hq + i;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float4 s = make_float4(acc[x][y][q * 4] * f, acc[x][y][q * 4 + 1] * f, acc[x][y][q * 4 + 2] * f, acc[x][y][q * 4 + 3] * f);
          if (c0 > 0) {
            const float4 old = reinterpret_cast<const float4*>(o)[q];
            s = make_float4(s.x + old.x, s.y + old.y, s.z + old.z, s.w + old.w);
          }
          reinterpret_cast<float4*>(o)[q] = s;
        }
      } else {
        R v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = Elem<T>::down(acc[x][y][r] * f);
        R* o = (R*)a.dw + (uint64_t)j * a.h + i;
        if (i + 16 <= a.h) {
          store_run<R, 16>(o, v);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (i + r < a.h) o[r] = v[r];
        }
      }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_head_dw_round(const HeadArgs a) {
  using R = typename Elem<T>::raw;
  for (uint64_t j = blockIdx.x; j < a.v; j += gridDim.x)
    for (uint32_t k = threadIdx.x; k < a.h; k += 256) ((R*)a.dw)[j * a.h + k] = Elem<T>::down(a.dw_sum[j * a.hq + k]);
}

// ------------------------------------------------------------------ launches
#define HEAD_TRY(expr)                   \
  do {                                   \
    const hipError_t e_ = (expr);        \
    if (e_ != hipSuccess) return e_;     \
  } while (0)

// a kernel with more LDS than a launch gets by default says so once per device
template <auto K>
hipError_t launch_lds(uint32_t grid, uint32_t nt, uint32_t lds, hipStream_t st, const HeadArgs& a, uint32_t c0) {
  static std::atomic<uint64_t> asked{0};
  int dev = 0;
  HEAD_TRY(hipGetDevice(&dev));
  if (dev >= 64 || !(asked.load(std::memory_order_relaxed) >> dev & 1u)) {
    HEAD_TRY(hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    if (dev < 64) asked.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL(K, dim3((grid + 7) / 8 * 8), dim3(nt), lds, st, a, c0);
  return hipGetLastError();
}

template <typename T, int J, bool GRAD>
hipError_t chunk_of(HeadArgs& a, uint32_t c0, uint32_t rows, hipStream_t st) {
  using G = Cfg<typename Type<T>::V8, J>;
  const uint32_t nj = (rows + G::TJ - 1) / G::TJ;
  const uint32_t ni = ((uint32_t)a.v + G::TI - 1) / G::TI;
  constexpr uint32_t PIECE = G::WI * 32;
  const uint32_t pieces = ((uint32_t)a.v + PIECE - 1) / PIECE;
  hipLaunchKernelGGL((k_head_pack<T, false>), dim3((a.h + 63) / 64, (rows + 63) / 64), dim3(256), 0, st, a, c0, a.xr,
                     GRAD ? a.xc : nullptr);
  HEAD_TRY(hipGetLastError());
  if constexpr (!GRAD && Type<T>::PLANES == 1) {
    if (!a.wr) {
      HEAD_TRY((launch_lds<k_head_logits<T, J, false, true>>(ni * nj, G::NT, G::LDS, st, a, c0)));
    } else {
      HEAD_TRY((launch_lds<k_head_logits<T, J, false, false>>(ni * nj, G::NT, G::LDS, st, a, c0)));
    }
  } else {
    HEAD_TRY((launch_lds<k_head_logits<T, J, GRAD, false>>(ni * nj, G::NT, G::LDS, st, a, c0)));
  }
  hipLaunchKernelGGL(k_head_loss, dim3((rows + 63) / 64), dim3(SNT), 0, st, a, c0, pieces);
  HEAD_TRY(hipGetLastError());
  if constexpr (GRAD) {
    hipLaunchKernelGGL((k_head_softmax<T>), dim3((uint32_t)(a.v + 127) / 128, (rows + 63) / 64), dim3(256), 0, st, a, c0,
                       PIECE == 128 ? 7u : 6u);
    HEAD_TRY(hipGetLastError());
    const uint32_t nh = (a.h + G::TI - 1) / G::TI;
    HEAD_TRY((launch_lds<k_head_dx<T, J>>(nh * nj * a.splits, G::NT, G::LDS, st, a, c0)));
    hipLaunchKernelGGL((k_head_dx_sum<T>), dim3(rows), dim3(256), 0, st, a, c0);
    HEAD_TRY(hipGetLastError());
    using W = Cfg<typename Type<T>::V8, 256>;
    const uint32_t tiles = ((a.h + W::TI - 1) / W::TI) * (((uint32_t)a.v + W::TJ - 1) / W::TJ);
    HEAD_TRY((launch_lds<k_head_dw<T>>(tiles, W::NT, W::LDS, st, a, c0)));
  }
  return hipSuccess;
}

template <typename T>
hipError_t head_of(HeadArgs& a, bool grad, hipStream_t st) {
  hipLaunchKernelGGL(k_head_rows, dim3(1), dim3(RNT), 0, st, a);
  HEAD_TRY(hipGetLastError());
  if (grad && a.n > 0) {
    hipLaunchKernelGGL((k_head_zero<T>), dim3((uint32_t)a.n), dim3(256), 0, st, a);
    HEAD_TRY(hipGetLastError());
  }
  if (Type<T>::PLANES == 2) {
    hipLaunchKernelGGL(k_head_top, dim3((uint32_t)std::min<uint64_t>(a.n + 1, 2048)), dim3(256), 0, st, a, false);
    HEAD_TRY(hipGetLastError());
    hipLaunchKernelGGL(k_head_top, dim3((uint32_t)std::min<uint64_t>(a.v, 2048)), dim3(256), 0, st, a, true);
    HEAD_TRY(hipGetLastError());
  }
  if (a.wr || grad) {
    hipLaunchKernelGGL((k_head_pack<T, true>), dim3((a.h + 63) / 64, ((uint32_t)a.v + 63) / 64), dim3(256), 0, st, a, 0u,
                       a.wr, grad ? a.wc : nullptr);
    HEAD_TRY(hipGetLastError());
  }
  // (without a token one chunk still writes a dw of zeros)
  for (uint64_t c0 = 0; c0 == 0 || c0 < a.n; c0 += a.chunk) {
    const uint32_t rows = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(a.chunk, a.n - c0));
    const uint32_t tokens = tile_tokens(rows), c = (uint32_t)c0;
    HEAD_TRY(tokens == 64    ? (grad ? chunk_of<T, 64, true>(a, c, rows, st) : chunk_of<T, 64, false>(a, c, rows, st))
             : tokens == 128 ? (grad ? chunk_of<T, 128, true>(a, c, rows, st) : chunk_of<T, 128, false>(a, c, rows, st))
                             : (grad ? chunk_of<T, 256, true>(a, c, rows, st) : chunk_of<T, 256, false>(a, c, rows, st)));
  }
  if (grad && a.dw_sum) {
    hipLaunchKernelGGL((k_head_dw_round<T>), dim3((uint32_t)std::min<uint64_t>(a.v, 8192)), dim3(256), 0, st, a);
    HEAD_TRY(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace

// -------------------------------------------------------------- the workspace
// Sizes and places; `base` may be null (sizes only; a null w
// counts as one that has to be laid out).  Returns the bytes.
uint64_t head_plan(HeadArgs& a, int dt, bool grad, char* base) {
  const uint64_t e = dt_size(dt), planes = dt == DT_F32 ? 2 : 1;
  auto blocks = [](uint64_t rows) { return (uint32_t)((rows + 255) / 256 * 16); };
  a.k_logits = (uint32_t)((a.h + KSTAGE - 1) / KSTAGE);
  a.k_dx = (uint32_t)((a.v + KSTAGE - 1) / KSTAGE);
  a.h_blocks = blocks(a.h);
  a.v_blocks = blocks(a.v);
  a.hq = (a.h + 15) / 16 * 16;
  // per token of a chunk: the softmax by tokens and by entries, and for
  // binary32 the numerators apart (16-bit ones are replaced in place)
  const uint64_t per_row = grad ? (uint64_t)a.k_dx * KSTAGE * (planes == 2 ? 12 : 4) : (a.v + 63) / 64 * 8;
  if (a.chunk == 0) a.chunk = HEAD_CHUNK_BYTES / per_row;
  a.chunk = std::min<uint64_t>(std::max<uint64_t>(a.chunk, 128), (a.n + 64) / 64 * 64);
  a.chunk = (a.chunk + 63) / 64 * 64;
  a.c_blocks = blocks(a.chunk);
  const bool one = a.chunk >= a.n;
  // the loss alone reads w as it is where its rows are 16-byte aligned, whole
  // stages, and near enough for 32-bit offsets within a tile
  const bool direct = !grad && planes == 1 && a.h % KSTAGE == 0 && (uintptr_t)a.w % 16 == 0 && a.ldw * e % 16 == 0 &&
                      a.ldw * e < (1u << 24);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    char* p = base ? base + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  a.info = take(sizeof(Info));
  a.rows = (uint32_t*)take(a.n * 4);
  a.zt = (float*)take(a.chunk * 4);
  a.row_lse = (float*)take(a.chunk * 4);
  a.stats = (float2*)take((a.v + 63) / 64 * a.chunk * 8);
  a.wr_plane = (uint64_t)a.v_blocks * a.k_logits * 1024;
  a.xr_plane = (uint64_t)a.c_blocks * a.k_logits * 1024;
  a.wr = direct ? nullptr : take(planes * a.wr_plane);
  a.xr = take(planes * a.xr_plane);
  if (grad) {
    const uint64_t kc = a.chunk / KSTAGE;
    a.wc_plane = (uint64_t)a.h_blocks * a.k_dx * 1024;
    a.xc_plane = (uint64_t)a.h_blocks * kc * 1024;
    a.pr_plane = (uint64_t)a.c_blocks * a.k_dx * 1024;
    a.pc_plane = (uint64_t)a.v_blocks * kc * 1024;
    a.wc = take(planes * a.wc_plane);
    a.xc = take(planes * a.xc_plane);
    a.pr = take(planes * a.pr_plane);
    a.pc = take(planes * a.pc_plane);
    a.pt = planes == 2 ? take(a.pr_plane * 2) : a.pr;
    // as many parts of the vocabulary as give every compute unit its
    // workgroups, none below 16 stages
    const uint64_t tj = tile_tokens(a.chunk), tiles = (a.h + 255) / 256 * ((a.chunk + tj - 1) / tj);
    const uint64_t stages = (planes == 2 ? 3 : 1) * (uint64_t)a.k_dx, room = (tj == 256 ? 1 : 2) * (uint64_t)device_cus();
    a.splits = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(room / std::max<uint64_t>(tiles, 1), stages / 16));
    a.dx_part = (float*)take(a.splits * a.chunk * a.hq * 4);
    a.dw_sum = one ? nullptr : (float*)take(a.v * a.hq * 4);
  }
  return at;
}

hipError_t launch_head(HeadArgs& a, int dt, bool grad, hipStream_t st) {
  return dt == DT_F32 ? head_of<float>(a, grad, st) : dt == DT_BF16 ? head_of<bf16_t>(a, grad, st) : head_of<f16_t>(a, grad, st);
}

TC_DEFINE_ERROR_READER(errors_head)

}  // namespace tc
