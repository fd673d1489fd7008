// k_head.hip -- the loss of a model's last stage: softmax cross entropy of
// x w^T over a large vocabulary, and its gradients.  No logit is stored; with
// gradients, softmax numerators of a chunk of tokens are.
//
//   z = x w^T,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_{i,t_i}
//   d_iv = g_i (exp(z_iv - lse_i) - [v = t_i]),  dx = d w,  dw = d^T x
//
// Tokens without a target are left out before anything is computed: the first
// kernel lists the others, and every later one works on that list, whose
// length stays on the device (tiles past it end at once).
//
// The loss needs one product.  Its epilogue reduces each token's logits, a
// piece of 64 vocabulary entries at a time, to their maximum and the
// sum of their exponentials; a small kernel joins the pieces.  With gradients
// the epilogue also leaves exp(z - piece's maximum), 16 bits each, so that the
// logits are computed once (6 n v h operations, not 8); another pass turns
// them in place, now that lse is known, into d, the operand of the two
// gradient products.  d exists for a chunk of tokens only.
//
// w, x and d are laid out once as blocks (tc_gemm.hpp) and used from both
// sides: dx sums over the rows of w, dw over the rows of x and d, through the
// LDS's transposing reads.
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

// How a softmax numerator (0 .. 1) is held between the two passes over it:
// in binary32 for binary32 and wherever one tile holds all tokens (J = 64;
// there the sums have too few terms to average its rounding), else in 16
// bits, none for a sign.  bfloat16 needs the range of
// binary32 rather than the bits: 7 exponent bits are all that a number up to 1
// uses, 9 mantissa bits follow them.  binary16 needs the bits: 5 exponent bits
// (2^-30, and evenly down to 2^-41) and 11 mantissa bits.
template <typename T, bool WIDE> struct Numerator {
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
template <typename T> struct Numerator<T, true> {
  using R = float;
  static __device__ __forceinline__ float down(float p) { return p; }
  static __device__ __forceinline__ float up(float p, float f) { return p * f; }
};

template <typename T, int J> constexpr bool WIDE = J == 64 || std::is_same_v<T, float>;

// A second plane of d in 16-bit types: what its rounding took.  Over many tokens
// that averages out of dw (its error against 64 bits is sqrt 2 times that of
// rounding exact sums); where up to LOW_TOKENS are left, dw, whose rows then
// often hold one token's entry, sums both planes.  Chunks of more than
// LOW_CHUNK tokens have no room for it.
constexpr uint32_t LOW_TOKENS = 512, LOW_CHUNK = 2048;

template <typename V8, int J> struct Cfg;
// 256 x 256, one workgroup of 8 wavefronts per compute unit.  For fewer tokens
// 128 x 128 and 128 x 64, two of 4 and 2 wavefronts: those products are bound
// by reading w, and with 256-row tiles a vocabulary of 32000 keeps half of the
// device busy (h 4096, w not in the caches: one token 101 us, in 128 x 128 66,
// in 128 x 64 60, 4.4 TB/s; vocabulary of 131072 320, 231 and 213; 100 tokens
// 101 and 65).
template <typename V8> struct Cfg<V8, 256> : Gemm<V8, 4, 2, 2, 4, 4> { static constexpr uint32_t PER_CU = 1; };
template <typename V8> struct Cfg<V8, 128> : Gemm<V8, 2, 2, 2, 2, 4> { static constexpr uint32_t PER_CU = 2; };
template <typename V8> struct Cfg<V8, 64> : Gemm<V8, 2, 2, 2, 1, 6> { static constexpr uint32_t PER_CU = 2; };
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

// The pattern of a magnitude for such a maximum.  Infinities and NaN stay out:
// they spoil what they take part in, and a scaling by them would all the rest.
__device__ __forceinline__ uint32_t magnitude(float v) {
  const uint32_t m = __float_as_uint(v) & 0x7FFFFFFFu;
  return m < 0x7F800000u ? m : 0u;
}

// exponent that scales a binary32 operand: the largest magnitude becomes 2^14 .. 2^15
__device__ __forceinline__ int plane_exp(uint32_t top) { return top == 0 ? 0 : 14 - ((int)(top >> 23) - 127); }

constexpr float LOG2E = 1.44269504f;

// A gradient from the sum of its products: times the largest weight, and the
// operands' scalings taken back.  Of binary32 the power of two goes to the
// product, in one step: as a factor it could lie outside of binary32 where the
// gradient does not.
template <typename T>
struct OutScale {
  float f;
  int e;
  __device__ __forceinline__ OutScale(uint32_t top_g, uint32_t top) {
    if constexpr (Type<T>::PLANES == 2) {
      f = __builtin_amdgcn_frexp_mantf(__uint_as_float(top_g));
      e = __builtin_amdgcn_frexp_expf(__uint_as_float(top_g)) - 14 - plane_exp(top);
    } else {
      f = __uint_as_float(top_g) * (1.0f / P_SCALE<T>);
    }
  }
  __device__ __forceinline__ float operator()(float s) const {
    if constexpr (Type<T>::PLANES == 2) return __builtin_ldexpf(s * f, e);
    else return s * f;
  }
};

template <typename T>
__device__ __forceinline__ uint16_t narrow(float v) {
  if constexpr (std::is_same_v<T, bf16_t>) return Elem<bf16_t>::down(v);
  else return Elem<f16_t>::down(v);
}

// ------------------------------------------------- tokens that have a target
// rows: those that have one from the front, in order, the others after them.
// NT threads take NT * RE tokens at a time; place(i, kept, at) is called for
// each with its place in the list.  Returns how many have a target.
constexpr int RE = 8;

__device__ __forceinline__ bool has_target(const HeadArgs& a, int64_t t) { return t != a.ignore && t >= 0 && (uint64_t)t < a.v; }

template <int NT, typename Place>
__device__ __forceinline__ uint32_t list_rows(const HeadArgs& a, Place place) {
  constexpr int COUNTS = RE * NT / WAVE, PER = (COUNTS + 63) / 64;
  __shared__ uint32_t part[COUNTS], all;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  uint32_t kept = 0;
  for (uint64_t i0 = 0; i0 < a.n; i0 += NT * RE) {
    int64_t t[RE];
#pragma unroll
    for (int e = 0; e < RE; ++e) {
      const uint64_t i = i0 + e * NT + threadIdx.x;
      t[e] = i < a.n ? a.target[i] : a.ignore;
    }
    uint64_t ones[RE];
#pragma unroll
    for (int e = 0; e < RE; ++e) ones[e] = __ballot(has_target(a, t[e]));
    __syncthreads();
    if (lane == 0)
#pragma unroll
      for (int e = 0; e < RE; ++e) part[e * (NT / WAVE) + wave] = (uint32_t)__popcll(ones[e]);
    __syncthreads();
    if (wave == 0) {
      // exclusive sums over the counts, PER of them a lane
      uint32_t c[PER], sum = 0;
#pragma unroll
      for (int k = 0; k < PER; ++k) sum += c[k] = lane * PER + k < COUNTS ? part[lane * PER + k] : 0u;
      const uint32_t own = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t v = (uint32_t)__shfl_up((int)sum, d);
        if (lane >= (uint32_t)d) sum += v;
      }
      uint32_t before = sum - own;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (lane * PER + k < COUNTS) part[lane * PER + k] = before;
        before += c[k];
      }
      if (lane == 63) all = sum;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < RE; ++e) {
      const uint64_t i = i0 + e * NT + threadIdx.x;
      // kept tokens before token i
      const uint32_t mine = kept + part[e * (NT / WAVE) + wave] + (uint32_t)__popcll(ones[e] & ((1ull << lane) - 1));
      const bool keep = ones[e] >> lane & 1u;
      if (i < a.n) place((uint32_t)i, keep, keep ? mine : (uint32_t)a.n - 1u - ((uint32_t)i - mine));
    }
    kept += all;
  }
  return kept;
}

// largest of a workgroup's values, in every thread
template <int NT>
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  __shared__ uint32_t part[NT / WAVE];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  __syncthreads();
  if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int k = 0; k < NT / WAVE; ++k) v = max(v, part[k]);
  return v;
}

// The list as the other kernels read it, zero losses for the others, and the
// largest weight.  also(i, keep, at) is called as list_rows would.
template <int NT, typename Also>
__device__ __forceinline__ uint32_t write_rows(const HeadArgs& a, Also also) {
  uint32_t top = 0;
  const uint32_t kept = list_rows<NT>(a, [&](uint32_t i, bool keep, uint32_t at) {
    also(i, keep, at);
    a.rows[at] = i;
    if (keep) {
      top = max(top, a.weight ? magnitude(a.weight[i]) : 0x3F800000u);
    } else {
      a.loss[i] = a.lse[i] = 0.0f;
      if (a.target[i] != a.ignore) raise_error(KERR_BAD_INDEX);
    }
  });
  top = block_max<NT>(top);
  if (threadIdx.x == 0) {
    ((Info*)a.info)->count = kept;
    ((Info*)a.info)->top_g = top;
  }
  return kept;
}

// The first workgroup lists the tokens; for binary32 the others find the
// largest magnitudes of x's rows that have a target and of w, one for each of
// top_x and top_w workgroups (k_head_pack joins them).
constexpr int BNT = 1024;

__global__ __launch_bounds__(BNT) void k_head_begin(const HeadArgs a) {
  if (blockIdx.x == 0) {
    write_rows<BNT>(a, [](uint32_t, bool, uint32_t) {});
    return;
  }
  const uint32_t b = blockIdx.x - 1u, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  const bool of_w = b >= a.top_x;
  const uint64_t rows = of_w ? a.v : a.n, first = of_w ? b - a.top_x : b, step = (of_w ? a.top_w : a.top_x) * (uint64_t)(BNT / WAVE);
  // A lane takes 4 consecutive elements, a wavefront several short rows at a
  // time, and 4 rows' loads go out together (32000 x 768: 76 -> 30 us).
  constexpr uint32_t ROWS = 4;
  struct __attribute__((packed, aligned(4))) Run { float v[4]; };
  uint32_t wide = 64;
  while (wide > 1 && wide / 2 * 4 >= a.h) wide /= 2;
  const uint32_t at_once = 64 / wide, k0 = (lane & (wide - 1)) * 4;
  uint32_t top = 0;
  for (uint64_t r = (first * (BNT / WAVE) + wave) * at_once + lane / wide; r < rows; r += step * at_once * ROWS) {
    const float* p[ROWS];
#pragma unroll
    for (uint32_t q = 0; q < ROWS; ++q) {
      // (a row that is not looked at: the one before it again, or none)
      const uint64_t row = r + q * step * at_once;
      const bool counts = row < rows && (of_w || has_target(a, a.target[row]));
      const float* own = of_w ? (const float*)a.w + row * a.ldw : (const float*)a.x + row * a.ldx;
      p[q] = counts ? own : q > 0 ? p[q - 1] : nullptr;
    }
#pragma unroll
    for (uint32_t q = ROWS - 1; q > 0; --q)
      if (!p[q - 1]) p[q - 1] = p[q];
    if (!p[0]) continue;
#pragma unroll 2
    for (uint32_t k = k0; k < a.h; k += wide * 4) {
      if (k + 4 <= a.h) {
        Run v[ROWS];
#pragma unroll
        for (uint32_t q = 0; q < ROWS; ++q) v[q] = *reinterpret_cast<const Run*>(p[q] + k);
#pragma unroll
        for (uint32_t q = 0; q < ROWS; ++q)
#pragma unroll
          for (uint32_t z = 0; z < 4; ++z) top = max(top, magnitude(v[q].v[z]));
      } else {
        for (uint32_t z = k; z < a.h; ++z)
#pragma unroll
          for (uint32_t q = 0; q < ROWS; ++q) top = max(top, magnitude(p[q][z]));
      }
    }
  }
  top = block_max<BNT>(top);
  if (threadIdx.x == 0) a.tops[b] = top;
}

// ------------------------------------------------------ operands laid out
// x (the chunk's listed rows) or w into blocks, zeros past the end of a row
// and in the rows that fill the last stage of a sum over rows; binary32 as
// two planes.  A workgroup takes 16 rows by 512 elements, a lane a piece of 8.
constexpr uint32_t PACK_KB = 16;

template <typename T, bool OF_W>
__device__ __forceinline__ void pack_rows(const HeadArgs& a, uint32_t rows, const uint32_t* list, uint32_t top, uint32_t rb, uint32_t kb0) {
  using R = typename Elem<T>::raw;
  constexpr int PL = Type<T>::PLANES;
  if (rb * 16u >= (rows + KSTAGE - 1) / KSTAGE * KSTAGE) return;
  const int e = PL == 2 ? plane_exp(top) : 0;
  const uint32_t lane = threadIdx.x & 63u, row = lane >> 2, piece = (lane & 3u) ^ turn(row), r = rb * 16u + row;
  const R* src = nullptr;
  if (r < rows) src = (const R*)(OF_W ? a.w : a.x) + (uint64_t)(OF_W ? r : list[row]) * (OF_W ? a.ldw : a.ldx);
  struct __attribute__((packed, aligned(sizeof(R)))) Run { R v[8]; };
#pragma unroll
  for (uint32_t q = 0; q < PACK_KB / 4; ++q) {
    const uint32_t kb = kb0 + q * 4u + (threadIdx.x >> 6), k = kb * 32u + piece * 8u;
    if (kb >= a.k_logits) break;
    Run v = {};
    if (src) {
      if (k + 8 <= a.h) v = *reinterpret_cast<const Run*>(src + k);
      else
#pragma unroll
        for (uint32_t z = 0; z < 8; ++z)
          if (k + z < a.h) v.v[z] = src[k + z];
    }
    char* o = (OF_W ? a.wr : a.xr) + ((uint64_t)kb * (OF_W ? a.v_blocks : a.c_blocks) + rb) * 1024u + lane * 16u;
    if constexpr (PL == 2) {
      uint16_t hi[8], lo[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const float s = __builtin_ldexpf(v.v[z], e);
        hi[z] = Elem<f16_t>::down(s);
        lo[z] = (hi[z] & 0x7FFFu) == 0x7C00u ? (uint16_t)0 : Elem<f16_t>::down(s - Elem<f16_t>::up(hi[z]));
      }
      __builtin_memcpy(o, hi, 16);
      __builtin_memcpy(o + (OF_W ? a.wr_plane : a.xr_plane), lo, 16);
    } else {
      __builtin_memcpy(o, v.v, 16);
    }
  }
}

// The first `of_w` workgroups lay out w, the others the chunk's tokens.
// ALONE: there is no k_head_begin before it; with few tokens each workgroup
// lists them for itself, which takes less time than a launch.
constexpr uint32_t ALONE_TOKENS = 256 * RE;

template <typename T, bool ALONE>
__global__ __launch_bounds__(256) void k_head_pack(const HeadArgs a, uint32_t c0, uint32_t of_w) {
  __shared__ uint32_t list[16];
  const uint32_t wide = (a.k_logits + PACK_KB - 1) / PACK_KB;
  const bool is_w = blockIdx.x < of_w;
  const uint32_t b = is_w ? blockIdx.x : blockIdx.x - of_w, rb = b / wide, kb0 = b % wide * PACK_KB;
  uint32_t top = 0;
  if constexpr (Type<T>::PLANES == 2) {
    // (the last workgroup leaves both for the kernels after this one)
    const uint32_t x = block_max<256>(threadIdx.x < a.top_x ? a.tops[threadIdx.x] : 0u);
    const uint32_t w = block_max<256>(threadIdx.x < a.top_w ? a.tops[a.top_x + threadIdx.x] : 0u);
    top = is_w ? w : x;
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) {
      ((Info*)a.info)->top_x = x;
      ((Info*)a.info)->top_w = w;
    }
  }
  if (is_w) {
    pack_rows<T, true>(a, (uint32_t)a.v, nullptr, top, rb, kb0);
    return;
  }
  uint32_t rows;
  if constexpr (ALONE) {
    auto mine = [&](uint32_t i, bool keep, uint32_t at) {
      if (keep && at >> 4 == rb) list[at & 15u] = i;
    };
    rows = b == 0 ? write_rows<256>(a, mine) : list_rows<256>(a, mine);
  } else {
    rows = chunk_tokens(a, c0);
    if (threadIdx.x < 16 && rb * 16u + threadIdx.x < rows) list[threadIdx.x] = a.rows[c0 + rb * 16u + threadIdx.x];
  }
  __syncthreads();
  pack_rows<T, false>(a, rows, list, top, rb, kb0);
}

// ---------------------------------------------------------------- the logits
// Tile order: 8 tiles of j wide, so that the workgroups that run together on a
// die share rows of both operands.
struct Tile { uint32_t i, j; };
__device__ __forceinline__ Tile tile_of(uint32_t t, uint32_t ni, uint32_t nj) {
  const uint32_t group = t / (8u * ni), rem = t - group * 8u * ni, width = min(8u, nj - group * 8u);
  return {rem / width, group * 8u + rem % width};
}

// The n-th of a workgroup's tiles out of `total` (false: it has no more).
// Many tiles: every die takes an eighth of them in a row; few: every round of
// tiles is dealt out anew.  (Losses in a row against dealt out, us, vocabularies
// of 16384 to 131072, 4096 to 8192 tokens.  h 4096: 12 rounds 1318, 1327; 16
// 1641, 1658; 24 2448, 2494; 32 3252, 3330; 64 6503, 6650.  h 2048: 12 693,
// 693; 24 1282, 1290; 32 1695, 1722; 64 3354, 3450.  h 768: 12 316, 317; 16 388,
// 383; 24 555, 557; 32 730, 722; 64 1444, 1427.)
__device__ __forceinline__ bool nth_tile(uint32_t n, uint32_t total, uint32_t& t) {
  if (total >= 32u * gridDim.x) {
    const uint32_t per = (total + 7u) >> 3, local = n * (gridDim.x >> 3) + (blockIdx.x >> 3);
    t = (blockIdx.x & 7u) * per + local;
    return local < per && t < total;
  }
  t = n * gridDim.x + die_tile(blockIdx.x, gridDim.x);
  return t < total;
}

// The thread, for what is done after a tile: opaque, or all addresses that
// follow from it are computed before the tiles' loop and held throughout, in
// registers that there are not (score of 4096 x 50257 x 768: 294 -> 287 us).
__device__ __forceinline__ uint32_t own_thread() {
  uint32_t t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// pt: softmax numerators relative to their piece's maximum, in the blocks of d
// (in binary32: blocks of 2 KB, pieces where they are)
template <typename T, int J, bool GRAD, bool DIRECT>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, J>::NT), 2) void k_head_logits(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, J>;
  constexpr int PL = Type<T>::PLANES;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const Info info = *(const Info*)a.info;
  const uint32_t left = chunk_tokens(a, c0);
  const uint32_t ni = ((uint32_t)a.v + G::TI - 1) / G::TI, nj = (left + G::TJ - 1) / G::TJ;
  const uint32_t per = a.k_logits, count = (PL == 2 ? 3 : 1) * per;
  auto work = [&](uint32_t n, typename G::Work& w) {
    uint32_t t;
    if (!nth_tile(n, ni * nj, t)) return false;
    const Tile tile = tile_of(t, ni, nj);
    w = {tile.i * G::TI, tile.j * G::TJ, 0u, count};
    return true;
  };
  const Blocks B{a.xr, a.c_blocks, a.xr_plane};
  auto done = [&](uint32_t, const typename G::Work& at, f32x16 (&acc)[G::WI][G::WJ]) {
    const uint32_t thread = own_thread();
    const uint32_t lane = thread & 63u, wave = __builtin_amdgcn_readfirstlane(thread >> 6), h = lane >> 5;
    const uint32_t iw = at.i0 + (wave % G::NWI) * (G::WI * 32), jw = at.j0 + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u);
    if (iw >= a.v) return;
    const uint32_t piece = iw / (G::WI * 32);
    const int back = Type<T>::PLANES == 2 ? -plane_exp(info.top_w) - plane_exp(info.top_x) : 0;
    // entries past the vocabulary's end, in its last tile
    if (iw + G::WI * 32 > a.v) {
#pragma unroll
      for (int y = 0; y < G::WJ; ++y)
#pragma unroll
        for (int x = 0; x < G::WI; ++x)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (iw + x * 32 + h * 16 + r >= a.v) acc[x][y][r] = -__builtin_inff();
    }
#pragma unroll
    for (int y = 0; y < G::WJ; ++y) {
      const uint32_t j = jw + y * 32;
      float top = -__builtin_inff();
#pragma unroll
      for (int x = 0; x < G::WI; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (Type<T>::PLANES == 2) acc[x][y][r] = __builtin_ldexpf(acc[x][y][r], back);
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
      // The maximum comes off before the scaling: its entry is 1 exactly and no
      // other is more, whatever the logits' size (off the scaled one, rounding
      // would move all entries by 2^-24 of the logit in the exponent, and from
      // logits of 1e7 on the largest out of a numerator's range).
      // (a piece of logits that are all -inf adds nothing)
      const float base = top > -__builtin_inff() ? top : 0.0f;
#pragma unroll
      for (int x = 0; x < G::WI; ++x) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f((acc[x][y][r] - base) * LOG2E);
          acc[x][y][r] = p;
          sum += p;
        }
        if (GRAD && j < left) {
          const uint32_t kb = (iw >> 5) + x;
          if (kb < a.k_dx) {
            using N = Numerator<T, WIDE<T, J>>;
            using R = typename N::R;
            R v[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) v[r] = N::down(acc[x][y][r]);
            constexpr uint32_t PIECE = 8 * sizeof(R);
            char* o = a.pt + ((uint64_t)kb * a.c_blocks + (j >> 4)) * (64u * PIECE) + (j & 15u) * 4u * PIECE;
            if constexpr (WIDE<T, J>) {
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
  };
  if constexpr (DIRECT) {
    const Rows A{(const char*)a.w, a.ldw * 2, (uint32_t)a.v};
    G::template stream<1>(A, B, per, lds, work, done);
  } else {
    const Blocks A{a.wr, a.v_blocks, a.wr_plane};
    G::template stream<PL == 2 ? 3 : 1>(A, B, per, lds, work, done);
  }
}

// ------------------------------------------------- pieces joined, the losses
// and what d needs to know of a token: the largest logit, the weight over the
// sum of exponentials, the target, and d at the target.  (lse would do for the
// first two, but of large logits it is known to 2^-24 of their size only.)  The
// weight is a share of the largest (for binary16's range; and with equal
// weights the entries of unlikely targets are nearly -1 and not all off by the
// rounding of one weight).
constexpr int SNT = 1024, SR = 16;     // threads, tokens of a workgroup

__global__ __launch_bounds__(SNT) void k_head_loss(const HeadArgs a, uint32_t c0, uint32_t pieces) {
  __shared__ float2 part[SNT / SR][SR];
  const uint32_t left = chunk_tokens(a, c0);
  const uint32_t r = threadIdx.x % SR, q = threadIdx.x / SR, j = blockIdx.x * SR + r;
  if (blockIdx.x * SR >= left) return;
  float m = -__builtin_inff(), s = 0.0f;
  if (j < left) {
    constexpr uint32_t B = 8;         // pieces at a time: their loads go out together
    for (uint32_t p = q; p < pieces; p += B * (SNT / SR)) {
      float2 v[B];
      float top = m;
#pragma unroll
      for (uint32_t k = 0; k < B; ++k) {
        const uint32_t at = p + k * (SNT / SR);
        v[k] = at < pieces ? a.stats[(uint64_t)at * a.chunk + j] : make_float2(-__builtin_inff(), 0.0f);
      }
#pragma unroll
      for (uint32_t k = 0; k < B; ++k) top = fmaxf(top, v[k].x);
      // (where all logits are -inf so far the sums are 0, or NaN where one is)
      const bool any = top > -__builtin_inff();
      s *= any ? __expf(m - top) : 1.0f;
#pragma unroll
      for (uint32_t k = 0; k < B; ++k) s = __builtin_fmaf(v[k].y, any ? __expf(v[k].x - top) : 1.0f, s);
      m = top;
    }
  }
  part[q][r] = make_float2(m, s);
  __syncthreads();
  // 64 parts of each token: 4 by every of 16 threads, those by their shuffles
  const uint32_t rr = threadIdx.x / 16u, qq = threadIdx.x % 16u;
  if (rr < SR) {
    m = -__builtin_inff();
    for (uint32_t k = qq; k < SNT / SR; k += 16) m = fmaxf(m, part[k][rr].x);
    for (uint32_t d = 8; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    s = 0.0f;
    for (uint32_t k = qq; k < SNT / SR; k += 16) s += part[k][rr].y * __expf(part[k][rr].x - m);
    for (uint32_t d = 8; d > 0; d >>= 1) s += __shfl_xor(s, d);
  }
  const uint32_t jj = blockIdx.x * SR + rr;
  if (rr < SR && qq == 0 && jj < left) {
    // (the difference first: a small loss is not the difference of two large numbers)
    const float log_s = logf(s), lse = m + log_s, loss = (m - a.zt[jj]) + log_s;
    const uint32_t i = a.rows[c0 + jj];
    a.lse[i] = lse;
    a.loss[i] = loss;
    if (a.row_info) {
      const float g = a.weight ? a.weight[i] : 1.0f, most = __uint_as_float(((const Info*)a.info)->top_g);
      const float weight = most > 0.0f ? g / most : g;
      a.row_info[jj] = make_float4(m, weight / s, __uint_as_float((uint32_t)a.target[i]), expm1f(-loss) * weight);
    }
  }
}

// --------------------------------- d: softmax minus target, times the weight
// A workgroup takes 128 tokens by up to 128 vocabulary entries, a lane half a
// row of a block (32 bytes) at a time: one pass over the memory, bound by it.

template <typename T, int J, bool LOW>
__global__ __launch_bounds__(256, 5) void k_head_softmax(const HeadArgs a, uint32_t c0, uint32_t piece_bits, uint32_t blocks) {
  constexpr int PL = LOW ? 2 : Type<T>::PLANES;
  using N = Numerator<T, WIDE<T, J>>;
  using R = typename N::R;
  // (the tokens that the logits' kernel wrote last, and the caches may hold, first)
  const uint32_t left = chunk_tokens(a, c0), j = (gridDim.y - 1u - blockIdx.y) * 128u + (threadIdx.x >> 1), half = threadIdx.x & 1u;
  // (rows that fill the last stage of the sum over tokens are zeros)
  if (j >= (left + KSTAGE - 1) / KSTAGE * KSTAGE) return;
  const bool in = j < left;
  using D = std::conditional_t<std::is_same_v<T, float>, f16_t, T>;
  const int planes = LOW && left > LOW_TOKENS ? 1 : PL;
  const float4 row = in ? a.row_info[j] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const uint32_t goal = __float_as_uint(row.z);
  const float w = row.y * P_SCALE<T>;
#pragma unroll 4
  for (uint32_t kb = blockIdx.x * blocks; kb < min(a.k_dx, blockIdx.x * blocks + blocks); ++kb) {
    const uint64_t at = ((uint64_t)kb * a.c_blocks + (j >> 4)) * 64u + (j & 15u) * 4u;    // in pieces
    uint16_t v[PL][16] = {};
    if (in) {
      const float f = __expf(a.stats[(uint64_t)((kb * 32u) >> piece_bits) * a.chunk + j].x - row.x);
#pragma unroll
      for (uint32_t z = 0; z < 2; ++z) {
        const uint32_t place = 2u * half + z, piece = place ^ turn(j);
        R n[8];
        __builtin_memcpy(n, a.pt + (at + (WIDE<T, J> ? piece : place)) * sizeof(n), sizeof(n));
#pragma unroll
        for (uint32_t y = 0; y < 8; ++y) {
          const float p = N::up(n[y], f) * w;
          const uint16_t hi = narrow<T>(p);
          v[0][z * 8 + y] = hi;
          if constexpr (PL == 2) v[1][z * 8 + y] = narrow<T>(p - Elem<D>::up(hi));
        }
      }
    }
#pragma unroll
    for (int l = 0; l < PL; ++l)
      if (l < planes) __builtin_memcpy(a.pr + l * a.pr_plane + (at + 2u * half) * 16u, v[l], 32);
    // the target's entry, from the loss (its numerator less 1 would be a small
    // difference) and after the others (no entry is compared with the target)
    if (in && goal >> 5 == kb && (((goal >> 3 & 3u) ^ turn(j)) >> 1) == half) {
      const float p = row.w * P_SCALE<T>;
      const uint16_t hi = narrow<T>(p);
      const float low = p - Elem<D>::up(hi);
      char* o = a.pr + (at + ((goal >> 3 & 3u) ^ turn(j))) * 16u + (goal & 7u) * 2u;
      *reinterpret_cast<uint16_t*>(o) = hi;
      // (the largest entry of most tokens: dx adds what its rounding took)
      if (Type<T>::PLANES == 1) a.rest[j] = low;
      if (PL == 2 && planes == 2) *reinterpret_cast<uint16_t*>(o + a.pr_plane) = narrow<T>(low);
    }
  }
}

// ------------------------------------------------------------- the gradients
// dx of the chunk's tokens: sums over parts of the vocabulary.  The host
// chose their number for a full chunk; where tokens without a target left
// fewer tiles than workgroups, the tokens that are left have room for more.
struct DxPlan {
  uint32_t ni, nj, all, splits;
  __device__ __forceinline__ DxPlan(const HeadArgs& a, uint32_t left, uint32_t ti, uint32_t tj, uint32_t pairs) {
    ni = (a.h + ti - 1) / ti;
    nj = (left + tj - 1) / tj;
    all = pairs * a.k_dx;
    splits = a.splits;
    const uint32_t tiles = max(ni * nj, 1u), room = (uint32_t)min((uint64_t)a.splits * a.chunk / max(left, 1u), (uint64_t)max(all / 16u, 1u));
    const uint32_t more = min(a.dx_grid / tiles, room);
    // (rounds of tiles, by the length of a part)
    auto rounds = [&](uint32_t s) { return (tiles * s + a.dx_grid - 1) / a.dx_grid; };
    if (more > splits && (uint64_t)rounds(more) * splits < (uint64_t)rounds(splits) * more) splits = more;
  }
};

template <typename T, int J>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, J>::NT), 2) void k_head_dx(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, J>;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const uint32_t left = chunk_tokens(a, c0);
  const DxPlan plan(a, left, G::TI, G::TJ, Type<T>::PLANES == 2 ? 3 : 1);
  const uint32_t tiles = plan.ni * plan.nj, all = plan.all, splits = plan.splits;
  auto work = [&](uint32_t n, typename G::Work& w) {
    uint32_t t;
    if (!nth_tile(n, tiles * splits, t)) return false;
    // a part's tiles together: they share its rows of w and of d
    const uint32_t split = t / tiles;
    const Tile tile = tile_of(t - split * tiles, plan.ni, plan.nj);
    const uint32_t s0 = (uint32_t)((uint64_t)all * split / splits), s1 = (uint32_t)((uint64_t)all * (split + 1) / splits);
    w = {tile.i * G::TI, tile.j * G::TJ, s0, s1 - s0};
    return true;
  };
  auto done = [&](uint32_t, const typename G::Work& at, f32x16 (&acc)[G::WI][G::WJ]) {
    const uint32_t thread = own_thread();
    const uint32_t lane = thread & 63u, wave = __builtin_amdgcn_readfirstlane(thread >> 6), h = lane >> 5;
    const uint32_t iw = at.i0 + (wave % G::NWI) * (G::WI * 32) + h * 16, jw = at.j0 + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u);
    // (the part that starts at s0: the first that does not end before it)
    uint32_t split = (uint32_t)((uint64_t)at.s0 * splits / all);
    if ((uint64_t)all * split / splits != at.s0) ++split;
#pragma unroll
    for (int y = 0; y < G::WJ; ++y)
#pragma unroll
      for (int x = 0; x < G::WI; ++x) {
        const uint32_t i = iw + x * 32, j = jw + y * 32;
        if (i >= a.hq || j >= left) continue;
        float4* o = reinterpret_cast<float4*>(a.dx_part + ((uint64_t)split * left + j) * a.hq + i);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          o[q] = make_float4(acc[x][y][q * 4], acc[x][y][q * 4 + 1], acc[x][y][q * 4 + 2], acc[x][y][q * 4 + 3]);
      }
  };
  const BlocksT A{a.wr, a.v_blocks, a.wr_plane};
  const Blocks B{a.pr, a.c_blocks, a.pr_plane};
  G::template stream<Type<T>::PLANES == 2 ? 3 : 1>(A, B, a.k_dx, lds, work, done);
}

// dx of the list's places c0 + blockIdx.x: the parts' sum, and what the target's entry of d lost when it was rounded:
// for a token that the model is sure of, dx is a small difference and that
// entry's rounding would be most of its error.
template <typename T>
__global__ __launch_bounds__(256) void k_head_dx_sum(const HeadArgs a, uint32_t c0, uint32_t ti, uint32_t tj) {
  using R = typename Elem<T>::raw;
  const Info info = *(const Info*)a.info;
  const uint32_t j = blockIdx.x, i = a.rows[c0 + j];
  R* o = (R*)a.dx + (uint64_t)i * a.h;
  if (c0 + j >= info.count) {
    // (a token without a target)
    for (uint32_t k = threadIdx.x; k < a.h; k += 256) o[k] = R{};
    return;
  }
  const OutScale<T> scaled(info.top_g, info.top_w);
  const uint32_t left = chunk_tokens(a, c0), splits = DxPlan(a, left, ti, tj, Type<T>::PLANES == 2 ? 3 : 1).splits;
  const float rest = Type<T>::PLANES == 1 ? a.rest[j] : 0.0f;
  const R* w = (const R*)a.w + (uint64_t)a.target[i] * a.ldw;
  for (uint32_t k = threadIdx.x; k < a.h; k += 256) {
    float s = 0.0f;
#pragma unroll 4
    for (uint32_t q = 0; q < splits; ++q) s += a.dx_part[((uint64_t)q * left + j) * a.hq + k];
    if (Type<T>::PLANES == 1) s += rest * Elem<T>::up(w[k]);
    o[k] = Elem<T>::down(scaled(s));
  }
}

// dw: tiles of vocabulary entries by hidden positions, summed over the chunk's
// tokens.  Whole rounds of tiles (one for every workgroup) are summed by one
// workgroup each; those of the last, partial round are split along the
// tokens, so that it takes a part of a round, and joined by k_head_dw_tail.
// One chunk: rounded to its dtype here.  More: binary32 sums from chunk to
// chunk, rounded by k_head_dw_round after the last.
template <typename T, int W>
struct DwPlan {
  using G = Cfg<typename Type<T>::V8, W>;
  uint32_t ni, nj, whole, rest, all, parts;
  __device__ __forceinline__ DwPlan(const HeadArgs& a, uint32_t left) {
    ni = (a.h + G::TI - 1) / G::TI;
    nj = ((uint32_t)a.v + G::TJ - 1) / G::TJ;
    whole = a.dw_parts ? ni * nj / a.dw_grid * a.dw_grid : ni * nj;
    rest = ni * nj - whole;
    all = (Type<T>::PLANES == 2 ? 3 : a.d_low && left <= LOW_TOKENS ? 2 : 1) * ((left + KSTAGE - 1) / KSTAGE);
    parts = min(a.dw_parts, all);       // (each has a stage at least)
  }
  __device__ __forceinline__ Tile tile(uint32_t t) const {
    const Tile x = tile_of(t, nj, ni);
    return {x.j, x.i};
  }
};

template <typename T>
__device__ __forceinline__ void dw_store(const HeadArgs& a, uint32_t c0, const OutScale<T>& scaled, uint32_t i, uint32_t j, const float (&v)[16]) {
  using R = typename Elem<T>::raw;
  if (i >= a.h || j >= a.v) return;
  if (a.dw_sum) {
    float* o = a.dw_sum + (uint64_t)j * a.hq + i;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float4 s = make_float4(scaled(v[q * 4]), scaled(v[q * 4 + 1]), scaled(v[q * 4 + 2]), scaled(v[q * 4 + 3]));
      if (c0 > 0) {
        const float4 old = reinterpret_cast<const float4*>(o)[q];
        s = make_float4(s.x + old.x, s.y + old.y, s.z + old.z, s.w + old.w);
      }
      reinterpret_cast<float4*>(o)[q] = s;
    }
  } else {
    R w[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] = Elem<T>::down(scaled(v[r]));
    R* o = (R*)a.dw + (uint64_t)j * a.h + i;
    if (i + 16 <= a.h) {
      // (the hardware stores vectors at any element's address)
      struct __attribute__((packed, aligned(sizeof(R)))) Run { uint32_t w[4]; } run[sizeof(w) / 16];
      __builtin_memcpy(run, w, sizeof(w));
#pragma unroll
      for (uint32_t q = 0; q < sizeof(w) / 16; ++q) {
        reinterpret_cast<Run*>(o)[q] = run[q];
        // (else the compiler joins and splits them into pieces of 12 and 4 bytes)
        asm volatile("" ::: "memory");
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (i + r < a.h) o[r] = w[r];
    }
  }
}

// A wavefront's sums, rounded, into rows of dw.  A lane has 16 consecutive
// elements of a row, 32 or 64 bytes; stored as they are, 64 lanes touch 32 rows
// at once.  Through 4 KB of the LDS they become runs of 256 bytes of 4 rows
// (1024 tokens, 32768 entries, h 4096 in bfloat16: dw 383 -> 275 us).
// (The LDS is reached by instructions written out: the compiler would have
// every one of them wait for the stages that are being loaded.)  Piece p of row
// r lies at place p ^ r, so that the 16 rows of a write are in different banks.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t RUN_LDS = 4096;       // of a wavefront: 16 rows of 256 bytes

template <typename T, int WI, int WJ>
__device__ __forceinline__ void dw_store_runs(const HeadArgs& a, const OutScale<T>& scaled, char* lds, uint32_t lane, uint32_t i0, uint32_t j0, f32x16 (&acc)[WI][WJ]) {
  using R = typename Elem<T>::raw;
  // XF fragments side by side make a run (128 bytes where a wavefront has no
  // more), Q pieces of PER elements to a lane's row of each
  constexpr uint32_t E = sizeof(R), XF = 8 / E < WI ? 8 / E : WI, RUN = XF * 32, Q = E, PER = 16 / E;
  constexpr uint32_t PIECES = RUN / PER, READ_ROWS = 64 / PIECES, READS = 16 / READ_ROWS;
  static_assert(WI % XF == 0 && (READS == 2 || READS == 4), "whole runs");
  struct __attribute__((packed, aligned(sizeof(R)))) Run { u32x4 w; };
  struct __attribute__((packed, aligned(sizeof(R)))) Run8 { uint32_t w[2]; };
  struct __attribute__((packed, aligned(sizeof(R)))) Run4 { uint32_t w; };
  const uint32_t h = lane >> 5, r = lane & 15u, p = lane % PIECES, group = lane / PIECES;
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const uint32_t to = at + r * RUN * E;
  uint32_t from[READS];
#pragma unroll
  for (uint32_t q = 0; q < READS; ++q) {
    const uint32_t row = q * READ_ROWS + group;
    from[q] = at + (row * PIECES + (p ^ (row % PIECES))) * 16u;
  }
#pragma unroll
  for (int y = 0; y < WJ; ++y)
#pragma unroll
    for (uint32_t g = 0; g < WI / XF; ++g) {
      // (one run's values in registers at a time)
      __builtin_amdgcn_sched_barrier(0);
      u32x4 v[XF][Q];
#pragma unroll
      for (uint32_t x = 0; x < XF; ++x) {
        R w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = Elem<T>::down(scaled(acc[g * XF + x][y][e]));
        __builtin_memcpy(v[x], w, sizeof(w));
      }
#pragma unroll
      for (uint32_t s = 0; s < 2; ++s) {
        if ((lane >> 4 & 1u) == s) {
#pragma unroll
          for (uint32_t x = 0; x < XF; ++x)
#pragma unroll
            for (uint32_t q = 0; q < Q; ++q)
              asm volatile("ds_write_b128 %0, %1" ::"v"(to + (((x * 2u + h) * Q + q) ^ (r % PIECES)) * 16u), "v"(v[x][q]) : "memory");
        }
        __builtin_amdgcn_sched_barrier(0);
        u32x4 o[READS];
        if constexpr (READS == 4)
          asm volatile("s_waitcnt lgkmcnt(0)\n\tds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\t"
                       "ds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                       : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3])
                       : "v"(from[0]), "v"(from[1]), "v"(from[2]), "v"(from[3])
                       : "memory");
        else
          asm volatile("s_waitcnt lgkmcnt(0)\n\tds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)"
                       : "=&v"(o[0]), "=&v"(o[1])
                       : "v"(from[0]), "v"(from[1])
                       : "memory");
        const uint32_t i = i0 + g * RUN + p * PER;
#pragma unroll
        for (uint32_t q = 0; q < READS; ++q) {
          const uint32_t j = j0 + y * 32u + s * 16u + q * READ_ROWS + group;
          if (j >= a.v || i >= a.h) continue;
          R* d = (R*)a.dw + (uint64_t)j * a.h + i;
          // (the hardware stores vectors at any element's address)
          if (i + PER <= a.h) {
            *reinterpret_cast<Run*>(d) = {o[q]};
          } else {
            const uint32_t bytes = (a.h - i) * E;
            char* c = (char*)d;
            if (bytes & 8u) {
              *reinterpret_cast<Run8*>(c) = {{o[q].x, o[q].y}};
              o[q].x = o[q].z;
              o[q].y = o[q].w;
              c += 8;
            }
            if (bytes & 4u) {
              *reinterpret_cast<Run4*>(c) = {o[q].x};
              o[q].x = o[q].y;
              c += 4;
            }
            if (E == 2 && (bytes & 2u)) *reinterpret_cast<uint16_t*>(c) = (uint16_t)o[q].x;
          }
        }
      }
    }
}

template <typename T>
__device__ __forceinline__ OutScale<T> dw_scale(const HeadArgs& a) {
  const Info info = *(const Info*)a.info;
  return OutScale<T>(info.top_g, info.top_x);
}

template <typename T, int W, bool LOW>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, W>::NT), 2) void k_head_dw(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, W>;
  extern __shared__ __attribute__((aligned(128))) char lds[];
  const uint32_t left = chunk_tokens(a, c0);
  if (c0 > 0 && left == 0) return;
  const DwPlan<T, W> plan(a, left);
  const OutScale<T> scaled = dw_scale<T>(a);
  const uint32_t mine = die_tile(blockIdx.x, gridDim.x);
  auto done = [&](uint32_t n, const typename G::Work& at, f32x16 (&acc)[G::WI][G::WJ]) {
    const uint32_t thread = own_thread();
    const uint32_t lane = thread & 63u, wave = __builtin_amdgcn_readfirstlane(thread >> 6), h = lane >> 5;
    const uint32_t iw = at.i0 + (wave % G::NWI) * (G::WI * 32) + h * 16, jw = at.j0 + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u);
    const bool part = a.dw_parts && n * gridDim.x >= plan.whole;
    if (!part && !a.dw_sum) {
      dw_store_runs<T>(a, scaled, lds + G::LDS + wave * RUN_LDS, lane, iw - h * 16, jw - (lane & 31u), acc);
      return;
    }
#pragma unroll
    for (int y = 0; y < G::WJ; ++y)
#pragma unroll
      for (int x = 0; x < G::WI; ++x) {
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = acc[x][y][r];
        if (part) {
          if (iw + x * 32 >= a.h || jw + y * 32 >= a.v) continue;
          // as the lanes hold them: k_head_dw_tail reads them the same way
          float4* o = reinterpret_cast<float4*>(a.dw_part + ((uint64_t)mine * (G::WI * G::WJ) + y * G::WI + x) * (G::NT * 16)) + thread;
#pragma unroll
          for (int q = 0; q < 4; ++q) o[q * G::NT] = make_float4(v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]);
        } else {
          dw_store<T>(a, c0, scaled, iw + x * 32, jw + y * 32, v);
        }
      }
  };
  if (left == 0) {
    // nothing to sum: zeros
    for (uint64_t r = blockIdx.x; r < a.v; r += gridDim.x)
      for (uint32_t k = threadIdx.x; k < a.h; k += G::NT) {
        if (a.dw_sum) a.dw_sum[r * a.hq + k] = 0.0f;
        else ((typename Elem<T>::raw*)a.dw)[r * a.h + k] = {};
      }
    return;
  }
  auto work = [&](uint32_t n, typename G::Work& w) {
    uint32_t t = n * gridDim.x + mine, s0 = 0, s1 = plan.all;
    if (!a.dw_parts) {
      if (t >= plan.whole) return false;
    } else if (n * gridDim.x >= plan.whole) {
      if (n * gridDim.x > plan.whole || mine >= plan.rest * plan.parts) return false;
      const uint32_t split = mine / plan.rest;
      t = plan.whole + mine - split * plan.rest;
      s0 = plan.all * split / plan.parts;
      s1 = plan.all * (split + 1) / plan.parts;
    }
    const Tile x = plan.tile(t);
    w = {x.i * G::TI, x.j * G::TJ, s0, s1 - s0};
    return true;
  };
  const BlocksT A{a.xr, a.c_blocks, a.xr_plane}, B{a.pr, a.c_blocks, a.pr_plane};
  G::template stream<Type<T>::PLANES == 2 ? 3 : LOW ? 2 : 1>(A, B, (left + KSTAGE - 1) / KSTAGE, lds, work, done);
}

// one fragment row of a tile of the last round per workgroup
template <typename T, int W>
__global__ __launch_bounds__((Cfg<typename Type<T>::V8, W>::NT)) void k_head_dw_tail(const HeadArgs a, uint32_t c0) {
  using G = Cfg<typename Type<T>::V8, W>;
  const uint32_t left = chunk_tokens(a, c0);
  if (left == 0) return;
  const DwPlan<T, W> plan(a, left);
  const uint32_t tile = blockIdx.x / (G::WI * G::WJ), xy = blockIdx.x % (G::WI * G::WJ), x = xy % G::WI, y = xy / G::WI;
  float v[16] = {};
  for (uint32_t p = 0; p < plan.parts; ++p) {
    const float4* s = reinterpret_cast<const float4*>(a.dw_part + ((uint64_t)(p * plan.rest + tile) * (G::WI * G::WJ) + xy) * (G::NT * 16)) + threadIdx.x;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 u = s[q * G::NT];
      v[q * 4] += u.x;
      v[q * 4 + 1] += u.y;
      v[q * 4 + 2] += u.z;
      v[q * 4 + 3] += u.w;
    }
  }
  const Tile at = plan.tile(plan.whole + tile);
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
  const uint32_t i = at.i * G::TI + (wave % G::NWI) * (G::WI * 32) + h * 16 + x * 32;
  const uint32_t j = at.j * G::TJ + (wave / G::NWI) * (G::WJ * 32) + (lane & 31u) + y * 32;
  dw_store<T>(a, c0, dw_scale<T>(a), i, j, v);
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
  hipLaunchKernelGGL(K, dim3(grid), dim3(nt), lds, st, a, c0);
  return hipGetLastError();
}

// workgroups of a product's kernel: as many as run at once, or as there are
// tiles, in eights
template <typename G>
uint32_t grid_of(uint64_t tiles) {
  const uint64_t room = (uint64_t)(device_cus() * G::PER_CU + 7) / 8 * 8;
  return (uint32_t)std::min<uint64_t>(room, (tiles + 7) / 8 * 8);
}

// whether k_head_pack lists the tokens by itself
template <typename T>
bool alone(const HeadArgs& a) { return Type<T>::PLANES == 1 && a.n <= ALONE_TOKENS && a.n <= a.chunk; }

template <typename T, int W>
hipError_t launch_dw(const HeadArgs& a, uint32_t c0, hipStream_t st) {
  using G = Cfg<typename Type<T>::V8, W>;
  constexpr uint32_t LDS = G::LDS + G::NW * RUN_LDS;
  HEAD_TRY((a.d_low ? launch_lds<k_head_dw<T, W, Type<T>::PLANES == 1>>(a.dw_grid, G::NT, LDS, st, a, c0)
                    : launch_lds<k_head_dw<T, W, false>>(a.dw_grid, G::NT, LDS, st, a, c0)));
  if (a.dw_parts) {
    const uint32_t tiles = ((a.h + G::TI - 1) / G::TI) * (((uint32_t)a.v + G::TJ - 1) / G::TJ);
    hipLaunchKernelGGL((k_head_dw_tail<T, W>), dim3(tiles % a.dw_grid * (G::WI * G::WJ)), dim3(G::NT), 0, st, a, c0);
    HEAD_TRY(hipGetLastError());
  }
  return hipSuccess;
}

template <typename T, int J, bool GRAD>
hipError_t chunk_of(HeadArgs& a, uint32_t c0, uint32_t rows, hipStream_t st) {
  using G = Cfg<typename Type<T>::V8, J>;
  const uint32_t nj = (rows + G::TJ - 1) / G::TJ;
  const uint32_t ni = ((uint32_t)a.v + G::TI - 1) / G::TI;
  constexpr uint32_t PIECE = G::WI * 32;
  const uint32_t pieces = ((uint32_t)a.v + PIECE - 1) / PIECE;
  const uint32_t wide = (a.k_logits + PACK_KB - 1) / PACK_KB, of_w = a.wr && c0 == 0 ? a.k_dx * 2 * wide : 0;
  const dim3 pack(of_w + (rows + 31) / 32 * 2 * wide);
  if (alone<T>(a)) {
    if constexpr (Type<T>::PLANES == 1) hipLaunchKernelGGL((k_head_pack<T, true>), pack, dim3(256), 0, st, a, c0, of_w);
  } else {
    hipLaunchKernelGGL((k_head_pack<T, false>), pack, dim3(256), 0, st, a, c0, of_w);
  }
  HEAD_TRY(hipGetLastError());
  if constexpr (!GRAD && Type<T>::PLANES == 1) {
    if (!a.wr) {
      HEAD_TRY((launch_lds<k_head_logits<T, J, false, true>>(grid_of<G>(ni * nj), G::NT, G::LDS, st, a, c0)));
    } else {
      HEAD_TRY((launch_lds<k_head_logits<T, J, false, false>>(grid_of<G>(ni * nj), G::NT, G::LDS, st, a, c0)));
    }
  } else {
    HEAD_TRY((launch_lds<k_head_logits<T, J, GRAD, false>>(grid_of<G>(ni * nj), G::NT, G::LDS, st, a, c0)));
  }
  hipLaunchKernelGGL(k_head_loss, dim3((rows + SR - 1) / SR), dim3(SNT), 0, st, a, c0, pieces);
  HEAD_TRY(hipGetLastError());
  if constexpr (GRAD) {
    const uint32_t high = (rows + 127) / 128, blocks = std::max(1u, std::min(4u, a.k_dx * high / 2048u));
    const auto softmax = a.d_low ? k_head_softmax<T, J, Type<T>::PLANES == 1> : k_head_softmax<T, J, false>;
    hipLaunchKernelGGL(softmax, dim3((a.k_dx + blocks - 1) / blocks, high), dim3(256), 0, st, a, c0, PIECE == 128 ? 7u : 6u, blocks);
    HEAD_TRY(hipGetLastError());
    HEAD_TRY((launch_lds<k_head_dx<T, J>>(a.dx_grid, G::NT, G::LDS, st, a, c0)));
    if (a.n > 0) {
      hipLaunchKernelGGL((k_head_dx_sum<T>), dim3(rows), dim3(256), 0, st, a, c0, G::TI, G::TJ);
      HEAD_TRY(hipGetLastError());
    }
    HEAD_TRY((a.dw_small ? launch_dw<T, 64>(a, c0, st) : launch_dw<T, 256>(a, c0, st)));
  }
  return hipSuccess;
}

template <typename T>
hipError_t head_of(HeadArgs& a, bool grad, hipStream_t st) {
  if (!alone<T>(a)) {
    hipLaunchKernelGGL(k_head_begin, dim3(1 + (Type<T>::PLANES == 2 ? a.top_x + a.top_w : 0)), dim3(BNT), 0, st, a);
    HEAD_TRY(hipGetLastError());
  }
  // (without a token one chunk still writes a dw of zeros)
  for (uint64_t c0 = 0; c0 == 0 || c0 < a.n; c0 += a.chunk) {
    const uint32_t rows = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(a.chunk, a.n - c0));
    // (one choice for every chunk: the buffers go by it)
    const uint32_t tokens = tile_tokens(a.chunk), c = (uint32_t)c0;
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
  a.v_blocks = blocks(a.v);
  a.hq = (a.h + 15) / 16 * 16;
  // per token of a chunk: d, and binary32 numerators apart (16-bit ones are
  // replaced in place)
  const uint64_t per_row = grad ? (uint64_t)a.k_dx * KSTAGE * (planes == 2 ? 8 : 2) : (a.v + 63) / 64 * 8;
  if (a.chunk == 0) a.chunk = std::min<uint64_t>(HEAD_CHUNK_BYTES / per_row, 1u << 22);
  a.chunk = std::min<uint64_t>(std::max<uint64_t>(a.chunk, 128), std::max<uint64_t>(a.n, 1));
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
  // (up to 256 maxima of x and of w: k_head_pack has a thread for each)
  a.top_x = planes == 2 ? (uint32_t)std::min<uint64_t>(128, (a.n + 63) / 64) : 0;
  a.top_w = planes == 2 ? (uint32_t)std::min<uint64_t>(256, (a.v + 63) / 64) : 0;
  a.tops = (uint32_t*)take((a.top_x + a.top_w) * 4);
  a.zt = (float*)take(a.chunk * 4);
  a.stats = (float2*)take((a.v + 63) / 64 * a.chunk * 8);
  // (a tile of 256 rows of the transposed operand: 8 blocks along k)
  const uint64_t kh = (a.k_logits + 7) / 8 * 8, kv = (a.k_dx + 7) / 8 * 8;
  a.wr_plane = a.v_blocks * kh * 1024;
  a.xr_plane = a.c_blocks * kh * 1024;
  a.wr = direct ? nullptr : take(planes * a.wr_plane);
  a.xr = take(planes * a.xr_plane);
  if (grad) {
    a.pr_plane = a.c_blocks * kv * 1024;
    a.d_low = planes == 1 && a.chunk <= LOW_CHUNK;
    a.pr = take((a.d_low ? 2 : planes) * a.pr_plane);
    a.pt = planes == 2 || a.chunk <= 64 ? take(a.pr_plane * 2) : a.pr;
    a.row_info = (float4*)take(a.chunk * 16);
    a.rest = (float*)take(a.chunk * 4);
    // dx: parts of the vocabulary, as many as cost least: rounds of tiles
    // (about half a microsecond a stage) and the parts' sums written and read
    const uint64_t tj = tile_tokens(a.chunk), ti = tj == 256 ? 256 : 128;
    const uint64_t tiles = (a.h + ti - 1) / ti * ((a.chunk + tj - 1) / tj);
    const uint64_t stages = (planes == 2 ? 3 : 1) * (uint64_t)a.k_dx, room = (tj == 256 ? 1 : 2) * (uint64_t)device_cus();
    double best = 0.0;
    a.splits = 0;
    for (uint64_t s = 1; s <= std::max<uint64_t>(1, std::min<uint64_t>(stages / 16, room)); ++s) {
      const double cost = (double)((tiles * s + room - 1) / room) * ((double)stages / (double)s + 8.0) * 0.5e-6 +
                          (double)(s * a.chunk * a.hq) * 8.0 / 5e12;
      if (a.splits == 0 || cost < best) {
        best = cost;
        a.splits = (uint32_t)s;
      }
    }
    a.dx_part = (float*)take(a.splits * a.chunk * a.hq * 4);
    a.dx_grid = (uint32_t)((std::min(room, tiles * std::max<uint64_t>(stages / 16, 1)) + 7) / 8 * 8);
    // dw: 256 x 256 tiles, or 128 x 64 where those would leave two thirds of
    // the compute units idle (4096 tokens, 4000 entries, h 1024, 64 tiles: the
    // step in 189 us, not 220; 61 x 1009 x 97 in binary32: 41.5, not 44.4)
    const uint64_t cus = (uint64_t)(device_cus() + 7) / 8 * 8;
    a.dw_small = (a.h + 255) / 256 * ((a.v + 255) / 256) * 3 <= cus;
    const uint64_t wi = a.dw_small ? 128 : 256, wj = a.dw_small ? 64 : 256, slots = a.dw_small ? 2 * cus : cus;
    const uint64_t wt = (a.h + wi - 1) / wi * ((a.v + wj - 1) / wj), rows = (planes == 2 ? 3 : a.d_low && a.chunk <= LOW_TOKENS ? 2 : 1) * ((a.chunk + KSTAGE - 1) / KSTAGE);
    a.dw_grid = (uint32_t)std::min<uint64_t>(slots, (wt + 7) / 8 * 8);
    a.dw_parts = 0;
    if (wt < slots) {
      // less than a round: in parts of 16 stages at least, where that makes it a
      // third as long (4096 x 1009 x 97 in binary32: the step 178 -> 93 us; two
      // parts gain nothing on the kernel that joins them)
      const uint64_t parts = std::min<uint64_t>(std::min<uint64_t>(slots / wt, rows / 16), 16);
      if (parts >= 3) {
        a.dw_parts = (uint32_t)parts;
        a.dw_grid = (uint32_t)((wt * parts + 7) / 8 * 8);
      }
    } else if (const uint64_t rest = wt % a.dw_grid; rest && a.dw_grid >= 2 * rest) {
      // the tiles past the last whole round in as many parts as fill one
      a.dw_parts = (uint32_t)std::min<uint64_t>(a.dw_grid / rest, 16);
    }
    a.dw_part = (float*)take(wt % a.dw_grid * a.dw_parts * wi * wj * 4);
    a.dw_sum = one ? nullptr : (float*)take(a.v * a.hq * 4);
  }
  return at;
}

hipError_t launch_head(HeadArgs& a, int dt, bool grad, hipStream_t st) {
  return dt == DT_F32 ? head_of<float>(a, grad, st) : dt == DT_BF16 ? head_of<bf16_t>(a, grad, st) : head_of<f16_t>(a, grad, st);
}

TC_DEFINE_ERROR_READER(errors_head)

}  // namespace tc
