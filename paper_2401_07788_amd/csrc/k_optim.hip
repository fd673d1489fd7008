// k_optim.hip -- what every pipeline stage does with its gradients once the
// backward pass is over: their global norm, and one AdamW step over a list of
// tensors with moments in binary32 or in 8 bits.
//
//   g' = c g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p  = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Both are one pass over the data and bound by HBM: an element of the norm
// reads 2 or 4 bytes, one of the step moves 28 (binary32 throughout), 22
// (16-bit p and g, binary32 moments) or 10 (16-bit p and g, 8-bit moments).
// A list goes out in launches of as many tensors as fit the kernel arguments,
// so that a call uploads no table and keeps none.
//
// 8-bit moments.  256 consecutive positions of a tensor share a power of two
// 2^E just above their largest magnitude.  m: sign, 4 exponent bits and 3
// mantissa bits; v: 5 exponent bits and 3 mantissa bits.  A step changes v by
// a thousandth, and m by a tenth of what it is off, where codes are an eighth
// apart: rounding to nearest would never move v and stop m at two thirds of a
// steady gradient, so both are rounded up or down at random with the distance
// as the chance, and their averages are right.  E leaves room above the
// largest magnitude for its rounding up.  A v that is not zero never becomes
// zero (it would make a step of m / eps).  With exponents of two, scaling is
// exact and a code is bits of the binary32 pattern: a shift and a power of two
// read it, an add and a shift write it.
#include "tc_internal.hpp"
#include "tc_device.hpp"

namespace tc {

namespace {

constexpr int ONT = 256;               // threads of a workgroup
constexpr int OV = 8;                  // consecutive elements of a thread
constexpr uint32_t UNIT = ONT * OV;    // elements a workgroup takes at once: 8 blocks of 256 positions

// tensors are often views into one buffer: the hardware takes a vector access
// at any element's address, so that alignment needs no second path
template <int BYTES, int ALIGN>
struct __attribute__((packed, aligned(ALIGN))) Raw { uint32_t w[BYTES / 4]; };

template <typename R, int N>
__device__ __forceinline__ void get(const void* base, uint64_t i, R (&out)[N]) {
  using V = Raw<N * (int)sizeof(R), (int)sizeof(R) < 4 ? (int)sizeof(R) : 4>;
  const V v = *reinterpret_cast<const V*>(static_cast<const R*>(base) + i);
  __builtin_memcpy(out, &v, sizeof(v));
}
template <typename R, int N>
__device__ __forceinline__ void put(void* base, uint64_t i, const R (&in)[N]) {
  using V = Raw<N * (int)sizeof(R), (int)sizeof(R) < 4 ? (int)sizeof(R) : 4>;
  V v;
  __builtin_memcpy(&v, in, sizeof(v));
  *reinterpret_cast<V*>(static_cast<R*>(base) + i) = v;
}

// `left` of OV elements exist (left <= 0: none); the others read as zero.
// FULL: all of them do, for every lane.
template <typename T, bool FULL>
__device__ __forceinline__ void load_up(const void* base, uint64_t i, int64_t left, float (&out)[OV]) {
  using R = typename Elem<T>::raw;
  R r[OV];
  if (FULL || left >= OV) {
    get<R, OV>(base, i, r);
#pragma unroll
    for (int k = 0; k < OV; ++k) out[k] = Elem<T>::up(r[k]);
  } else {
#pragma unroll
    for (int k = 0; k < OV; ++k) out[k] = k < left ? Elem<T>::up(static_cast<const R*>(base)[i + k]) : 0.0f;
  }
}
// (a NaN's pattern equals itself)
__device__ __forceinline__ uint32_t pattern(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t pattern(uint16_t v) { return v; }

// Parameters with masters in binary32: the masters, but where a parameter is
// not the rounding of its master it was set since the last step (a checkpoint
// copied into it, say) and counts instead.  Reading the parameters for this
// takes 2 of 30 bytes an element, or of 18 (161 M elements in bfloat16: 879 us
// become 944, with 8-bit moments 513 become 575).
template <typename P, bool FULL>
__device__ __forceinline__ void load_masters(const void* w32, const void* p, uint64_t i, int64_t left, float (&out)[OV]) {
  using R = typename Elem<P>::raw;
  load_up<float, FULL>(w32, i, left, out);
  R r[OV] = {};
  if (FULL || left >= OV) {
    get<R, OV>(p, i, r);
  } else {
#pragma unroll
    for (int k = 0; k < OV; ++k)
      if (k < left) r[k] = static_cast<const R*>(p)[i + k];
  }
#pragma unroll
  for (int k = 0; k < OV; ++k) {
    if (pattern(Elem<P>::down(out[k])) != pattern(r[k])) out[k] = Elem<P>::up(r[k]);
  }
}
template <typename T, bool FULL>
__device__ __forceinline__ void store_down(void* base, uint64_t i, int64_t left, const float (&in)[OV]) {
  using R = typename Elem<T>::raw;
  R r[OV];
#pragma unroll
  for (int k = 0; k < OV; ++k) r[k] = Elem<T>::down(in[k]);
  if (FULL || left >= OV) {
    put<R, OV>(base, i, r);
  } else {
#pragma unroll
    for (int k = 0; k < OV; ++k)
      if (k < left) static_cast<R*>(base)[i + k] = r[k];
  }
}

// the tensor that chunk c lies in: the last whose first chunk is not after it
template <typename A>
__device__ __forceinline__ uint32_t find_tensor(const A& a, uint32_t c) {
  uint32_t lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// ------------------------------------------------------------ 8-bit moments
__device__ __forceinline__ float code_up(uint32_t u, int e) { return __builtin_ldexpf(__uint_as_float(u << 20), e); }

// the code bits of a magnitude below 2^(E + 1), with 20 random bits under the last one kept
__device__ __forceinline__ uint32_t code_of(float x, int e, uint32_t noise, uint32_t most) {
  const uint32_t u = (__float_as_uint(__builtin_ldexpf(__builtin_fabsf(x), e)) + noise) >> 20;
  return u < most ? u : most;    // (only an infinite moment reaches past the largest)
}
__device__ __forceinline__ uint32_t encode_m(float m, int e, uint32_t noise) {
  return code_of(m, -112 - e, noise, 127u) | ((__float_as_uint(m) >> 24) & 0x80u);
}
__device__ __forceinline__ uint32_t encode_v(float v, int e, uint32_t noise) {
  const uint32_t u = code_of(v, -96 - e, noise, 255u);
  return v > 0.0f && u == 0 ? 1u : u;
}
// E from the pattern of a block's largest magnitude: the exponent after
// rounding up to 3 mantissa bits (an infinite one: the largest there is)
__device__ __forceinline__ int block_exponent(uint32_t top) {
  const int e = (int)((top + 0xFFFFFu) >> 23) - 127;
  return e < 127 ? e : 127;
}
// 32 random bits for the pair of positions j: two rounds of multiply and fold
// (odd constants from the golden ratio and from e)
__device__ __forceinline__ uint32_t pair_hash(uint32_t j, uint32_t seed) {
  uint32_t h = (j ^ seed) * 0x9E3779B9u;
  h = (h ^ (h >> 15)) * 0xB7E15163u;
  return h ^ (h >> 16);
}

// largest value of the 32 lanes of a half wavefront, in all of them (patterns
// of magnitudes, so that unsigned order is the order of the values)
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
  return x > y ? x : y;
}
__device__ __forceinline__ uint32_t half_wave_max(uint32_t x) {
  x = dpp_max<0xB1>(x);    // lanes 1, 0, 3, 2
  x = dpp_max<0x4E>(x);    // lanes 2, 3, 0, 1
  x = dpp_max<0x141>(x);   // mirrored in 8
  x = dpp_max<0x140>(x);   // mirrored in 16
  const uint32_t y = (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401F);   // lane ^ 16
  return x > y ? x : y;
}

}  // namespace

// ------------------------------------------------------------------- AdamW
// p after the step.  Next to 28 or 22 bytes an element the exact division and
// square root cost nothing; next to 10 they would be the bound, and the
// hardware's (each within an ulp, of a step that is far smaller than p) are
// used.  Those take a v below 2^-126 for 0, which eps covers.
template <bool EIGHT>
__device__ __forceinline__ float adamw_p(const AdamwArgs& a, float p, float m, float v) {
  if constexpr (EIGHT)
    return p * a.decay - m * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v * a.r2) + a.eps) * a.rate;
  else
    return p * a.decay - m / (__builtin_sqrtf(v * a.r2) + a.eps) * a.rate;
}

// OV elements of one tensor per lane
template <typename P, typename G, bool EIGHT, bool FULL>
__device__ __forceinline__ void adamw_unit(const AdamwArgs& a, const ListEntry& t, float c, uint64_t i, int64_t left) {
  float g[OV], p[OV], m[OV], v[OV];
  const uint64_t pos = t.pos + i, blk = pos >> 8;
  load_up<G, FULL>(t.g, i, left, g);
  if (t.w32) load_masters<P, FULL>(t.w32, t.p, i, left, p);
  else load_up<P, FULL>(t.p, i, left, p);
  if constexpr (EIGHT) {
    // the codes of a tensor's last block exist in full
    uint8_t cm[OV] = {}, cv[OV] = {};
    int em = 0, ev = 0;
    if (FULL || left > 0) {
      __builtin_memcpy(cm, static_cast<const uint8_t*>(a.m) + pos, OV);
      __builtin_memcpy(cv, static_cast<const uint8_t*>(a.v) + pos, OV);
      em = 112 + a.em[blk];
      ev = 96 + a.ev[blk];
    }
#pragma unroll
    for (int k = 0; k < OV; ++k) {
      const float x = code_up(cm[k] & 127u, em);
      m[k] = __uint_as_float(__float_as_uint(x) | ((uint32_t)(cm[k] & 128u) << 24));
      v[k] = code_up(cv[k], ev);
    }
  } else {
    load_up<float, FULL>(a.m, pos, left, m);
    load_up<float, FULL>(a.v, pos, left, v);
  }
  uint32_t tm = 0, tv = 0;
#pragma unroll
  for (int k = 0; k < OV; ++k) {
    const float gc = g[k] * c;
    m[k] = m[k] * a.b1 + gc * a.a1;
    v[k] = v[k] * a.b2 + gc * gc * a.a2;
    p[k] = adamw_p<EIGHT>(a, p[k], m[k], v[k]);
    if (EIGHT) {
      // (positions past the tensor's end hold zeros)
      if (!FULL && k >= left) m[k] = v[k] = 0.0f;
      const uint32_t bm = __float_as_uint(m[k]) & 0x7FFFFFFFu, bv = __float_as_uint(v[k]);
      tm = tm > bm ? tm : bm;
      tv = tv > bv ? tv : bv;
    }
  }
  if (t.w32) store_down<float, FULL>(t.w32, i, left, p);
  store_down<P, FULL>(t.p, i, left, p);
  if constexpr (EIGHT) {
    const int em = block_exponent(half_wave_max(tm)), ev = block_exponent(half_wave_max(tv));
    uint8_t cm[OV], cv[OV];
#pragma unroll
    for (int k = 0; k < OV; k += 2) {
      // 16 bits of the pair's hash for v, the others for m
      const uint32_t h = pair_hash((uint32_t)(pos >> 1) + k / 2, a.seed);
      const uint32_t low = ((h & 0xFFFFu) << 4) | 8u, high = ((h >> 12) & 0xFFFF0u) | 8u;
      cm[k] = (uint8_t)encode_m(m[k], em, high);
      cv[k] = (uint8_t)encode_v(v[k], ev, low);
      cm[k + 1] = (uint8_t)encode_m(m[k + 1], em, low);
      cv[k + 1] = (uint8_t)encode_v(v[k + 1], ev, high);
    }
    if (FULL || left > 0) {
      __builtin_memcpy(static_cast<uint8_t*>(a.m) + pos, cm, OV);
      __builtin_memcpy(static_cast<uint8_t*>(a.v) + pos, cv, OV);
      if ((threadIdx.x & 31u) == 0) {
        a.em[blk] = (int8_t)em;
        a.ev[blk] = (int8_t)ev;
      }
    }
  } else {
    store_down<float, FULL>(a.m, pos, left, m);
    store_down<float, FULL>(a.v, pos, left, v);
  }
}

template <typename P, typename G, bool EIGHT>
__global__ __launch_bounds__(ONT) void k_adamw(const AdamwArgs a) {
  float c = 1.0f;
  if (a.clip) {
    // a norm that is not finite: this step is left out, for every tensor
    if (!(__builtin_fabsf(a.clip[0]) < __builtin_inff())) return;
    c = a.clip[1];
  }
  const uint32_t k = find_tensor(a, blockIdx.x);
  const ListEntry t = a.t[k];
  const uint64_t first = (uint64_t)(blockIdx.x - a.first[k]) * a.chunk;
  uint64_t i = first + threadIdx.x * OV;
  if (first + a.chunk <= t.n) {
    for (uint32_t done = 0; done < a.chunk; done += UNIT, i += UNIT) adamw_unit<P, G, EIGHT, true>(a, t, c, i, OV);
  } else {
    // (wavefronts leave whole: the block exponents need all lanes)
    for (uint32_t done = 0; done < a.chunk && __ballot(i < t.n) != 0; done += UNIT, i += UNIT)
      adamw_unit<P, G, EIGHT, false>(a, t, c, i, (int64_t)(t.n - i));
  }
}

template <typename P>
static void* adamw_fn(int g_dt, int bits) {
  if (bits == 8)
    return g_dt == DT_F32 ? (void*)k_adamw<P, float, true> : g_dt == DT_BF16 ? (void*)k_adamw<P, bf16_t, true>
                                                                             : (void*)k_adamw<P, f16_t, true>;
  return g_dt == DT_F32 ? (void*)k_adamw<P, float, false> : g_dt == DT_BF16 ? (void*)k_adamw<P, bf16_t, false>
                                                                            : (void*)k_adamw<P, f16_t, false>;
}

hipError_t launch_adamw(int p_dt, int g_dt, int bits, AdamwArgs& a, const ListEntry* list, uint64_t n_list, hipStream_t st) {
  uint64_t total = 0;
  for (uint64_t k = 0; k < n_list; ++k) total += list[k].n;
  // few elements: as many workgroups as there are units; many: longer chunks,
  // so that a workgroup's start and search are a small part of it
  a.chunk = total > (uint64_t)UNIT * 4096u ? 4 * UNIT : UNIT;
  void* fn = p_dt == DT_F32 ? adamw_fn<float>(g_dt, bits) : p_dt == DT_BF16 ? adamw_fn<bf16_t>(g_dt, bits)
                                                                            : adamw_fn<f16_t>(g_dt, bits);
  for (uint64_t k = 0; k < n_list;) {
    a.n = 0;
    uint64_t chunks = 0;
    for (; k < n_list && a.n < ADAMW_LIST; ++k) {
      if (list[k].n == 0) continue;
      const uint64_t c = (list[k].n + a.chunk - 1) / a.chunk;
      if (chunks + c > 0x7FFFFFFFu) break;
      a.t[a.n] = list[k];
      a.first[a.n++] = (uint32_t)chunks;
      chunks += c;
    }
    if (a.n == 0) break;
    void* args[] = {&a};
    const hipError_t e = hipLaunchKernel(fn, dim3((uint32_t)chunks), dim3(ONT), args, 0, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------- 8-bit moments as their values
// a wavefront takes a block at a time: 4 codes a lane, so that its stores of
// 16 bytes a lane are 1 KB in a row
constexpr uint32_t MB = 4;     // blocks of a wavefront

__global__ __launch_bounds__(ONT) void k_moments(const MomentsArgs a) {
  const uint64_t first = ((uint64_t)blockIdx.x * (ONT / WAVE) + (threadIdx.x >> 6)) * MB;
  const uint32_t at = (threadIdx.x & 63u) * 4u;
  uint32_t cm[MB], cv[MB];
  int em[MB], ev[MB];
#pragma unroll
  for (uint32_t b = 0; b < MB; ++b) {
    const uint64_t blk = first + b;
    if (blk >= a.n >> 8) break;
    __builtin_memcpy(&cm[b], a.m + (blk << 8) + at, 4);
    __builtin_memcpy(&cv[b], a.v + (blk << 8) + at, 4);
    em[b] = 112 + a.em[blk];
    ev[b] = 96 + a.ev[blk];
  }
#pragma unroll
  for (uint32_t b = 0; b < MB; ++b) {
    const uint64_t blk = first + b;
    if (blk >= a.n >> 8) break;
    float m[4], v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t x = cm[b] >> (8 * k);
      m[k] = __uint_as_float(__float_as_uint(code_up(x & 127u, em[b])) | (x & 128u) << 24);
      v[k] = code_up((cv[b] >> (8 * k)) & 255u, ev[b]);
    }
    put<float, 4>(a.m_out, (blk << 8) + at, m);
    put<float, 4>(a.v_out, (blk << 8) + at, v);
  }
}

hipError_t launch_moments(const MomentsArgs& a, hipStream_t st) {
  const uint64_t per = (uint64_t)(ONT / WAVE) * MB * 256u;
  for (uint64_t at = 0; at < a.n;) {
    const uint64_t n = a.n - at < per << 30 ? a.n - at : per << 30;
    const MomentsArgs part = {a.m + at, a.v + at, a.em + (at >> 8), a.ev + (at >> 8), a.m_out + at, a.v_out + at, n};
    hipLaunchKernelGGL(k_moments, dim3((uint32_t)((n + per - 1) / per)), dim3(ONT), 0, st, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    at += n;
  }
  return hipSuccess;
}

// -------------------------------------------------------------------- norm
// Squares are summed in binary64: gradients of 1e20 and of 1e-25 square out of
// binary32's range, and the sum costs no time next to the loads.  Every
// workgroup leaves one partial sum; the last one to finish adds them in their
// order, so that the result does not depend on which one that is.
__device__ __forceinline__ double block_sum(double s) {
  __shared__ double part[ONT / WAVE];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  double r = 0;
#pragma unroll
  for (int k = 0; k < ONT / WAVE; ++k) r += part[k];
  __syncthreads();
  return r;
}

template <typename G>
__global__ __launch_bounds__(ONT) void k_grad_norm(const NormArgs a) {
  double s = 0;
  for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const uint32_t t = find_tensor(a, c);
    const uint64_t n = a.t[t].n, i0 = (uint64_t)(c - a.first[t]) * a.chunk;
    const uint64_t i = i0 + threadIdx.x * OV;
    if (i0 + a.chunk <= n) {
      // (whole units: the loads of four go out together)
#pragma unroll 4
      for (uint32_t done = 0; done < a.chunk; done += UNIT) {
        float g[OV];
        load_up<G, true>(a.t[t].g, i + done, OV, g);
#pragma unroll
        for (int k = 0; k < OV; ++k) s += (double)g[k] * (double)g[k];
      }
    } else {
      for (uint32_t done = 0; done < a.chunk; done += UNIT) {
        float g[OV];
        load_up<G, false>(a.t[t].g, i + done, (int64_t)(n - i - done), g);
#pragma unroll
        for (int k = 0; k < OV; ++k) s += (double)g[k] * (double)g[k];
      }
    }
  }
  s = block_sum(s);
  __shared__ uint32_t last;
  if (threadIdx.x == 0) {
    __hip_atomic_store(&a.part[a.slot + blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __builtin_amdgcn_s_waitcnt(0);
    last = a.slots != 0 &&
           __hip_atomic_fetch_add(a.count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  double r = 0;
  for (uint32_t k = threadIdx.x; k < a.slots; k += ONT) {
    r += __hip_atomic_load(&a.part[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a.part[k] = 0.0;
  }
  r = block_sum(r);
  if (threadIdx.x == 0) {
    const float norm = (float)__builtin_sqrt(r);
    a.out[0] = norm;
    const float f = a.max_norm / (norm + 1e-6f);
    a.out[1] = f > 1.0f ? 1.0f : f;
    __hip_atomic_store(a.count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

uint64_t grad_norm_ws_bytes(uint64_t n_list) {
  const uint64_t launches = n_list / NORM_LIST + 1;
  return 64 + launches * NORM_GRID * sizeof(double);
}

hipError_t launch_grad_norm(int g_dt, const ListEntry* list, uint64_t n_list, float max_norm, float* out, void* ws,
                            hipStream_t st) {
  NormArgs a{};
  a.count = (uint32_t*)ws;
  a.part = (double*)((char*)ws + 64);
  a.out = out;
  a.max_norm = max_norm;
  uint64_t total = 0;
  for (uint64_t k = 0; k < n_list; ++k) total += list[k].n;
  a.chunk = total > (uint64_t)UNIT * 4 * NORM_GRID ? 4 * UNIT : UNIT;
  void* const fn = g_dt == DT_F32 ? (void*)k_grad_norm<float> : g_dt == DT_BF16 ? (void*)k_grad_norm<bf16_t>
                                                                          : (void*)k_grad_norm<f16_t>;
  uint64_t k = 0;
  do {
    a.n = 0;
    uint64_t chunks = 0;
    for (; k < n_list && a.n < NORM_LIST; ++k) {
      if (list[k].n == 0) continue;
      const uint64_t c = (list[k].n + a.chunk - 1) / a.chunk;
      if (chunks + c > 0x7FFFFFFFu) break;
      a.t[a.n] = {list[k].g, list[k].n};
      a.first[a.n++] = (uint32_t)chunks;
      chunks += c;
    }
    a.chunks = (uint32_t)chunks;
    const uint32_t grid = chunks == 0 ? 1u : chunks < NORM_GRID ? (uint32_t)chunks : NORM_GRID;
    // the last launch adds every launch's partial sums
    while (k < n_list && list[k].n == 0) ++k;
    a.slots = k == n_list ? a.slot + grid : 0;
    void* args[] = {&a};
    const hipError_t e = hipLaunchKernel(fn, dim3(grid), dim3(ONT), args, 0, st);
    if (e != hipSuccess) return e;
    a.slot += grid;
  } while (k < n_list);
  return hipSuccess;
}

}  // namespace tc
