// tc_gemm.hpp -- the matrix product inside the vocabulary loss: a tile of
// D[i][j] = sum_k A[i][k] B[j][k], k contiguous in both operands, accumulated
// in binary32 by the matrix units.
//
// A workgroup owns a tile of TI x TJ and walks k in stages of 32 elements (64
// bytes of every row).  A stage's rows go from memory straight into one of NS
// LDS slots, 16 bytes per lane, NS - 1 stages ahead; its fragments are read
// into registers while the matrix units work on the stage before.  One
// barrier per stage: behind it the slot of the previous stage is free.
//
// Binary32 operands come as two binary16 planes, high and low (x = high + low
// to 22 bits after a scaling by a power of two): the k loop runs three times,
// over high high, high low and low high.
#pragma once

#include "tc_device.hpp"

namespace tc {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma(half8 a, half8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(bhalf8 a, bhalf8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

constexpr uint32_t KSTAGE = 32;                 // elements of k per stage
constexpr uint32_t ROW_BYTES = KSTAGE * 2;      // of one row in an LDS slot

// One operand: row r's first element at p + r * ld bytes (16-byte aligned);
// rows past the last one read the last one (their results are dropped).
struct GemmOperand {
  const char* p;
  uint64_t ld;           // bytes from row to row, below 2^24
  uint32_t rows;         // >= 1
  const uint32_t* map;   // or nullptr: row r is row map[r] of the memory, which then ends below 4 GiB
  uint64_t plane;        // bytes from the high to the low plane (binary32)
};

template <typename V8, int WI_, int WJ_, int NWI_, int NWJ_, int NS_>
struct Gemm {
  static constexpr int WI = WI_, WJ = WJ_, NWI = NWI_, NWJ = NWJ_, NS = NS_;
  static constexpr uint32_t TI = 32 * WI * NWI, TJ = 32 * WJ * NWJ, NW = NWI * NWJ, NT = 64 * NW;
  static constexpr uint32_t LA = TI / 16 / NW, LB = TJ / 16 / NW;   // loads of a wavefront per stage (16 rows each)
  static constexpr uint32_t SLOT = (TI + TJ) * ROW_BYTES, LDS = NS * SLOT;
  static_assert(LA * 16 * NW == TI && LB * 16 * NW == TJ, "whole loads");
  static_assert(NS >= 3 && LDS <= 160 * 1024, "slots");

  // 16-byte piece c of row r lies at piece c ^ turn(r): the 16 rows that a
  // quarter of a wavefront reads at one piece then lie in 16 different places
  static __device__ __forceinline__ uint32_t turn(uint32_t r) { return ((r >> 2) + 2u * (r >> 4)) & 3u; }
  // The row of A that a lane feeds in: with it the accumulators of a lane hold
  // 16 consecutive i (acc[fi][fj][r] is i = 32 fi + 16 (lane / 32) + r of the
  // wavefront's rows, j = 32 fj + lane % 32).
  static __device__ __forceinline__ uint32_t a_row(uint32_t a) { return ((a >> 2) & 1u) * 16u + (a >> 3) * 4u + (a & 3u); }

  // stages [s0, s0 + count) of the walk over the plane pairs, `per` stages each
  static __device__ __forceinline__ void run(const GemmOperand& A, uint32_t i0, const GemmOperand& B, uint32_t j0,
                                             uint32_t per, uint32_t s0, uint32_t count, char* lds, f32x16 (&acc)[WI][WJ]) {
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int x = 0; x < WI; ++x)
#pragma unroll
      for (int y = 0; y < WJ; ++y) acc[x][y] = f32x16{};
    if (count == 0) return;

    const char* const a0 = A.map ? A.p : A.p + (uint64_t)i0 * A.ld;
    const char* const b0 = B.map ? B.p : B.p + (uint64_t)j0 * B.ld;
    uint32_t offa[LA], offb[LB];
#pragma unroll
    for (uint32_t t = 0; t < LA; ++t) {
      const uint32_t r = (wave * LA + t) * 16u + (lane >> 2), piece = (lane & 3u) ^ turn(r);
      const uint32_t row = min(i0 + r, A.rows - 1u);
      offa[t] = (A.map ? A.map[row] : row - i0) * (uint32_t)A.ld + piece * 16u;
    }
#pragma unroll
    for (uint32_t t = 0; t < LB; ++t) {
      const uint32_t r = (wave * LB + t) * 16u + (lane >> 2), piece = (lane & 3u) ^ turn(r);
      const uint32_t row = min(j0 + r, B.rows - 1u);
      offb[t] = (B.map ? B.map[row] : row - j0) * (uint32_t)B.ld + piece * 16u;
    }

    // the next stage to load: past the last one it is loaded again, into a
    // slot that nobody reads, so that every stage has the same loads out
    uint32_t next = s0, pair = s0 / per, k = s0 - pair * per;
    const uint32_t end = s0 + count;
    auto load = [&](uint32_t slot) {
      const char* ga = a0 + (pair == 2 ? A.plane : 0) + (uint64_t)k * ROW_BYTES;
      const char* gb = b0 + (pair == 1 ? B.plane : 0) + (uint64_t)k * ROW_BYTES;
      char* la = lds + slot * SLOT + wave * LA * 1024u;
      char* lb = lds + slot * SLOT + TI * ROW_BYTES + wave * LB * 1024u;
#pragma unroll
      for (uint32_t t = 0; t < LA; ++t)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(ga + offa[t]),
                                         (__attribute__((address_space(3))) void*)(la + t * 1024u), 16, 0, 0);
#pragma unroll
      for (uint32_t t = 0; t < LB; ++t)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(gb + offb[t]),
                                         (__attribute__((address_space(3))) void*)(lb + t * 1024u), 16, 0, 0);
      if (next + 1 < end) {
        ++next;
        if (++k == per) { k = 0; ++pair; }
      }
    };

    const uint32_t wi = wave % NWI, wj = wave / NWI, l = lane & 31u, h = lane >> 5;
    uint32_t ra[2], rb[2];     // this lane's piece of k step 0 and 1 in the first fragment
    {
      const uint32_t ar = a_row(l);
#pragma unroll
      for (uint32_t q = 0; q < 2; ++q) {
        ra[q] = (wi * WI * 32u + ar) * ROW_BYTES + (((2u * q + h) ^ turn(ar)) * 16u);
        rb[q] = TI * ROW_BYTES + (wj * WJ * 32u + l) * ROW_BYTES + (((2u * q + h) ^ turn(l)) * 16u);
      }
    }
    // (32 rows on, turn() is the same)
    struct Frags { V8 a[2][WI], b[2][WJ]; } f0, f1;
    auto read = [&](uint32_t slot, Frags& f) {
      const char* s = lds + slot * SLOT;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int x = 0; x < WI; ++x) f.a[q][x] = *reinterpret_cast<const V8*>(s + ra[q] + x * 32 * ROW_BYTES);
#pragma unroll
        for (int y = 0; y < WJ; ++y) f.b[q][y] = *reinterpret_cast<const V8*>(s + rb[q] + y * 32 * ROW_BYTES);
      }
    };
    auto multiply = [&](const Frags& f) {
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int x = 0; x < WI; ++x)
#pragma unroll
          for (int y = 0; y < WJ; ++y) acc[x][y] = mfma(f.a[q][x], f.b[q][y], acc[x][y]);
    };

    constexpr uint32_t PER_STAGE = LA + LB;
#pragma unroll
    for (uint32_t s = 0; s < NS - 1; ++s) load(s);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 2) * PER_STAGE) : "memory");
    read(0, f0);
    uint32_t fill = NS - 1, from = 1;       // slots of the stage to load and to read
    auto step = [&](const Frags& now, Frags& then) {
      // the stage to read has landed for every wavefront, and every wavefront
      // has the stage before the present one in registers or behind it
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 3) * PER_STAGE) : "memory");
      load(fill);
      read(from, then);
      multiply(now);
      fill = fill + 1 == NS ? 0 : fill + 1;
      from = from + 1 == NS ? 0 : from + 1;
    };
    for (uint32_t s = 0; s < count; s += 2) {
      step(f0, f1);
      if (s + 1 < count) step(f1, f0);
    }
    // loads that nobody reads must not land in what the caller puts there
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
};

// Workgroups go round the 8 dies in turn; tiles that share operands should
// share a die's cache: die d takes the d-th run of consecutive tiles.
__device__ __forceinline__ uint32_t die_tile(uint32_t block, uint32_t blocks) { return (block & 7u) * (blocks >> 3) + (block >> 3); }

}  // namespace tc
