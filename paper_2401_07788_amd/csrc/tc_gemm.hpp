// tc_gemm.hpp -- the matrix product inside the vocabulary loss: tiles of
// D[i][j] = sum_k A[i][k] B[j][k], accumulated in binary32 by the matrix units.
//
// A workgroup owns a tile of TI x TJ and walks k in stages of 32 elements (64
// bytes of every row).  A stage goes from memory straight into one of NS LDS
// slots, 16 bytes per lane, NS - 1 stages ahead; its fragments are read into
// registers while the matrix units work on the stage before.  One barrier per
// stage: behind it the slot of the previous stage is free.
//
// What it measured (131072 x 8192 x 4096 in bfloat16, 256 x 256 tiles of 8
// wavefronts): 1097 TFLOP/s with 16-row pieces read from rows in memory, 1238
// from 1 KB blocks (half as many requests to the L2), 1358 once a stage's
// scalar work was down to a few adds, 1374 with the tiles as one stream of
// stages.  On zeros it reaches 1830: on real data the card's power is the
// next bound.
//
// Binary32 operands come as two binary16 planes, high and low (x = high + low
// to 22 bits after a scaling by a power of two): the walk goes three times
// along k, over high high, high low and low high.
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

// 16-byte piece c (of 4) of row r lies at place c ^ turn(r) of the row: the 16
// rows that a quarter of a wavefront reads at one piece then lie in 16
// different places of the banks.
__device__ __forceinline__ uint32_t turn(uint32_t r) { return (r >> 2) & 3u; }

// An operand that lies in memory as the LDS wants it: blocks of 16 rows by 32
// elements, 1 KB each, pieces turned; a k stage's blocks one after the other.
// Every load is then 1 KB in a row, from a scalar address.
struct Blocks {
  const char* p;
  uint32_t rows;         // row blocks, a multiple of 16: a tile never reaches past them
  uint64_t plane;        // bytes from the high to the low plane (binary32)
};
// The same memory seen from the other side: what its blocks call k are the
// operand's rows, and the sum runs along its rows (two row blocks to a
// stage).  The LDS gives such an operand to the matrix units by its
// transposing reads, so that no transposed copy is made of anything.
struct BlocksT {
  const char* p;
  uint32_t rows;         // row blocks of the memory
  uint64_t plane;
};
// An operand as the caller has it: row r's first element at p + r * ld bytes
// (16-byte aligned).  A load takes 64 bytes of 16 rows.
struct Rows {
  const char* p;
  uint64_t ld;           // bytes from row to row, below 2^24
  uint32_t rows;         // >= 1; rows past the last one read the last one (their results are dropped)
};

// 16 bytes per lane from memory to 1 KB of the LDS; AT goes to either address
template <int AT>
__device__ __forceinline__ void load16(const char* g, char* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g, (__attribute__((address_space(3))) void*)to, 16, AT, 0);
}

// A transposing read.  Nothing else writes *p while this function runs, and
// saying so spares it a wait for every load to the LDS that is under way (the
// stages' own waits order them).
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
__device__ __forceinline__ short4v read_tr(__attribute__((address_space(3))) short4v* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
}

// A wavefront's L loads of one operand per stage, and the walk along k.  What
// a stage needs in scalar instructions is counted: they are issued in order
// with the products, and 45 of them a stage cost a third of the kernel's time.
template <typename O, uint32_t L> struct Loader;
template <uint32_t L> struct Loader<Blocks, L> {
  const char* at;
  uint64_t stage, plane;
  uint32_t lane16;
  __device__ __forceinline__ Loader(const Blocks& o, uint32_t row0, uint32_t wave, uint32_t k) {
    stage = (uint64_t)o.rows * 1024u;
    plane = o.plane;
    lane16 = (threadIdx.x & 63u) * 16u;
    at = o.p + (uint64_t)((row0 >> 4) + wave * L) * 1024u + k * stage;
  }
  __device__ __forceinline__ void go(uint32_t t, char* to) {
    // (as a scalar base and a 32-bit offset)
    asm volatile("" : "+v"(lane16));
    const char* g = at + lane16;
    static_assert(L <= 4, "offsets");
    if (t == 0) load16<0>(g, to);
    else if (t == 1) load16<1024>(g, to);
    else if (t == 2) load16<2048>(g, to);
    else load16<3072>(g, to);
  }
  __device__ __forceinline__ void next() { at += stage; }
  __device__ __forceinline__ void stay() { at -= stage; stage = 0; }
  // from the end of one walk over k to the start of another, in the same plane (0) or the other (+1, -1)
  __device__ __forceinline__ void again(uint32_t per, int to) { at += (int64_t)plane * to - (int64_t)(stage * per); }
};
template <uint32_t L> struct Loader<BlocksT, L> {
  const char* at;
  uint64_t plane;
  uint32_t pitch, lane16, stage = 2048;
  __device__ __forceinline__ Loader(const BlocksT& o, uint32_t row0, uint32_t wave, uint32_t k) {
    // load b of the stage is block (b & 1) along the sum, 32 rows from row0 + 32 (b >> 1) on
    const uint32_t b = wave * L;
    pitch = o.rows * 1024u;
    plane = o.plane;
    lane16 = (threadIdx.x & 63u) * 16u;
    at = o.p + (uint64_t)((row0 >> 5) + (b >> 1)) * pitch + (2u * k + (b & 1u)) * 1024u;
  }
  __device__ __forceinline__ void go(uint32_t t, char* to) {
    asm volatile("" : "+v"(lane16));
    const char* g = at + (t >= 2 ? pitch : 0u) + lane16;
    static_assert(L == 1 || L == 2 || L == 4, "pairs of blocks");
    if (t & 1) load16<1024>(g, to + (t & 2) * 1024u);
    else load16<0>(g, to + (t & 2) * 1024u);
  }
  __device__ __forceinline__ void next() { at += stage; }
  __device__ __forceinline__ void stay() { at -= stage; stage = 0; }
  __device__ __forceinline__ void again(uint32_t per, int to) { at += (int64_t)plane * to - (int64_t)(2048u * per); }
};
template <uint32_t L> struct Loader<Rows, L> {
  const char* at;
  uint32_t off[L], stage = ROW_BYTES;
  __device__ __forceinline__ Loader(const Rows& o, uint32_t row0, uint32_t wave, uint32_t k) {
    const uint32_t lane = threadIdx.x & 63u;
    at = o.p + (uint64_t)row0 * o.ld + (uint64_t)k * ROW_BYTES;
#pragma unroll
    for (uint32_t t = 0; t < L; ++t) {
      const uint32_t r = (wave * L + t) * 16u + (lane >> 2), row = min(row0 + r, o.rows - 1u);
      off[t] = (row - row0) * (uint32_t)o.ld + ((lane & 3u) ^ turn(r)) * 16u;
    }
  }
  __device__ __forceinline__ void go(uint32_t t, char* to) {
    asm volatile("" : "+v"(off[t]));
    load16<0>(at + off[t], to + t * 1024u);
  }
  __device__ __forceinline__ void next() { at += stage; }
  __device__ __forceinline__ void stay() { at -= stage; stage = 0; }
  __device__ __forceinline__ void again(uint32_t, int) {}
};

template <typename V8, int WI_, int WJ_, int NWI_, int NWJ_, int NS_>
struct Gemm {
  static constexpr int WI = WI_, WJ = WJ_, NWI = NWI_, NWJ = NWJ_, NS = NS_;
  static constexpr uint32_t TI = 32 * WI * NWI, TJ = 32 * WJ * NWJ, NW = NWI * NWJ, NT = 64 * NW;
  static constexpr uint32_t LA = TI / 16 / NW, LB = TJ / 16 / NW;   // loads of a wavefront per stage (16 rows each)
  static constexpr uint32_t SLOT = (TI + TJ) * ROW_BYTES, LDS = NS * SLOT;
  static_assert(LA * 16 * NW == TI && LB * 16 * NW == TJ, "whole loads");
  static_assert(NS >= 3 && LDS <= 160 * 1024, "slots");

  // A wavefront's fragments of one operand: get(stage's operand, k step of 16,
  // fragment).  A lane feeds in 8 consecutive k of one row.  IS_A: of row
  // a_row(lane), with which the accumulators of a lane hold 16 consecutive i
  // (acc[fi][fj][r] is i = 32 fi + 16 (lane / 32) + r of the wavefront's rows,
  // j = 32 fj + lane % 32).
  static __device__ __forceinline__ uint32_t a_row(uint32_t a) { return ((a >> 2) & 1u) * 16u + (a >> 3) * 4u + (a & 3u); }
  template <typename O, bool IS_A> struct Reader {
    static constexpr int READS = 1;
    uint32_t at[2];
    __device__ __forceinline__ Reader(uint32_t first) {
      const uint32_t l = threadIdx.x & 31u, h = (threadIdx.x >> 5) & 1u, r = IS_A ? a_row(l) : l;
      // (32 rows on, turn() is the same)
#pragma unroll
      for (uint32_t q = 0; q < 2; ++q) at[q] = (first * 32u + r) * ROW_BYTES + ((2u * q + h) ^ turn(r)) * 16u;
    }
    __device__ __forceinline__ V8 get(const char* s, uint32_t q, uint32_t x) const {
      return *reinterpret_cast<const V8*>(s + at[q] + x * 32u * ROW_BYTES);
    }
  };
  // Transposing reads: 16 lanes put in 4 rows (of the sum) of 4 pieces of 4
  // elements, lane l of them gets element l of every row.
  template <bool IS_A> struct Reader<BlocksT, IS_A> {
    static constexpr int READS = 2;
    uint32_t at[2];
    __device__ __forceinline__ Reader(uint32_t first) {
      const uint32_t lane = threadIdx.x & 63u, a = lane >> 2 & 7u;      // a: which 4 of the fragment's 32 rows
      const uint32_t group = (a & 4u) | (lane & 3u), n = IS_A ? a_row(group * 4u) : group * 4u;
#pragma unroll
      for (uint32_t p = 0; p < 2; ++p) {
        const uint32_t k = (lane >> 5) * 8u + p * 4u + ((lane >> 2) & 3u);
        at[p] = first * 2048u + k * ROW_BYTES + ((n >> 3) ^ turn(k)) * 16u + (n & 7u) * 2u;
      }
    }
    __device__ __forceinline__ V8 get(const char* s, uint32_t q, uint32_t x) const {
      using P = __attribute__((address_space(3))) short4v*;
      const short4v lo = read_tr((P)(s + at[0] + x * 2048u + q * 1024u)), hi = read_tr((P)(s + at[1] + x * 2048u + q * 1024u));
      return __builtin_bit_cast(V8, (short8v)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };

  // A piece of work: stages [s0, s0 + count) of the tile at (i0, j0), count > 0.
  // The walk along k goes over the pairs of planes (up to PAIRS of high high,
  // high low, low high), `per` stages each.
  struct Work {
    uint32_t i0, j0, s0, count;
  };

  // The workgroup's pieces one after the other: work(n, w) gives the n-th or
  // returns false, done(n, w, acc) takes its sums.  The stages of all of them
  // are one stream: while the last ones of a piece are multiplied, the first
  // ones of the next are loaded, and they land while done() runs (which
  // therefore has the LDS past the slots only).
  template <int PAIRS, typename OA, typename OB, typename WorkOf, typename Done>
  static __device__ __forceinline__ void stream(const OA& A, const OB& B, uint32_t per, char* lds, WorkOf work, Done done) {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Work in;                                             // of the loads
    uint32_t n_in = 0;
    if (!work(0u, in)) return;
    Work out = in;                                       // of the products
    uint32_t pair, left, rest;         // stages to load until the next turn, and of the piece after that
    Loader<OA, LA> ga(A, 0, wave, 0);
    Loader<OB, LB> gb(B, 0, wave, 0);
    auto begin = [&] {
      pair = PAIRS > 1 ? in.s0 / per : 0;
      const uint32_t k = in.s0 - pair * per;
      left = PAIRS > 1 ? min(in.count, per - k) : in.count;
      rest = in.count - left;
      ga = Loader<OA, LA>(A, in.i0, wave, k);
      gb = Loader<OB, LB>(B, in.j0, wave, k);
      if constexpr (PAIRS > 1) {
        if (pair == 2) ga.again(0, 1);
        if (pair == 1) gb.again(0, 1);
      }
    };
    begin();
    // where the walk turns: to the next pair of planes, the next piece, or,
    // after the very last stage, to that stage again and again (into slots
    // that nobody reads, so that every stage has the same loads out)
    auto turn_over = [&] {
      if (PAIRS > 1 && rest > 0) {
        left = min(rest, per);
        rest -= left;
        ++pair;
        ga.again(per, pair == 2 ? 1 : 0);
        gb.again(per, pair == 1 ? 1 : -1);
      } else if (work(++n_in, in)) {
        begin();
      } else {
        --n_in;
        left = ~0u;
        ga.stay();
        gb.stay();
      }
    };
    char* const la = lds + wave * LA * 1024u;
    char* const lb = lds + TI * ROW_BYTES + wave * LB * 1024u;
    auto load = [&](uint32_t slot, uint32_t t) {
      if (t < LA) ga.go(t, la + slot);
      else gb.go(t - LA, lb + slot);
    };

    const uint32_t wi = wave % NWI, wj = wave / NWI;
    const Reader<OA, true> qa(wi * WI);
    const Reader<OB, false> qb(wj * WJ);
    struct Frags { V8 a[2][WI], b[2][WJ]; } f0, f1;
    constexpr uint32_t READS = 2 * (WI + WJ), LOADS = LA + LB, PRODUCTS = 2 * WI * WJ;
    auto read = [&](const char* s, Frags& f, uint32_t n) {
      const uint32_t q = n / (WI + WJ), x = n % (WI + WJ);
      if (x < WI) f.a[q][x] = qa.get(s, q, x);
      else f.b[q][x - WI] = qb.get(s + TI * ROW_BYTES, q, x - WI);
    };

#pragma unroll
    for (uint32_t s = 0; s < NS - 1; ++s) {
#pragma unroll
      for (uint32_t t = 0; t < LOADS; ++t) load(s * SLOT, t);
      ga.next();
      gb.next();
      if (--left == 0) turn_over();
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 2) * LOADS) : "memory");
#pragma unroll
    for (uint32_t n = 0; n < READS; ++n) read(lds, f0, n);
    uint32_t to = (NS - 1) * SLOT, from = SLOT;       // slots of the stage to load and to read
    f32x16 acc[WI][WJ];
    auto step = [&](const Frags& now, Frags& then) {
      // the stage to read has landed for every wavefront, and every wavefront
      // has the stage before the present one in registers or behind it
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 3) * LOADS) : "memory");
      __builtin_amdgcn_sched_barrier(0);
      const char* s = lds + from;
      // a read beside every product until all are out, and the loads spread
      // over the stage: a wavefront issues in order, and what it issues at once
      // holds up the products behind it
#pragma unroll
      for (uint32_t m = 0; m < PRODUCTS; ++m) {
        const uint32_t q = m / (WI * WJ), x = m / WJ % WI, y = m % WJ;
        acc[x][y] = mfma(now.a[q][x], now.b[q][y], acc[x][y]);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (m < READS) {
          read(s, then, m);
          if (m % (WI + WJ) < WI) __builtin_amdgcn_sched_group_barrier(0x100, Reader<OA, true>::READS, 0);
          else __builtin_amdgcn_sched_group_barrier(0x100, Reader<OB, false>::READS, 0);
        }
#pragma unroll
        for (uint32_t t = m * LOADS / PRODUCTS; t < (m + 1) * LOADS / PRODUCTS; ++t) {
          load(to, t);
          __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
      }
#pragma unroll
      for (uint32_t n = PRODUCTS; n < READS; ++n) read(s, then, n);
      ga.next();
      gb.next();
      to = to == (NS - 1) * SLOT ? 0 : to + SLOT;
      from = from == (NS - 1) * SLOT ? 0 : from + SLOT;
      __builtin_amdgcn_sched_barrier(0);
    };
    for (uint32_t n_out = 0;;) {
#pragma unroll
      for (int x = 0; x < WI; ++x)
#pragma unroll
        for (int y = 0; y < WJ; ++y) acc[x][y] = f32x16{};
      for (uint32_t s = 0; s < out.count;) {
        // (no stage asks whether the walk turns there)
        const uint32_t run = min(out.count - s, left);
        for (uint32_t r = 0; r < run; r += 2) {
          step(f0, f1);
          if (r + 1 < run) step(f1, f0);
        }
        if (run & 1) f0 = f1;
        s += run;
        left -= run;
        if (left == 0) turn_over();
      }
      done(n_out, out, acc);
      if (!work(++n_out, out)) break;
      // the next piece's first stage again: held across done(), its fragments
      // would take the registers that done() needs
      const char* s = lds + (from == 0 ? (NS - 1) * SLOT : from - SLOT);
#pragma unroll
      for (uint32_t n = 0; n < READS; ++n) read(s, f0, n);
    }
    // the last loads land before the LDS is given up
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  }
};

// Workgroups go round the 8 dies in turn; tiles that share operands should
// share a die's cache: of `blocks` tiles, a multiple of 8, die d takes the
// d-th run of consecutive ones.
__device__ __forceinline__ uint32_t die_tile(uint32_t block, uint32_t blocks) { return (block & 7u) * (blocks >> 3) + (block >> 3); }

}  // namespace tc
