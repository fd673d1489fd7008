// tc_internal.hpp -- launch plans and launcher entry points shared by the
// C-ABI layer (tc_api.cpp) and the kernel translation units.  Not installed.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tc {

enum Dt : int { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };

inline size_t dt_size(int dt) { return dt == DT_F32 ? 4u : 2u; }

// How one segmented kernel is laid out on the device: NT threads per
// workgroup, VPT consecutive elements per thread, P workgroups per segment
// (a "group"), n_groups groups resident at once (grid = n_groups * P), each
// looping over segments group, group + n_groups, ...
struct SegPlan {
  int nt = 0;
  int vpt = 0;
  uint32_t P = 1;
  uint32_t n_groups = 0;
  uint32_t grid = 0;
  uint64_t capacity = 0;   // workgroups of this kernel the device holds at once
  uint64_t ws_words = 0;   // 32-bit words of zero-initialised workspace needed
  uint64_t ws_used = 0;    // of which this launch touches (its n_groups groups)
  bool lds = false;        // TopK: one workgroup per segment held in LDS (k_topk_lds)
};

// ------------------------------------------------------------------- TopK
enum SelKind : int { SEL_PLAIN = 0, SEL_EF = 1, SEL_AQSGD = 2, SEL_EFMIX = 3 };

struct TopkArgs {
  const void* x;         // PLAIN/EF: [n_seg][L] input; AQSGD: activations [n_seg][L]
  float* e;              // EF: [n_seg][L] residual (in-out)
  void* m;               // AQSGD: buffer [n_samples][L] (in-out)
  const int64_t* ids;    // AQSGD: [n_seg] sample ids (device)
  uint64_t n_samples;
  uint32_t* idx;         // [n_seg][k]
  void* val;             // [n_seg][k] in the input dtype
  uint32_t* blk;         // optional [n_seg][nblk + 1] block table
  uint64_t n_seg, L, k;
  uint32_t P;
  uint32_t* ws;
  // EFMIX: the error buffer's list (idx, val, blk above hold the input's)
  uint32_t* idx2;        // [n_seg][k2]
  void* val2;            // [n_seg][k2] in the input dtype
  uint32_t* blk2;        // optional block table of that list
  uint64_t k2;
};

constexpr uint64_t BLOCK_LEN = 4096;   // TC_BLOCK_LEN
__host__ __device__ constexpr uint64_t n_blocks(uint64_t L) { return (L + BLOCK_LEN - 1) / BLOCK_LEN; }

SegPlan plan_topk(int sel, int dt, uint64_t n_seg, uint64_t L);
// the LDS engine (one workgroup per segment of at most LDS_SEG_MAX elements)
// for any such length; EF-mixed always takes it
constexpr uint64_t LDS_SEG_MAX = 32768;
SegPlan plan_lds(int sel, int dt, uint64_t n_seg);
hipError_t launch_topk(int sel, int dt, const SegPlan& plan, const TopkArgs& a, hipStream_t st);

// ----------------------------------------------------------- quantization
struct QuantArgs {
  const void* x;         // [n_grp][G]
  float* e;              // EF residual [n_grp][G] or nullptr
  uint32_t* codes;       // [n_grp][wpg] words
  float* meta;           // [n_grp][2]
  uint64_t n_grp, G, wpg;
  uint32_t P;
  uint32_t* ws;
};

SegPlan plan_quant(int dt, uint32_t bits, bool ef, uint64_t n_grp, uint64_t G);
hipError_t launch_quant(int dt, int out_dt, uint32_t bits, bool ef, const SegPlan& plan,
                        const QuantArgs& a, hipStream_t st);

struct UnpackArgs {
  const uint32_t* codes;
  const float* meta;
  void* y;
  uint64_t n_grp, G, wpg;
};
hipError_t launch_unpack(int out_dt, uint32_t bits, const UnpackArgs& a, hipStream_t st);

// --------------------------------------------------------- receiver side
struct ScatterArgs {
  const uint32_t* idx;   // [n_seg][k]
  const uint32_t* blk;   // optional [n_seg][nblk + 1] block table
  const void* val;       // [n_seg][k] wire values (TopK)
  const uint32_t* codes; // TopK+quant: [n_seg][wpg] codes of the kept list
  const float* meta;     // TopK+quant: [n_seg][2]
  void* y;               // dense output [n_seg][L]
  void* m;               // AQ-SGD receiver buffer [n_samples][L]
  const int64_t* ids;
  uint64_t n_samples;
  uint64_t n_seg, L, k, wpg;
  // EF-mixed: the error buffer's list, added after the input's
  const uint32_t* idx2;  // [n_seg][k2]
  const uint32_t* blk2;  // optional block table of that list
  const void* val2;      // [n_seg][k2] wire values
  uint64_t k2;
};
hipError_t launch_topk_decompress(int wire, int out_dt, const ScatterArgs& a, hipStream_t st);
hipError_t launch_efmix_recv(int wire, int out_dt, const ScatterArgs& a, hipStream_t st);

// EF-mixed residual after both selections (the sender's second kernel)
struct EfmixResidArgs {
  const void* x;         // [n_seg][L] input
  float* e;              // [n_seg][L] residual (in-out)
  const uint32_t* idx;   // the input's list [n_seg][k]
  const uint32_t* blk;   // its block table or nullptr
  const uint32_t* idx2;  // the buffer's list [n_seg][k2]
  const uint32_t* blk2;  // its block table or nullptr
  uint64_t n_seg, L, k, k2;
};
hipError_t launch_efmix_resid(int dt, const EfmixResidArgs& a, hipStream_t st);

// TopK at given indices (another tensor's TopK payload), optionally inside
// error feedback
struct GatherArgs {
  const uint32_t* idx;   // [n_seg][k], ascending per segment
  const uint32_t* blk;   // optional block table of that payload
  const void* x;         // [n_seg][L]
  float* e;              // EF residual [n_seg][L] (in-out) or nullptr
  void* val;             // [n_seg][k] in x's dtype
  uint64_t n_seg, L, k;
};
hipError_t launch_gather(int dt, const GatherArgs& a, hipStream_t st);
hipError_t launch_aqsgd_recv(int dt, const ScatterArgs& a, hipStream_t st);

// ------------------------------------------------ segments too long to hold
// TopK over one segment with a chain of kernels (a sampled band, candidate
// or whole-segment radix passes, per-tile counts and their offsets, an emit
// pass that writes each tile's kept entries at its offset, the kept-list
// quantizer)
struct GlobalArgs {
  const void* x;         // [L] input
  float* e;              // [L] residual (in-out) or nullptr
  uint32_t* idx;         // [k]
  void* val;             // [k] wire values (plain TopK) or nullptr
  uint32_t* codes;       // quantized kept list: [wpg] words
  float* meta;           // quantized kept list: [2]
  uint32_t* blk;         // optional [n_blocks(L) + 1]
  uint64_t L, k, wpg, n_tiles;
  uint32_t* state;       // workspace pieces (global_ws_carve)
  uint32_t* hist;
  uint32_t* tiles;       // 4 words per tile
  uint32_t* wgs;         // tile-count workgroup totals / prefixes
  uint32_t* cand;        // candidate sub-lists: binary32 bits of the values in the band
  uint64_t cand_cap;     // all sub-lists together
  uint32_t bits;         // quantized kept list: b (0: values)
  uint32_t sample_stride;
  uint32_t n_sub;        // candidate sub-lists (<= 8, <= the chain's grid)
  uint32_t tpw;          // tiles per tile-count workgroup
};
uint64_t global_ws_words(uint64_t L);
void global_ws_carve(uint32_t* ws, uint64_t L, GlobalArgs& a);
hipError_t launch_global(int dt, bool ef, uint32_t qbits, const GlobalArgs& a, hipStream_t st);

// ------------------------------------- loss over a vocabulary (k_head.hip)
struct HeadArgs {
  // the call
  const void* x;         // [n][h], rows ldx elements apart
  const void* w;         // [v][h], rows ldw elements apart
  const int64_t* target; // [n]
  const float* weight;   // [n] or nullptr (1)
  float* loss;           // [n]
  float* lse;            // [n]
  void* dx;              // [n][h]
  void* dw;              // [v][h]
  uint64_t n, v, ldx, ldw;
  uint32_t h;
  int64_t ignore;
  uint64_t chunk;        // tokens whose softmax is held at once (0: head_plan chooses)
  // head_plan
  uint64_t hq;           // h rounded up to 16
  uint32_t k_logits, k_dx;                      // stages of 32 along h and along v
  uint32_t splits, dx_grid;                     // parts of dx's sum; workgroups of its product
  uint32_t top_x, top_w;                        // maxima of x and of w in `tops` (binary32)
  uint32_t v_blocks, c_blocks;                  // row blocks of 16, up to whole tiles
  uint64_t wr_plane, xr_plane, pr_plane;        // bytes
  char* info;
  uint32_t* rows;        // [n] tokens that have a target, then the others
  uint32_t* tops;
  float* zt;             // [chunk] logit of the target
  float4* row_info;      // [chunk] largest logit, weight over the sum, target, d at the target (gradients only)
  float* rest;           // [chunk] what rounding took from d's entry at the target
  float2* stats;         // [pieces][chunk] maximum and sum of a piece of the vocabulary
  // in blocks (tc_gemm.hpp), rows by elements of a row
  char *wr, *xr;         // v by h (nullptr: the call's own w), tokens by h
  char* pr;              // d: tokens by v
  char* pt;              // numerators, tokens by v (16-bit types: pr)
  float* dx_part;        // [splits][chunk][hq]
  float* dw_sum;         // [v][hq], or nullptr with one chunk
  uint32_t dw_grid, dw_parts;   // workgroups of dw's product; parts of its last round's tiles
  bool d_low;                   // d has a second plane of 16 bits (16-bit types)
  bool dw_small;                // 128 x 64 tiles, not 256 x 256
  float* dw_part;        // [dw_parts][tiles of the last round][a tile]
};
// bytes that the per-token buffers of a chunk may take unless the caller chooses
constexpr uint64_t HEAD_CHUNK_BYTES = 4ull << 30;
uint64_t head_plan(HeadArgs& a, int dt, bool grad, char* base);
hipError_t launch_head(HeadArgs& a, int dt, bool grad, hipStream_t st);

// ------------------------------------------- lists of tensors (k_optim.hip)
struct ListEntry {
  void* p;               // parameters
  const void* g;         // gradients
  float* w32;            // binary32 parameters that p is the rounding of, or nullptr
  uint64_t n;            // elements
  uint64_t pos;          // first position in the moments
};
// as many tensors as keep a launch's arguments under 4 KB
constexpr uint32_t ADAMW_LIST = 88, NORM_LIST = 192;
struct AdamwArgs {
  ListEntry t[ADAMW_LIST];
  uint32_t first[ADAMW_LIST];   // each tensor's first chunk
  void* m;               // binary32 values or codes
  void* v;
  int8_t* em;            // 8 bits: exponents, one per 256 positions
  int8_t* ev;
  const float* clip;     // (norm, factor) or nullptr
  uint32_t n, chunk;     // tensors; elements of a workgroup
  float b1, a1, b2, a2;  // beta and 1 - beta
  float decay;           // 1 - lr wd
  float r2, eps, rate;   // 1 / (1 - beta2^t), eps, lr / (1 - beta1^t)
  uint32_t seed;
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");
hipError_t launch_adamw(int p_dt, int g_dt, int bits, AdamwArgs& a, const ListEntry* list, uint64_t n_list, hipStream_t st);

struct MomentsArgs {
  const uint8_t* m;
  const uint8_t* v;
  const int8_t* em;
  const int8_t* ev;
  float* m_out;
  float* v_out;
  uint64_t n;            // positions, a multiple of 256
};
hipError_t launch_moments(const MomentsArgs& a, hipStream_t st);

constexpr uint32_t NORM_GRID = 2048;   // workgroups of a launch, each with one partial sum
struct NormArgs {
  struct { const void* g; uint64_t n; } t[NORM_LIST];
  uint32_t first[NORM_LIST];
  double* part;          // partial sums of every launch
  uint32_t* count;       // workgroups of the last launch that are done
  float* out;            // (norm, factor)
  uint32_t n, chunk, chunks;
  uint32_t slot, slots;  // this launch's first partial sum; all of them (0: not the last launch)
  float max_norm;
};
static_assert(sizeof(NormArgs) <= 4096, "kernel arguments");
uint64_t grad_norm_ws_bytes(uint64_t n_list);
hipError_t launch_grad_norm(int g_dt, const ListEntry* list, uint64_t n_list, float max_norm, float* out, void* ws,
                            hipStream_t st);

// ------------------------------------ preconditions (debug library only)
// Bits the check kernels of k_check.hip report; each call synchronizes the
// stream and returns the bits found (and clears them).
enum : uint32_t { CHK_NONFINITE = 1u, CHK_RANGE = 2u };
hipError_t check_values(int dt, const void* x, const float* e, uint64_t n, hipStream_t st, uint32_t* flags);
hipError_t check_aqsgd(int dt, const void* a, const void* m, const int64_t* ids, uint64_t n_ids, uint64_t L,
                       uint64_t n_samples, hipStream_t st, uint32_t* flags);

// sticky kernel error bits of each kernel translation unit
hipError_t errors_topk(uint32_t* bits, bool clear);
hipError_t errors_quant(uint32_t* bits, bool clear);
hipError_t errors_scatter(uint32_t* bits, bool clear);
hipError_t errors_global(uint32_t* bits, bool clear);
hipError_t errors_head(uint32_t* bits, bool clear);
// the same words set from the host (tests of the recovery path)
hipError_t errors_topk_raise(uint32_t bits);
hipError_t errors_quant_raise(uint32_t bits);
hipError_t errors_scatter_raise(uint32_t bits);
hipError_t errors_global_raise(uint32_t bits);
hipError_t errors_head_raise(uint32_t bits);

// device properties (cached per device)
int device_cus();
// workgroups of kernel fn (always launched with nt threads) one compute unit
// holds, 0 when the runtime does not say; asked once per kernel
int resident_per_cu(const void* fn, int nt);

// ---- library-owned scratch of the allocation-free entry point (k_scratch.hip)
constexpr uint64_t NOALLOC_SCRATCH_BYTES = 4ull << 20;    // TC_NOALLOC_SCRATCH_BYTES
hipError_t noalloc_scratch(void** ptr, hipStream_t st);
hipError_t noalloc_scratch_reset();

}  // namespace tc
