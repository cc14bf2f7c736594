// Internal declarations of the operators of xshare_ops.h.
#pragma once

#include <atomic>

#include "xs_internal.cuh"
#include "xshare_ops.h"

namespace xs {

constexpr int kMaxSlots = 32;        // routed slots per token of the float8 experts
constexpr int kPermChunk = 1024;     // pairs per CTA of the permutation kernels
constexpr int kF8PairTile = 256;     // token rows of a tile on CTA pairs
constexpr int kF8FewTile = 64;       // and at most in the form for few rows
constexpr int kF8Ctas = 152;         // CTAs of a float8 product at most (one per SM)
constexpr int kF8CutBlocks = 8;      // K blocks per CTA that sharing units has to save: joining costs about 5 us
constexpr uint64_t kF8WaitNs = 1000000000ull;   // 1 s per wait inside a product
constexpr int kF8Regs = 168;         // registers per thread of the product kernels at their launch
constexpr float kTinyAmax = 7.8886090522101181e-31f;   // 2^-100
constexpr float kE4m3Max = 448.f;
constexpr uint8_t kE4m3Nan = 0x7f;

// Facts of one permutation, read by the kernels after it.
struct PermMeta {
  int32_t n_pairs, n_tiles, n_used, status;
};

// Groups (token, slot) pairs by expert, ascending pair ids inside one
// (permute.cu).  Up to kPermChunk pairs one CTA does it all and pos holds final
// rows; above that pos holds ranks inside the pair's chunk of kPermChunk, to which
// first[chunk][expert] is to be added (perm_row()).
struct PermArgs {
  const int32_t *ids;    // [P]; outside 0 .. N - 1: not routed
  int P, N, tile_tok;
  int32_t *pos;          // [P]
  int32_t *cnt;          // [chunks][N] pairs per chunk, for more than one chunk
  int32_t *first;        // [chunks][N], for more than one chunk
  Tile *tiles;           // nullable
  PermMeta *meta;
  xs_stats *stats;       // nullable
  int32_t *counts_out, *offsets_out, *perm_out;   // nullable
  int32_t *zero;         // nullable: words cleared for the kernels after
  int zero_n;
};
inline int perm_chunks(int P) { return (P + kPermChunk - 1) / kPermChunk; }
cudaError_t launch_permute(const PermArgs &a, cudaStream_t s);
// Tiles of the grouped product: rows [offsets[e], offsets[e + 1]) of matrix e.
cudaError_t launch_offset_tiles(const int32_t *offsets, int E, int M, int tile_tok, Tile *tiles,
                                PermMeta *meta, xs_stats *stats, int32_t *zero, int zero_n, cudaStream_t s);
// Clears zero_n words and, if given, the statistics.
cudaError_t launch_zero(int32_t *zero, int zero_n, xs_stats *stats, cudaStream_t s);

struct GateArgs {
  const void *logits;
  const float *bias;
  const uint8_t *expert_mask, *token_mask;
  int B, N, k;
  xs_gate_params prm;
  int32_t *ids;
  float *w, *scores;
};
cudaError_t launch_gate(const GateArgs &a, int dtype, cudaStream_t s);

cudaError_t launch_quant_rows(const void *x, int dtype, int M, int K, uint8_t *q, float *scales,
                              cudaStream_t s);
cudaError_t launch_quant_blocks(const void *x, int dtype, int n, int R, int K, uint8_t *q, float *scales,
                                int n_sms, cudaStream_t s);
// Quantises every token's row and places it at the rows of its pairs.
struct TokenArgs {
  const uint16_t *x;     // [B, d] bf16
  const int32_t *ids;    // [B, k]
  const int32_t *pos;    // [B, k]
  const int32_t *first;  // [chunks][N]
  int32_t *rows;         // [B, k] out: the pairs' rows, -1 where there is none
  uint8_t *q;            // [rows, d]
  float *scales;         // [rows, d / 128]
  int B, k, d, N;
};
cudaError_t launch_quant_tokens(const TokenArgs &a, cudaStream_t s);
// The same with the permutation of up to kPermChunk pairs in the same kernel (p: ids, P, N,
// tile_tok, tiles, meta, stats, zero; a's pos and first are not used).
cudaError_t launch_quant_routed(const TokenArgs &a, const PermArgs &p, cudaStream_t s);
// y_t = sum over slots of w_ts out[row of pair (t, s)], bf16.
struct CombineArgs {
  const void *out;       // [rows, d] fp32, or with inv fp16
  const float *inv;      // nullable, [rows, d / 64]: the rows are out * inv
  const int32_t *rows;   // [B, k]
  const float *w;        // [B, k]
  uint16_t *y;           // [B, d] bf16
  int B, k, d;
};
cudaError_t launch_combine_f8(const CombineArgs &a, cudaStream_t s);

// One product on the tensor cores.
struct F8Args {
  const uint8_t *a;            // [rows, K] tokens
  const float *sa;             // [rows, ceil(K / 128)]
  const uint8_t *b0, *b1;      // [E, N, K] weights; b1: up (SwiGLU form), else nullptr
  const float *sb0, *sb1;      // [E, ceil(N / 128), ceil(K / 128)]
  int rows, N, K, E;
  const Tile *tiles;           // nullable: one matrix for all rows
  PermMeta *meta;              // with tiles: their number
  int max_tiles;
  int tile_tok;                // rows of a tile: kF8PairTile, or 64 or 32 in the form for few rows
  int split;                   // tiles of 32 rows: CTAs of a cluster that share a unit's K blocks (1: see gemm_f8_few.cu)
  bool early;                  // weights and tiles were complete before the launch before this one
  void *y;                     // [rows, N] of y_dtype
  int y_dtype;
  float *inv;                  // nullable, pairs only: y is fp16, [rows, N / 64] factors (N % 128 == 0)
  uint8_t *hq;                 // SwiGLU form: [rows, N] and scales [rows, N / 128]
  float *hs;
  xs_stats *stats;             // nullable
  int n_sms;
  float *part;                 // few rows: f8_part_bytes(), partial sums of cut units
  int32_t *cnt;                // and [kF8Ctas] arrivals, zero at the start
  uint64_t wait_ns;            // limit of the MMA issuers' waits for operands (the others': kF8WaitNs)
  uint32_t hold;               // self-test: in CTA 0 the barrier of stage hold - 1 waits for an arrival that never comes; 0: none
};
// The product kernels are launched with 168 registers for each of their 384 threads and hand
// them out again by warpgroup.  A split that asks for more than the launch holds would wait for
// ever, so a build that gave a kernel another number is refused (`seen`: this kernel's is right).
inline cudaError_t check_registers(const void *kernel, std::atomic<bool> *seen) {
  if (seen->load(std::memory_order_relaxed)) return cudaSuccess;
  cudaFuncAttributes at;
  const cudaError_t e = cudaFuncGetAttributes(&at, kernel);
  if (e != cudaSuccess) return e;
  if (at.numRegs != kF8Regs) return cudaErrorInvalidKernelImage;
  seen->store(true, std::memory_order_relaxed);
  return cudaSuccess;
}
// Rows of the box that loads a matrix's last N % 128 weight rows (128: a whole block's).
inline int edge_rows(int N) {
  const int n = N % 128;
  return n == 0 || n > 64 ? 128 : n > 32 ? 64 : n > 16 ? 32 : 16;
}
size_t f8_part_bytes();
// F8Args::split for a product of at most `units` units (gemm_f8_few.cu).
int f8_split(int tile_tok, long long units, int K);
cudaError_t launch_f8_pairs(const F8Args &a, cudaStream_t s);   // gemm_f8.cu
cudaError_t launch_f8_few(const F8Args &a, cudaStream_t s);     // gemm_f8_few.cu
// Sets wait_ns, and hold for the launch that xshare_selftest_f8_hold() has named (selftest.cu).
void f8_waits(F8Args *a);
inline cudaError_t launch_f8(F8Args a, cudaStream_t s) {
  f8_waits(&a);
  return a.tile_tok == kF8PairTile ? launch_f8_pairs(a, s) : launch_f8_few(a, s);
}

}  // namespace xs
