// Products of block-scaled float8 operands on the tensor cores (tcgen05
// kind::f8f6f4), dense or grouped by expert:
//
//   y[m, n] = sum_j sa[m, j] sb[n / 128, j] (sum_{k in block j} a[m, k] b[n, k])
//
// and the SwiGLU form, which takes two weight matrices and writes quantised
// activations: h = silu(g) u, hs = amax / 448 per row and 128 columns.
//
// The scales change every 128 elements of K, so the accumulator cannot stay in TMEM
// over K as it does for bf16: a block's products (MMAs of K = 32) go to one of two TMEM
// buffers, and the epilogue warps add them, scaled, to fp32 sums in their registers
// while the tensor cores fill the other.  The tokens are the MMA's M rows (one per TMEM
// lane), the weights its N columns: a thread then owns one token, whose scale is one
// register, and its columns' weight scales are two values, so a product costs half a
// (packed) multiply-add.
//
// Unit: (tile of token rows of one matrix, 256 weight rows in two blocks of 128: of one
// matrix, or SwiGLU: gate and up of the same hidden units).  Each of two epilogue
// warpgroups takes 64 columns of either block and has TMEM buffers of its own: a buffer
// of 128 columns is full after a quarter of the time in which both buffers of both
// are filled once, which leaves three quarters for its hand-over and its reading (half, with one
// buffer for both warpgroups).
//
// This form, for many rows per matrix, works on CTA pairs (cta_group::2) and tiles of
// 256 rows: each SM loads half of the weights of a unit, 62 bytes of operands per cycle
// at full rate instead of the 94 of a CTA of its own.  gemm_f8_few.cu has the form for few.
//
// Roles (three warpgroups): in the first, warp 0 loads by TMA and warp 1 issues the
// pair's MMAs (in rank 0); the other two are the epilogue (a warp per TMEM lane
// quarter), whose 128 sums per thread take the registers that the first gives up.
// Every wait is bounded in time.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "f8_num.cuh"
#include "f8_ptx.cuh"
#include "ops_internal.cuh"
#include "tc_ptx.cuh"
#include "tmap.cuh"

namespace xs {
namespace {

using namespace ptx;

constexpr int kEpiWarps = 8;
constexpr int kThreads = 128 + 32 * kEpiWarps;
constexpr int kBK = 128;                         // e4m3 per K block: one swizzle row, one scale
constexpr int kCols = 256;                       // weight rows of a unit, TMEM columns of a buffer
constexpr int kRows = 128;                       // token rows of one CTA
constexpr int kABytes = kRows * kBK;             // 16 KB of tokens
constexpr int kBoxes = 4;                        // token boxes of 16, 32, 64, 128 rows

constexpr int kBBytes = kCols / 2 * kBK;          // this CTA's weights of a K block: 16 KB
constexpr int kStageBytes = kABytes + kBBytes;
// Registers per thread of the first and the other two warpgroups.
constexpr int kIssueRegs = 104, kEpiRegs = 200;
static_assert(kIssueRegs + 2 * kEpiRegs <= 3 * kF8Regs, "the launch holds what the warpgroups ask for");
// kOut: bytes per epilogue warp for its rows on their way out.
template <int kOut>
struct Shape {
  static constexpr int kStages = kOut > 0 ? 5 : 6;
  static constexpr int kOutOffset = kStages * kStageBytes;
  static constexpr int kBarOffset = kOutOffset + kEpiWarps * kOut;
  static constexpr int kAmaxOffset = kBarOffset + 256;    // [2 turns][2 warpgroups][128] floats
  static constexpr int kSmemBytes = kAmaxOffset + 2048 + 1024;   // + alignment slack
};

struct F8Params {
  CUtensorMap tmA[kBoxes];
  CUtensorMap tmY;         // 16-bit rows: y, boxes of 32 rows x 64
  CUtensorMap tmB[3];      // weights [E N, K], boxes of 128 rows; [1]: up; [2]: of `edge` rows
  const float *sa, *sb0, *sb1;
  const Tile *tiles;
  PermMeta *meta;
  xs_stats *stats;
  void *y;
  float *inv;              // 16-bit rows: factor of every row and 64 columns
  uint8_t *hq;
  float *hs;
  int rows, N, KB, NB;     // NB: scale rows of a matrix, ceil(N / 128)
  int edge;                // box rows of a matrix's last 128-row block, if that is not whole
  int early;
  uint32_t hold;
  uint64_t wait_ns;
};

__device__ __forceinline__ void convert(float v, float *o) { *o = v; }
__device__ __forceinline__ void convert(float v, __nv_bfloat16 *o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void convert(float v, __half *o) { *o = __float2half_rn(v); }

// 64 columns of a row (v[kFrom ..]), of which the first n exist; rows are whole 32-byte words
// and aligned.
template <int kFrom, class T>
__device__ __forceinline__ void store_row(T *dst, const uint64_t (&v)[64], int n) {
  constexpr int kPer = 32 / sizeof(T);
#pragma unroll
  for (int c = 0; c < 64; c += kPer) {
    if (c >= n) break;
    T o[kPer];
#pragma unroll
    for (int j = 0; j < kPer; j += 2) {
      const float2 f = unpack2(v[kFrom + (c + j) / 2]);
      convert(f.x, &o[j]);
      convert(f.y, &o[j + 1]);
    }
    uint32_t w[8];
    memcpy(w, o, 32);
    store32(dst + c, w);
  }
}

// The same of a warp's first `rows` rows for any N, through shared memory, so that a store's
// lanes write neighbouring columns: by itself a thread would touch a line of its own with each
// element (2551 x 323 x 32, bf16: 38 -> 8 us).  Rows in `stage` are 33 words apart.
constexpr int kOddOut = 32 * 33 * 4;
template <int kFrom, class T>
__device__ __forceinline__ void store_rows_odd(uint32_t *stage, T *dst, int N, const uint64_t (&v)[64], int rows, int n) {
  const int lane = threadIdx.x & 31;
  constexpr int kPass = sizeof(T) == 4 ? 2 : 1;   // 32 words of a row at a time
#pragma unroll
  for (int h = 0; h < kPass; ++h) {
    __syncwarp();   // the words before these have been read
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      if constexpr (kPass == 2) {
        const float2 f = unpack2(v[kFrom + h * 16 + c / 2]);
        stage[lane * 33 + c] = __float_as_uint(c % 2 == 0 ? f.x : f.y);
      } else {
        const float2 f = unpack2(v[kFrom + c]);
        T o[2];
        convert(f.x, &o[0]);
        convert(f.y, &o[1]);
        memcpy(&stage[lane * 33 + c], o, 4);
      }
    }
    __syncwarp();
    if (kPass == 2) {
      if (h * 32 + lane < n)
#pragma unroll 4
        for (int r = 0; r < rows; ++r)
          reinterpret_cast<uint32_t *>(dst)[static_cast<size_t>(r) * N + h * 32 + lane] = stage[r * 33 + lane];
    } else if (N % 2 == 0) {
      if (2 * lane < n)
#pragma unroll 4
        for (int r = 0; r < rows; ++r)
          *reinterpret_cast<uint32_t *>(dst + static_cast<size_t>(r) * N + 2 * lane) = stage[r * 33 + lane];
    } else {
      const T *from = reinterpret_cast<const T *>(stage);
#pragma unroll 4
      for (int r = 0; r < rows; ++r) {
        T *to = dst + static_cast<size_t>(r) * N;
        if (lane < n) to[lane] = from[r * 66 + lane];
        if (lane + 32 < n) to[lane + 32] = from[r * 66 + lane + 32];
      }
    }
  }
}

// Rows16: y in fp16 with one power of two per row and 64 columns, which brings their
// largest value to 2^14 .. 2^15; fp16's 11 bits then hold for values down to 2^-28 of
// it.  (Rounding the expert outputs so costs an eighth of the final rounding to
// bf16, and halves what the product writes and the weighted sum reads.)
struct Rows16 {};

// The factor's exponent bits for the largest magnitude m: m < 2^(e - 126), factor 2^(141 - e),
// e >= 15 so that it is a number.
__device__ __forceinline__ uint32_t rows16_exponent(float m) { return max(__float_as_uint(m) >> 23, 15u); }

template <int kFrom>
__device__ __forceinline__ void convert_row16(float *inv, const uint64_t (&v)[64], uint32_t (&w)[32]) {
  float m = 0.f;
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    const float2 f = unpack2(v[kFrom + c]);
    m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
  }
  const uint32_t e = rows16_exponent(m);
  const float f = __uint_as_float((268u - e) << 23);
  if (inv != nullptr) *inv = __uint_as_float((e - 14u) << 23);
  const uint64_t f2 = pack2(f, f);
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    const float2 s = unpack2(mul2(v[kFrom + c], f2));
    const __half2 h = __floats2half2_rn(s.x, s.y);
    memcpy(&w[c], &h, 4);
  }
}

// A warp's 32 rows x 64 columns.  Rows that are all there go out by TMA through 4 KB of shared
// memory (a thread's own stores would touch 32 lines with every instruction, which the
// load-store unit takes one by one: the down products of 8192 tokens, eight of 128 experts
// each, d = 2048, F = 768, 180 -> 169 us); a tile's last rows by the threads themselves.
template <int kFrom>
__device__ __forceinline__ void store_row16(const CUtensorMap *tm, uint32_t stage, __half *dst, float *inv, int x, int y,
                                            bool live, const uint64_t (&v)[64]) {
  const int lane = threadIdx.x & 31;
  uint32_t w[32];
  convert_row16<kFrom>(live ? inv : nullptr, v, w);
  if (__all_sync(0xffffffffu, live)) {
    if (lane == 0) bulk_wait_read();   // the rows before these have left
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)   // 128-byte swizzle
      sts128(stage + lane * 128 + ((j ^ (lane & 7)) << 4), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(tm, stage, x, y);
      bulk_commit();
    }
  } else if (live) {
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
      uint32_t o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = w[c + j];
      store32(dst + 2 * c, o);
    }
  }
}

template <class T, bool kWide>
using ShapeOf = Shape<std::is_same_v<T, Rows16> ? 4096 : kWide ? 0 : kOddOut>;

// The units of a CTA pair in which a wait ran out become NaN, those that it had finished too, so that a
// call without `stats` does not pass for a whole one.
template <bool kGlu, class T>
__device__ __noinline__ void give_nan(const F8Params &p, int n_units) {
  using Out = std::conditional_t<std::is_same_v<T, Rows16>, __half, T>;
  const int w = static_cast<int>(threadIdx.x >> 5) - 4, half = w >> 2;
  const int trow = (w & 3) * 32 + static_cast<int>(threadIdx.x & 31) + static_cast<int>(cluster_ctarank()) * kRows;
  const int CB = kGlu ? p.NB : (p.N + kCols - 1) / kCols;
  for (int u = static_cast<int>(blockIdx.x >> 1); u < n_units; u += static_cast<int>(gridDim.x >> 1)) {
    const int i = u / CB, cb = u - i * CB;
    const int row0 = p.tiles != nullptr ? p.tiles[i].row0 : i * kF8PairTile;
    const int ntok = p.tiles != nullptr ? p.tiles[i].ntok : min(kF8PairTile, p.rows - row0);
    if (trow >= ntok) continue;
    const size_t at = static_cast<size_t>(row0 + trow) * p.N;
    for (int c = 0; c < (kGlu ? 64 : 128); ++c) {
      const int n = (kGlu ? cb * 128 : cb * kCols) + half * 64 + (c & 63) + (c >> 6) * 128;
      if constexpr (kGlu)
        p.hq[at + n] = kE4m3Nan;
      else if (n < p.N)
        convert(NAN, static_cast<Out *>(p.y) + at + n);
    }
  }
}

// T: the output's type (unused in the SwiGLU form); kWide: store_row() serves.  (An instance
// with both ways to store spilled registers in the loop over K.)
template <bool kGlu, class T, bool kWide>
__global__ void __launch_bounds__(kThreads, 1) f8_kernel(const __grid_constant__ F8Params p) {
  using S = ShapeOf<T, kWide>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t sbase = smem_u32(smem), bar0 = sbase + S::kBarOffset;
  // Rank 0's full and accempty barriers serve both CTAs.
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  // Accumulator b = 2 warpgroup + turn, TMEM columns 128 b ...
  auto accfull_bar = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
  auto accempty_bar = [&](int b) { return bar0 + 8u * (2 * kStages + 4 + b); };
  const uint32_t drain_bar = bar0 + 8u * (2 * kStages + 8), meet_bar = bar0 + 8u * (2 * kStages + 9);
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + S::kBarOffset + 8 * (2 * kStages + 10));
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  float *s_amax = reinterpret_cast<float *>(smem + S::kAmaxOffset);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1 + (blockIdx.x == 0 && p.hold == s + 1u));   // hold: see F8Args
      mbar_init(empty_bar(s), 2);   // both issuers' MMAs
    }
    for (int b = 0; b < 4; ++b) {
      mbar_init(accfull_bar(b), 1);
      mbar_init(accempty_bar(b), kEpiWarps);
    }
    mbar_init(drain_bar, 2);
    mbar_init(meet_bar, kEpiWarps);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&p.tmB[0]);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(tmem_slot), 2 * kCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();   // both CTAs' barriers are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  const bool listed = p.tiles != nullptr;
  // Without `early` nothing may be read before the kernels before this one are done.
  if (!p.early) pdl_wait();
  const int n_tiles = listed ? __ldcg(&p.meta->n_tiles) : (p.rows + kF8PairTile - 1) / kF8PairTile;
  const int CB = kGlu ? p.NB : (p.N + kCols - 1) / kCols, KB = p.KB;
  const int n_units = n_tiles * CB;   // below 2^26 within the limits of the calls
  if (threadIdx.x == 0) tmem_slot[2] = static_cast<uint32_t>(n_units);   // for give_nan()
  struct Unit {
    int expert, row0, ntok, cb;
  };
  auto unit_at = [&](int u) {
    const int i = u / CB;
    Unit r;
    r.cb = u - i * CB;
    if (listed) {
      const int4 t4 = __ldcg(reinterpret_cast<const int4 *>(p.tiles) + i);
      r.expert = t4.x;
      r.row0 = t4.y;
      r.ntok = t4.z;
    } else {
      r.expert = 0;
      r.row0 = i * kF8PairTile;
      r.ntok = min(kF8PairTile, p.rows - r.row0);
    }
    return r;
  };
  // Units u_first, u_first + unit_step, ...: n_blocks K blocks (below 2^32 within the limits).
  const int u_first = static_cast<int>(blockIdx.x >> 1), unit_step = static_cast<int>(gridDim.x >> 1);
  const uint32_t n_blocks =
      u_first < n_units ? static_cast<uint32_t>((n_units - u_first + unit_step - 1) / unit_step) * KB : 0;

  // Rows of a tile in this CTA, and the smallest box that holds them (-1: none).
  auto rows_here = [&](const Unit &t, uint32_t rk) { return min(max(t.ntok - static_cast<int>(rk) * kRows, 0), kRows); };
  auto box_of = [](int n) { return n == 0 ? -1 : n <= 16 ? 0 : n <= 32 ? 1 : n <= 64 ? 2 : 3; };
  auto box_bytes = [&](int n) { return n == 0 ? 0u : static_cast<uint32_t>(16 << box_of(n)) * kBK; };
  const uint32_t full0 = map_to_rank(full_bar(0), 0);
  const uint64_t pol_w = policy_evict_normal(), pol_x = policy_evict_last();
  // Weight rows that rank rk loads.  Rows beyond the matrix are left out: their products are not
  // stored, and many CTAs that fetch them at once wait for one another (see gemm_f8_few.cu).
  auto weights_of = [&](const Unit &t, uint32_t rk) {
    const int left = kGlu ? 128 : p.N - t.cb * kCols - 128 * static_cast<int>(rk);
    return left >= 128 ? 128 : left > 0 ? p.edge : 0;
  };
  auto load_b = [&](const Unit &t, int kb, int stage) {
    const uint32_t dst = sbase + stage * kStageBytes + kABytes, bar = full0 + 8u * stage;
    const int row = t.expert * p.N + t.cb * (kGlu ? 128 : kCols), n = weights_of(t, rank);
    if (n > 0)
      tma_load_2d_pair(dst, &p.tmB[kGlu ? rank : n == 128 ? 0 : 2], bar, kb * kBK,
                       kGlu ? row : row + 128 * static_cast<int>(rank), pol_w);
  };
  auto load_a = [&](const Unit &t, int kb, int stage) {
    const int box = box_of(rows_here(t, rank));
    if (box >= 0)
      tma_load_2d_pair(sbase + stage * kStageBytes, &p.tmA[box], full0 + 8u * stage, kb * kBK,
                       t.row0 + static_cast<int>(rank) * kRows, pol_x);
  };
  // Bytes that arrive for one step (both CTAs').
  auto step_bytes = [&](const Unit &t) {
    return static_cast<uint32_t>((weights_of(t, 0) + weights_of(t, 1)) * kBK) + box_bytes(rows_here(t, 0)) +
           box_bytes(rows_here(t, 1));
  };
  auto fail = [&]() {
    if (p.meta) atomicMax(&p.meta->status, XS_DEV_TIMEOUT);
    if (p.stats) atomicMax(&p.stats->status, XS_DEV_TIMEOUT);
    for (uint32_t r = 0; r < 2; ++r)  // both CTAs stop
      st_cluster_u32(map_to_rank(smem_u32(const_cast<int *>(abort_flag)), r), 1u);
  };

  const int n_pre = p.early ? static_cast<int>(n_blocks < kStages ? n_blocks : kStages) : 0;
  if (warp == 0 && n_pre > 0) {
    // Every stage is free at the start: its weights do not wait for the kernel before.
    int u = u_first;
    Unit t = unit_at(u);
    for (int i = 0, kb = 0; i < n_pre; ++i) {
      if (elect_one()) {
        if (rank == 0) mbar_arrive_expect_tx(full_bar(i), step_bytes(t));
        load_b(t, kb, i);
      }
      __syncwarp();
      if (++kb == KB && i + 1 < n_pre) {
        kb = 0;
        u += unit_step;
        t = unit_at(u);
      }
    }
  }
  if (p.early) pdl_wait();
  pdl_trigger();

  if (warp < 4) regs_dec<kIssueRegs>();
  if (warp == 0) {
    // ------------------------------------------------ TMA producer
    int stage = 0, kb = 0;
    uint32_t phase = 0;
    bool ok = true;
    int u = u_first;
    Unit t;
    if (n_blocks > 0) t = unit_at(u);
#pragma unroll 1
    for (uint32_t i = 0; i < n_blocks; ++i) {
      if (i >= kStages) {
        ok = mbar_wait_warp(empty_bar(stage), phase ^ 1u, kF8WaitNs, abort_flag);
        if (!ok) break;
      }
      if (elect_one()) {
        if (i >= n_pre) {
          if (rank == 0) mbar_arrive_expect_tx(full_bar(stage), step_bytes(t));
          load_b(t, kb, stage);
        }
        load_a(t, kb, stage);
      }
      __syncwarp();
      if (++kb == KB && i + 1 < n_blocks) {
        kb = 0;
        u += unit_step;
        t = unit_at(u);
      }
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    // The last MMAs have read every stage, and this CTA got every signal that is sent to it.
    if (n_blocks > 0)
      for (int j = 0; ok && j < kStages; ++j) {
        if (n_blocks + j >= static_cast<uint32_t>(kStages))
          ok = mbar_wait_warp(empty_bar(stage), phase ^ 1u, kF8WaitNs, abort_flag);
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    if (!ok) {
      if (lane == 0) fail();
      // Copies may be in flight whose barrier no longer completes: they land
      // in microseconds; stay for two milliseconds.
      const uint64_t t_end = globaltimer() + 2000000ull;
      while (globaltimer() < t_end) __nanosleep(1000);
    }
  } else if ((warp == 1 || warp == 2) && rank == 0) {
    // ------------------------------------------------ MMA issuers, one for each epilogue warpgroup
    const int g = warp - 1;
    const uint64_t desc0 = sw128_desc(__shfl_sync(0xffffffffu, sbase, 0));
    const uint32_t acc0 = __shfl_sync(0xffffffffu, tmem, 0), idesc = idesc_e4m3(kF8PairTile, kCols / 2);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
#pragma unroll 1
    for (uint32_t i = 0; i < n_blocks; ++i) {
      ok = mbar_wait_warp(full_bar(stage), phase, p.wait_ns, abort_flag);
      if (!ok) break;
      const uint64_t da = desc0 + static_cast<uint64_t>(stage * (kStageBytes >> 4));
      const uint32_t turn = i & 1u;
      const int b = 2 * g + static_cast<int>(turn);
      ok = mbar_wait_warp(accempty_bar(b), ((i >> 1) & 1u) ^ 1u, kF8WaitNs, abort_flag);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        // Warpgroup g's weights: 64 of the 128 rows of either CTA.
        const uint64_t db = da + ((kABytes + g * kBBytes / 2) >> 4);
#pragma unroll
        for (int ks = 0; ks < kBK / 32; ++ks) {
          const uint64_t k16 = static_cast<uint64_t>((ks * 32) >> 4);
          mma_e4m3_pair(acc0 + b * (kCols / 2), da + k16, db + k16, idesc, ks > 0 ? 1u : 0u);
        }
        mma_commit_pair(accfull_bar(b));
        mma_commit_pair(empty_bar(stage));
      }
      __syncwarp();
      if (!ok) break;
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (!ok && lane == 0) fail();
    // All issued MMAs done before TMEM is released.
    if (n_blocks > 0) {
      if (elect_one()) mma_commit_pair_local(drain_bar);
      volatile int no_abort = 0;
      mbar_wait_warp(drain_bar, 0, kF8WaitNs, &no_abort);
    }
  } else if (warp >= 4) {
    // ------------------------------------------------ epilogue
    regs_inc<kEpiRegs>();
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int row = q * 32 + lane;           // accumulator row
    const int trow = row + static_cast<int>(rank) * kRows;   // row of the tile
    // Columns 64 half .. 64 half + 63 of either block.
    const uint32_t tq = tmem + (static_cast<uint32_t>(q * 32) << 16) + half * kCols;
    const uint32_t accfull0 = accfull_bar(2 * half);
    const uint32_t accempty0 = map_to_rank(accempty_bar(2 * half), 0);
    uint32_t met = 0;      // meetings of the epilogue warps so far
    // All epilogue warps of this CTA have come here; what they wrote to shared memory is visible.
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(meet_bar);
      return mbar_wait_warp(meet_bar, met++ & 1u, kF8WaitNs, abort_flag);
    };
    uint32_t i = 0;
    int u = u_first;
    bool ok = true;
    // A unit's scales: of this thread's token, of the two blocks of weight rows.
    auto token_scale = [&](const Unit &t) { return p.sa + static_cast<size_t>(t.row0 + trow) * KB; };
    auto weight_scale = [&](const Unit &t, int block) {
      const int nb = kGlu ? t.cb : min(t.cb * 2 + block, p.NB - 1);
      return (kGlu && block == 1 ? p.sb1 : p.sb0) + (static_cast<size_t>(t.expert) * p.NB + nb) * KB;
    };
    // The next K block's scales are on their way while this one's products are awaited, and the
    // next unit's tile and first scales during this unit.
    Unit next;
    float a_next = 0.f, b0_next = 0.f, b1_next = 0.f;
    if (n_blocks > 0) {
      next = unit_at(u);
      if (trow < next.ntok) a_next = __ldg(token_scale(next));
      b0_next = __ldg(weight_scale(next, 0));
      b1_next = __ldg(weight_scale(next, 1));
    }
#pragma unroll 1
    while (i < n_blocks) {
      const Unit t = next;
      if (u + unit_step < n_units) next = unit_at(u + unit_step);
      const bool live = trow < t.ntok;
      const bool warp_live = trow - lane < t.ntok;
      const float *sa = token_scale(t), *sb0 = weight_scale(t, 0), *sb1 = weight_scale(t, 1);
      uint64_t acc[64];
#pragma unroll
      for (int j = 0; j < 64; ++j) acc[j] = 0ull;
#pragma unroll 1
      for (int kb = 0; kb < KB; ++kb, ++i) {
        const uint32_t turn = i & 1u;
        const float s0 = a_next * b0_next, s1 = a_next * b1_next;
        if (kb + 1 < KB) {
          a_next = live ? __ldg(sa + kb + 1) : 0.f;
          b0_next = __ldg(sb0 + kb + 1);
          b1_next = __ldg(sb1 + kb + 1);
        } else if (i + 1 < n_blocks) {
          a_next = trow < next.ntok ? __ldg(token_scale(next)) : 0.f;
          b0_next = __ldg(weight_scale(next, 0));
          b1_next = __ldg(weight_scale(next, 1));
        }
        ok = mbar_wait_warp(accfull0 + 8u * turn, (i >> 1) & 1u, kF8WaitNs, abort_flag);
        if (!ok) break;
        tc_fence_after();
        auto release = [&]() {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(accempty0 + 8u * turn);
        };
        if (warp_live) {
          const uint32_t tb = tq + turn * (kCols / 2);
          const uint64_t s0p = pack2(s0, s0), s1p = pack2(s1, s1);
#pragma unroll
          for (int c = 0; c < 2; ++c) {   // 64 columns of a block
            uint32_t v0[32], v1[32];
            tmem_ld32_async(tb + c * 64, v0);
            tmem_ld32_async(tb + c * 64 + 32, v1);
            tmem_wait32(v0);
            tmem_wait32(v1);
            if (c == 1) release();   // the last columns are in registers
            const uint64_t s = c == 0 ? s0p : s1p;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              acc[c * 32 + j] = fma2(pack2(v0[2 * j], v0[2 * j + 1]), s, acc[c * 32 + j]);
              acc[c * 32 + 16 + j] = fma2(pack2(v1[2 * j], v1[2 * j + 1]), s, acc[c * 32 + 16 + j]);
            }
          }
        } else {
          release();
        }
      }
      if (!ok) {
        if (lane == 0) fail();
        break;
      }
      const size_t out_row = static_cast<size_t>(t.row0 + trow);
      if constexpr (kGlu) {
        float h[64], m = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float2 g = unpack2(acc[j]), up = unpack2(acc[32 + j]);
          h[2 * j] = f8_silu(g.x) * up.x;
          h[2 * j + 1] = f8_silu(g.y) * up.y;
          m = fmaxf(m, fmaxf(fabsf(h[2 * j]), fabsf(h[2 * j + 1])));
        }
        // The two threads of a row meet; the next unit uses the other half of the buffer,
        // which all have left by then.
        const int side = static_cast<int>(met & 1u) * 2;
        s_amax[(side + half) * 128 + row] = m;
        ok = meet();
        if (!ok) {
          if (lane == 0) fail();
          break;
        }
        m = fmaxf(m, s_amax[(side + 1 - half) * 128 + row]);
        if (live) {
          const float s = f8_scale(m);
          const F8Divider div(s);
          uint8_t *dst = p.hq + out_row * p.N + t.cb * 128 + half * 64;
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
            float part[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) part[j] = h[c + j];
            uint32_t w[8];
            f8_quantise<32>(part, div, w);
            store32(dst + c, w);
          }
          if (half == 0) p.hs[out_row * p.NB + t.cb] = s;
        }
      } else if constexpr (std::is_same_v<T, Rows16>) {
        const int c0 = t.cb * kCols + half * 64, c1 = c0 + 128, y0 = t.row0 + trow - lane;
        __half *dst = static_cast<__half *>(p.y) + out_row * p.N;
        float *inv = p.inv + out_row * (p.N / 64);
        const uint32_t stage = sbase + S::kOutOffset + (warp - 4) * 4096;
        if (warp_live) {
          store_row16<0>(&p.tmY, stage, dst + c0, inv + c0 / 64, c0, y0, live, acc);
          if (c1 < p.N) store_row16<32>(&p.tmY, stage, dst + c1, inv + c1 / 64, c1, y0, live, acc);
        }
      } else {
        const int c0 = t.cb * kCols + half * 64, c1 = c0 + 128;
        T *dst = static_cast<T *>(p.y) + out_row * p.N;
        if (kWide) {
          if (live) {
            store_row<0>(dst + c0, acc, p.N - c0);
            store_row<32>(dst + c1, acc, p.N - c1);
          }
        } else if (warp_live) {
          uint32_t *stage = reinterpret_cast<uint32_t *>(smem + S::kOutOffset + (warp - 4) * kOddOut);
          T *first = dst - static_cast<size_t>(lane) * p.N;
          const int rows = min(t.ntok - (trow - lane), 32);
          if (c0 < p.N) store_rows_odd<0>(stage, first + c0, p.N, acc, rows, p.N - c0);
          if (c1 < p.N) store_rows_odd<32>(stage, first + c1, p.N, acc, rows, p.N - c1);
        }
      }
      u += unit_step;
    }
    if (std::is_same_v<T, Rows16> && lane == 0) bulk_wait_all();
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag && warp >= 4) give_nan<kGlu, T>(p, static_cast<int>(tmem_slot[2]));
  cluster_sync();   // neither CTA leaves while the other may still signal it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 2 * kCols);
  }
}

// ---------------------------------------------------------------- host side

// Row-major [outer, K] bytes, boxes of `rows` x 128, 128-byte swizzle.
bool make_map(CUtensorMap *m, const void *base, uint64_t K, uint64_t outer, uint32_t rows) {
  return encode_tmap_2d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, K, outer, kBK, rows,
                        CU_TENSOR_MAP_SWIZZLE_128B);
}

void launch_config(cudaLaunchConfig_t *cfg, cudaLaunchAttribute *attr, int pairs, int smem, cudaStream_t s) {
  cfg->gridDim = dim3(2 * pairs);
  cfg->blockDim = dim3(kThreads);
  cfg->dynamicSmemBytes = smem;
  cfg->stream = s;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg->attrs = attr;
  cfg->numAttrs = 2;
}

// CTA pairs that the current device runs at once (cached per device; host threads
// that race on it store the same value).
int resident_pairs(int sms) {
  constexpr int kDevs = 64;
  static std::atomic<int> cache[kDevs];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevs) return sms / 2;
  int n = cache[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  constexpr int kSmemBytes = ShapeOf<float, true>::kSmemBytes;
  launch_config(&cfg, attr, 1, kSmemBytes, nullptr);
  cfg.numAttrs = 1;   // the cluster alone
  // The query wants the shared-memory limit of the form it asks about.
  if (cudaFuncSetAttribute(reinterpret_cast<const void *>(f8_kernel<false, float, true>),
                           cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, f8_kernel<false, float, true>, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();  // a failed query leaves no sticky error
    n = sms / 2;
  }
  n = n < sms / 2 ? n : sms / 2;
  cache[dev].store(n, std::memory_order_relaxed);
  return n;
}

template <bool kGlu, class T, bool kWide>
cudaError_t launch(const F8Args &a, cudaStream_t s) {
  constexpr bool kRows16 = std::is_same_v<T, Rows16>;
  constexpr int kSmemBytes = ShapeOf<T, kWide>::kSmemBytes;
  static_assert(kSmemBytes <= 227 * 1024, "fits an SM");
  F8Params p;
  memset(&p, 0, sizeof(p));
  if (kRows16 && !encode_tmap_2d(&p.tmY, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.y, a.N, a.rows, 64, 32,
                                 CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  for (int i = 0; i < kBoxes; ++i)
    if (!make_map(&p.tmA[i], a.a, a.K, a.rows, 16u << i)) return cudaErrorInvalidValue;
  const uint64_t wrows = static_cast<uint64_t>(a.E) * a.N;
  if (!make_map(&p.tmB[0], a.b0, a.K, wrows, 128) || (kGlu && !make_map(&p.tmB[1], a.b1, a.K, wrows, 128)))
    return cudaErrorInvalidValue;
  p.edge = edge_rows(a.N);
  if (p.edge < 128 && !make_map(&p.tmB[2], a.b0, a.K, wrows, p.edge)) return cudaErrorInvalidValue;
  p.sa = a.sa;
  p.sb0 = a.sb0;
  p.sb1 = a.sb1;
  p.tiles = a.tiles;
  p.meta = a.meta;
  p.stats = a.stats;
  p.y = a.y;
  p.inv = a.inv;
  p.hq = a.hq;
  p.hs = a.hs;
  p.rows = a.rows;
  p.N = a.N;
  p.KB = (a.K + kBK - 1) / kBK;
  p.NB = (a.N + 127) / 128;
  p.early = a.early;
  p.hold = a.hold;
  p.wait_ns = a.wait_ns;
  const long long tiles = a.tiles != nullptr ? a.max_tiles : (a.rows + kF8PairTile - 1) / kF8PairTile;
  const long long units = tiles * (kGlu ? p.NB : (a.N + kCols - 1) / kCols);
  const int sms = a.n_sms < kF8Ctas ? a.n_sms : kF8Ctas;
  const int pairs = resident_pairs(sms);
  cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(f8_kernel<kGlu, T, kWide>),
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  static std::atomic<bool> seen{false};
  if (e == cudaSuccess) e = check_registers(reinterpret_cast<const void *>(f8_kernel<kGlu, T, kWide>), &seen);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  launch_config(&cfg, attr, static_cast<int>(units < pairs ? units : pairs), kSmemBytes, s);
  return cudaLaunchKernelEx(&cfg, f8_kernel<kGlu, T, kWide>, p);
}

template <class T>
cudaError_t launch_rows(const F8Args &a, cudaStream_t s) {
  const bool wide = (static_cast<size_t>(a.N) * sizeof(T)) % 32 == 0 && reinterpret_cast<uintptr_t>(a.y) % 32 == 0;
  return wide ? launch<false, T, true>(a, s) : launch<false, T, false>(a, s);
}

}  // namespace

cudaError_t launch_f8_pairs(const F8Args &a, cudaStream_t s) {
  if (a.b1 != nullptr) return launch<true, float, true>(a, s);
  if (a.inv != nullptr) return launch<false, Rows16, true>(a, s);
  if (a.y_dtype == XS_BF16) return launch_rows<__nv_bfloat16>(a, s);
  if (a.y_dtype == XS_F16) return launch_rows<__half>(a, s);
  return launch_rows<float>(a, s);
}

}  // namespace xs
