// Products of block-scaled float8 operands for few token rows per matrix (see
// gemm_f8.cu for the mathematics and the form for many): the weights' bytes bound
// them, and the kernel's business is to keep HBM streaming.
//
// The weights are the MMA's M rows (one per TMEM lane), up to kTok tokens its N
// columns: a K block of 256 weight rows (two blocks of 128; SwiGLU: gate and up of
// the same hidden units) is eight MMAs of N = 16 .. 64, a fraction of the time that its
// 32 KB take from HBM, and its products are kTok columns in one of four TMEM buffers.  An
// epilogue thread owns a weight row of one of the two blocks and adds its columns,
// each scaled by its token's scale times the block's, to kTok fp32 sums.
//
// Unit: (tile of up to kTok rows of one matrix, 256 weight rows).  Few units would leave most
// SMs idle, so several CTAs share a unit's K blocks, in one of two ways:
//   kSplit: where every unit finds a cluster of two to eight CTAs at once, each CTA of it takes its
//     part of K, and the first adds the others' sums from their shared memory: a
//     microsecond, where a meeting in global memory takes five.  One row of 4096 x 7168: 11.4 ->
//     9.0 us, 32 rows 18.3 -> 12.0; 16 rows of 2048 x 7168 14.9 -> 9.8.
//   Else, where whole units would leave CTAs idle for long, the K blocks of all units are
//     dealt to the CTAs in equal contiguous ranges; a unit cut between CTAs is finished by
//     the one that arrives last, from the partial sums in global memory.  (Clusters in two waves
//     lose: 16 units in 15 clusters of eight 16 us, 96 units of 12 blocks in pairs 10.6 | 10.5 without.)
// The sums are added in the order of K whoever adds them, so the result does not depend on
// the schedule.
//
// SwiGLU: one warpgroup has the gate rows, the other the up rows of the same hidden
// units; they exchange half of the tokens through shared memory, each finishes the
// other half, and the four warps' maxima over the 128 hidden units give the scales.
//
// Roles (three warpgroups): in the first, warp 0 loads by TMA and warp 1 issues the
// MMAs; the other two are the epilogue.  Every wait is bounded in time.
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
// Registers per thread of the first and the other two warpgroups.
constexpr int kIssueRegs = 104, kEpiRegs = 200;
static_assert(kIssueRegs + 2 * kEpiRegs <= 3 * kF8Regs, "the launch holds what the warpgroups ask for");
constexpr int kBK = 128;                         // e4m3 per K block: one swizzle row, one scale
constexpr int kRows = 256;                       // weight rows of a unit
constexpr int kWBytes = kRows * kBK;             // 32 KB of weights per K block
constexpr int kBufs = 4;                         // TMEM buffers
constexpr int kBoxes = 3;                        // token boxes of 16, 32, 64 rows
constexpr int kMinBlocks = 2;                    // K blocks per CTA at least

template <int kTok, bool kSplit>
struct Shape {
  static constexpr int kStageBytes = kWBytes + kTok * kBK;
  static constexpr int kStages = kTok <= 32 ? 5 : 4;
  static constexpr int kSwapOffset = kStages * kStageBytes;                  // [2][kTok / 2][128] floats; kSplit: or
                                                                             // [kTok][256], sums for the first CTA
  static constexpr int kScaleOffset = kSwapOffset + kTok * 128 * 4 * (kSplit ? 2 : 1);   // [8 warps][2][kTok] floats
  static constexpr int kMaxOffset = kScaleOffset + kEpiWarps * 2 * kTok * 4; // [8 warps][kTok / 2] floats
  static constexpr int kBarOffset = kMaxOffset + kEpiWarps * kTok * 2;
  static constexpr int kSmemBytes = kBarOffset + 256 + 1024;                 // + alignment slack
};

struct FewParams {
  CUtensorMap tmX[kBoxes]; // tokens
  CUtensorMap tmW[3];      // weights [E N, K], boxes of 128 rows; [1]: up; [2]: of `edge` rows
  const float *sa, *sb0, *sb1;
  const Tile *tiles;
  PermMeta *meta;
  xs_stats *stats;
  void *y;
  uint8_t *hq;
  float *hs;
  float *part;             // [CTA][2][kTok][256] partial sums
  int32_t *cnt;            // arrivals per CTA, zero at the start
  int rows, N, KB, NB;     // NB: scale rows of a matrix, ceil(N / 128)
  int edge;                // box rows of a matrix's last 128-row block, if that is not whole
  int early;
  uint32_t hold;
  uint64_t wait_ns;
};

__device__ __forceinline__ void convert(float v, float *o) { *o = v; }
__device__ __forceinline__ void convert(float v, __nv_bfloat16 *o) { *o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void convert(float v, __half *o) { *o = __float2half_rn(v); }

// The units of a CTA in which a wait ran out become NaN, those that it had finished too, so that a
// call without `stats` does not pass for a whole one.  (A cut unit without this CTA's part is
// finished by nobody else; all CTAs of a cluster give up together.)  `mine`: the first unit, the end, the step.
template <int kTok, bool kGlu, class T>
__device__ __noinline__ void give_nan(const FewParams &p, const uint32_t *mine) {
  const int w = static_cast<int>(threadIdx.x >> 5) - 4, g = w >> 2, row = (w & 3) * 32 + static_cast<int>(threadIdx.x & 31);
  const int CB = kGlu ? p.NB : (p.N + kRows - 1) / kRows;
  for (uint32_t v = mine[0]; v < mine[1]; v += mine[2]) {
    const int u = static_cast<int>(v);
    const int i = u / CB, cb = u - i * CB;
    const int row0 = p.tiles != nullptr ? p.tiles[i].row0 : i * kTok;
    const int ntok = p.tiles != nullptr ? p.tiles[i].ntok : min(kTok, p.rows - row0);
    const int n = kGlu ? cb * 128 + row : cb * kRows + g * 128 + row;
    const int j0 = kGlu ? g * (kTok / 2) : 0, j1 = kGlu ? min(ntok, j0 + kTok / 2) : ntok;
    for (int j = j0; j < j1 && n < p.N; ++j) {
      const size_t at = static_cast<size_t>(row0 + j) * p.N + n;
      if constexpr (kGlu)
        p.hq[at] = kE4m3Nan;
      else
        convert(NAN, static_cast<T *>(p.y) + at);
    }
  }
}

// T: the output's type (unused in the SwiGLU form).  kSplit: launched as a cluster for every unit.
template <int kTok, bool kGlu, class T, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1) f8_few_kernel(const __grid_constant__ FewParams p) {
  using S = Shape<kTok, kSplit>;
  constexpr int kStages = S::kStages, kStageBytes = S::kStageBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t sbase = smem_u32(smem), bar0 = sbase + S::kBarOffset;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto accfull_bar = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
  auto accempty_bar = [&](int b) { return bar0 + 8u * (2 * kStages + kBufs + b); };
  const uint32_t drain_bar = bar0 + 8u * (2 * kStages + 2 * kBufs), meet_bar = drain_bar + 8u;
  const uint32_t parts_bar = drain_bar + 16u;   // kSplit, the first CTA's: the others' sums are there
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + S::kBarOffset + 8 * (2 * kStages + 2 * kBufs + 3));
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  volatile uint32_t *s_cut = tmem_slot + 2;   // a cut unit's first and last CTA, and whether this one finishes it

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = kSplit ? cluster_ctarank() : 0, ranks = kSplit ? cluster_nctarank() : 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1 + (blockIdx.x == 0 && p.hold == s + 1u));   // hold: see F8Args
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      mbar_init(accfull_bar(b), 1);
      mbar_init(accempty_bar(b), kEpiWarps);
    }
    mbar_init(drain_bar, 1);
    mbar_init(meet_bar, kEpiWarps);
    mbar_init(parts_bar, kSplit ? (ranks - 1) * kEpiWarps : 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&p.tmW[0]);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kBufs * 2 * kTok);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  if (kSplit) cluster_sync();   // every CTA's barriers are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  const bool listed = p.tiles != nullptr;
  // Without `early` nothing may be read before the kernels before this one are done.
  if (!p.early) pdl_wait();
  const int n_tiles = listed ? __ldcg(&p.meta->n_tiles) : (p.rows + kTok - 1) / kTok;
  const int CB = kGlu ? p.NB : (p.N + kRows - 1) / kRows, KB = p.KB;
  const int n_units = n_tiles * CB;   // below 2^28 within the limits of the calls
  struct Unit {
    int expert, row0, ntok, cb, single;
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
      r.single = t4.w;
    } else {
      r.expert = 0;
      r.row0 = i * kTok;
      r.ntok = min(kTok, p.rows - r.row0);
      r.single = n_tiles == 1;
    }
    return r;
  };
  // Work: n_blocks K blocks from block kb_first of unit u_first on, in steps of unit_step units.
  const long long blocks = static_cast<long long>(n_units) * KB;
  // kSplit: one unit for each cluster, of which this CTA has the blocks kb_begin .. kb_end - 1.
  const int kb_begin = kSplit ? static_cast<int>(KB * rank / ranks) : 0;
  const int kb_end = kSplit ? static_cast<int>(KB * (rank + 1) / ranks) : KB;
  int u_first = static_cast<int>(blockIdx.x / ranks), kb_first = kb_begin, unit_step = static_cast<int>(gridDim.x / ranks);
  uint32_t n_blocks =
      u_first < n_units ? static_cast<uint32_t>((n_units - u_first + unit_step - 1) / unit_step) * (kb_end - kb_begin) : 0;
  uint32_t n_cta = 1;    // CTAs that share the blocks, if units are cut
  int n_mine = n_units;  // units from here on are other CTAs'
  if (!kSplit) {
    // What a CTA does at most with whole units, and with equal shares.
    const long long whole = static_cast<long long>((n_units + unit_step - 1) / unit_step) * KB;
    if (whole - blocks / unit_step >= kF8CutBlocks) {
      const long long want = (blocks + kMinBlocks - 1) / kMinBlocks;
      n_cta = want < unit_step ? static_cast<uint32_t>(want) : unit_step;
      const bool mine = blockIdx.x < n_cta;
      const long long first = mine ? blocks * blockIdx.x / n_cta : 0, last = mine ? blocks * (blockIdx.x + 1) / n_cta : 0;
      u_first = static_cast<int>(first / KB);
      kb_first = static_cast<int>(first - static_cast<long long>(u_first) * KB);
      n_blocks = static_cast<uint32_t>(last - first);
      n_mine = static_cast<int>((last + KB - 1) / KB);
      unit_step = 1;
    }
  }

  if (threadIdx.x == 0) {   // for give_nan()
    tmem_slot[5] = static_cast<uint32_t>(u_first);
    tmem_slot[6] = static_cast<uint32_t>(n_mine);
    tmem_slot[7] = static_cast<uint32_t>(unit_step);
  }

  auto box_of = [](int n) { return n <= 16 ? 0 : n <= 32 ? 1 : 2; };
  // An expert's weights are read once if it has a single tile; its tokens are read
  // again for every 256 weight rows.
  const uint64_t pol_once = policy_evict_first(), pol_again = policy_evict_normal(), pol_x = policy_evict_last();
  // Weight rows of block g that are loaded.  Rows beyond the matrix are left out: their products are not
  // stored, and many CTAs that fetch them at once wait for one another (1202 rows of 1 x
  // 5536: 60 -> 12.5 us).
  auto weights_of = [&](const Unit &t, int g) {
    const int left = kGlu ? 128 : p.N - t.cb * kRows - 128 * g;
    return left >= 128 ? 128 : left > 0 ? p.edge : 0;
  };
  auto load_w = [&](const Unit &t, int kb, int stage) {
    const int row = t.expert * p.N + t.cb * (kGlu ? 128 : kRows);
    const uint64_t pol = t.single ? pol_once : pol_again;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int n = weights_of(t, g);
      if (n > 0)
        tma_load_2d(sbase + stage * kStageBytes + g * (kWBytes / 2), &p.tmW[kGlu ? g : n == 128 ? 0 : 2], full_bar(stage),
                    kb * kBK, kGlu ? row : row + 128 * g, pol);
    }
  };
  auto load_x = [&](const Unit &t, int kb, int stage) {
    tma_load_2d(sbase + stage * kStageBytes + kWBytes, &p.tmX[box_of(t.ntok)], full_bar(stage), kb * kBK, t.row0, pol_x);
  };
  auto step_bytes = [&](const Unit &t) {
    return static_cast<uint32_t>((weights_of(t, 0) + weights_of(t, 1) + (16 << box_of(t.ntok))) * kBK);
  };
  auto fail = [&]() {
    if (p.meta) atomicMax(&p.meta->status, XS_DEV_TIMEOUT);
    if (p.stats) atomicMax(&p.stats->status, XS_DEV_TIMEOUT);
    if (kSplit)
      for (uint32_t r = 0; r < ranks; ++r)   // all CTAs of the cluster stop
        st_cluster_u32(map_to_rank(smem_u32(const_cast<int *>(abort_flag)), r), 1u);
    else
      *abort_flag = 1;
  };

  const int n_pre = p.early ? static_cast<int>(n_blocks < kStages ? n_blocks : kStages) : 0;
  if (warp == 0 && n_pre > 0) {
    // Every stage is free at the start: its weights do not wait for the kernel before.
    int u = u_first;
    Unit t = unit_at(u);
    for (int i = 0, kb = kb_first; i < n_pre; ++i) {
      if (elect_one()) {
        mbar_arrive_expect_tx(full_bar(i), step_bytes(t));
        load_w(t, kb, i);
      }
      __syncwarp();
      if (++kb == kb_end && i + 1 < n_pre) {
        kb = kb_begin;
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
    int stage = 0, kb = kb_first, u = u_first;
    uint32_t phase = 0;
    bool ok = true;
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
          mbar_arrive_expect_tx(full_bar(stage), step_bytes(t));
          load_w(t, kb, stage);
        }
        load_x(t, kb, stage);
      }
      __syncwarp();
      if (++kb == kb_end && i + 1 < n_blocks) {
        kb = kb_begin;
        u += unit_step;
        t = unit_at(u);
      }
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (!ok && lane == 0) fail();
  } else if (warp == 1) {
    // ------------------------------------------------ MMA issuer
    const uint64_t desc0 = sw128_desc(__shfl_sync(0xffffffffu, sbase, 0));
    const uint32_t acc0 = __shfl_sync(0xffffffffu, tmem, 0);
    int stage = 0, kb = kb_first, u = u_first;
    uint32_t phase = 0, idesc = 0;
    bool ok = true;
#pragma unroll 1
    for (uint32_t i = 0; i < n_blocks; ++i) {
      if (i == 0 || kb == kb_begin) {
        const Unit t = unit_at(u);
        idesc = __shfl_sync(0xffffffffu, idesc_e4m3(128, 16 << box_of(t.ntok)), 0);
      }
      const int buf = static_cast<int>(i % kBufs);
      ok = mbar_wait_warp(accempty_bar(buf), ((i / kBufs) & 1u) ^ 1u, kF8WaitNs, abort_flag) &&
           mbar_wait_warp(full_bar(stage), phase, p.wait_ns, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint64_t dw = desc0 + static_cast<uint64_t>(stage * (kStageBytes >> 4)), dx = dw + (kWBytes >> 4);
      if (elect_one()) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int ks = 0; ks < kBK / 32; ++ks) {
            const uint64_t k16 = static_cast<uint64_t>((ks * 32) >> 4);
            mma_e4m3(acc0 + (buf * 2 + g) * kTok, dw + g * (kWBytes >> 5) + k16, dx + k16, idesc, ks > 0 ? 1u : 0u);
          }
        mma_commit(accfull_bar(buf));
        mma_commit(empty_bar(stage));
      }
      __syncwarp();
      if (++kb == kb_end) {
        kb = kb_begin;
        u += unit_step;
      }
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (!ok && lane == 0) fail();
    // All issued MMAs done before TMEM is released.
    if (n_blocks > 0) {
      if (elect_one()) mma_commit(drain_bar);
      volatile int no_abort = 0;
      mbar_wait_warp(drain_bar, 0, kF8WaitNs, &no_abort);
    }
  } else if (warp >= 4) {
    // ------------------------------------------------ epilogue
    regs_inc<kEpiRegs>();
    const int q = warp & 3, g = (warp - 4) >> 2;   // TMEM lane quarter, block of weight rows
    const int row = q * 32 + lane;                 // weight row of the block
    const uint32_t tq = tmem + (static_cast<uint32_t>(q * 32) << 16) + g * kTok;
    float *s_scale = reinterpret_cast<float *>(smem + S::kScaleOffset) + (warp - 4) * 2 * kTok;
    float *s_swap = reinterpret_cast<float *>(smem + S::kSwapOffset);
    float *s_max = reinterpret_cast<float *>(smem + S::kMaxOffset);
    uint32_t met = 0;      // meetings of the epilogue warps so far
    // All epilogue warps have come here; what they wrote to shared memory is visible.
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(meet_bar);
      return mbar_wait_warp(meet_bar, met++ & 1u, kF8WaitNs, abort_flag);
    };
    uint32_t i = 0;
    int u = u_first;
    bool ok = true;
#pragma unroll 1
    while (i < n_blocks) {
      const Unit t = unit_at(u);
      const int kb0 = i == 0 ? kb_first : kb_begin;
      const int kb1 = static_cast<int>(min(static_cast<uint32_t>(kb_end), kb0 + n_blocks - i));
      const int cols = 16 << box_of(t.ntok);     // of the MMAs
      const int nb = kGlu ? t.cb : min(t.cb * 2 + g, p.NB - 1);
      const float *sb = (kGlu && g == 1 ? p.sb1 : p.sb0) + (static_cast<size_t>(t.expert) * p.NB + nb) * KB;
      // Lane l fetches the scales of tokens l and l + 32, a K block ahead.
      const float *sa = p.sa + static_cast<size_t>(t.row0) * KB;
      auto token_scale = [&](int tok, int kb) { return tok < t.ntok ? __ldg(sa + static_cast<size_t>(tok) * KB + kb) : 0.f; };
      float a0 = token_scale(lane, kb0), a1 = kTok > 32 ? token_scale(lane + 32, kb0) : 0.f, b = __ldg(sb + kb0);
      uint64_t acc[kTok / 2];
#pragma unroll
      for (int j = 0; j < kTok / 2; ++j) acc[j] = 0ull;
#pragma unroll 1
      for (int kb = kb0; kb < kb1; ++kb, ++i) {
        const int buf = static_cast<int>(i % kBufs);
        float *sc = s_scale + (i & 1u) * kTok;
        sc[lane] = a0 * b;
        if (kTok > 32) sc[lane + 32] = a1 * b;
        __syncwarp();
        if (kb + 1 < kb1) {
          a0 = token_scale(lane, kb + 1);
          if (kTok > 32) a1 = token_scale(lane + 32, kb + 1);
          b = __ldg(sb + kb + 1);
        }
        ok = mbar_wait_warp(accfull_bar(buf), (i / kBufs) & 1u, kF8WaitNs, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tb = tq + buf * 2 * kTok;
        auto release = [&]() {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(accempty_bar(buf));
        };
        const ulonglong2 *scale2 = reinterpret_cast<const ulonglong2 *>(sc);
        if (cols <= 16) {
          uint32_t v[16];
          tmem_ld16_async(tb, v);
          tmem_wait16(v);
          release();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const ulonglong2 s = scale2[j];
            acc[2 * j] = fma2(pack2(v[4 * j], v[4 * j + 1]), s.x, acc[2 * j]);
            acc[2 * j + 1] = fma2(pack2(v[4 * j + 2], v[4 * j + 3]), s.y, acc[2 * j + 1]);
          }
        } else {
#pragma unroll
          for (int c = 0; c < kTok; c += 32) {
            if (c >= cols) break;
            uint32_t v[32];
            tmem_ld32_async(tb + c, v);
            tmem_wait32(v);
            if (c + 32 >= cols) release();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const ulonglong2 s = scale2[c / 4 + j];
              acc[c / 2 + 2 * j] = fma2(pack2(v[4 * j], v[4 * j + 1]), s.x, acc[c / 2 + 2 * j]);
              acc[c / 2 + 2 * j + 1] = fma2(pack2(v[4 * j + 2], v[4 * j + 3]), s.y, acc[c / 2 + 2 * j + 1]);
            }
          }
        }
      }
      bool finish = ok;
      // Adds the sums of CTAs c_first .. c_last, read by load(c, token).  A value is a trip to L2 or
      // another SM: 16 of a thread (more would spill registers) are under way at a time, of
      // several CTAs where there are few tokens.  (What is read of tokens beyond the tile's counts for
      // nothing.)
      constexpr int kAtOnce = 16;
      auto add_parts = [&](uint32_t c_first, uint32_t c_last, auto load) {
        auto add = [&](auto tokens, int j0) {
          constexpr int kN = decltype(tokens)::value, kParts = kAtOnce / kN;
#pragma unroll 1
          for (uint32_t c = c_first; c <= c_last; c += kParts) {
            float v[kParts][kN];
#pragma unroll
            for (uint32_t k = 0; k < kParts; ++k)
              if (c + k <= c_last)
#pragma unroll
                for (int j = 0; j < kN; ++j) v[k][j] = load(c + k, j0 + j);
#pragma unroll
            for (uint32_t k = 0; k < kParts; ++k)
              if (c + k <= c_last)
#pragma unroll
                for (int j = 0; j < kN; j += 2)
                  acc[(j0 + j) / 2] = add2(acc[(j0 + j) / 2], pack2(v[k][j], v[k][j + 1]));
          }
        };
        if (t.ntok <= 4) {
          add(std::integral_constant<int, 4>(), 0);
        } else if (t.ntok <= kAtOnce / 2) {
          add(std::integral_constant<int, kAtOnce / 2>(), 0);
        } else {
#pragma unroll
          for (int j0 = 0; j0 < kTok; j0 += kAtOnce)
            if (j0 < t.ntok) add(std::integral_constant<int, kAtOnce>(), j0);
        }
      };
      if constexpr (kSplit) {
        if (ok && rank != 0) {
          // The sums stay in this CTA's shared memory until the first CTA has read them.
          float *dst = s_swap + g * 128 + row;
#pragma unroll
          for (int j = 0; j < kTok; j += 2) {
            const float2 v = unpack2(acc[j / 2]);
            if (j < t.ntok) {
              dst[j * kRows] = v.x;
              dst[(j + 1) * kRows] = v.y;
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_rank(parts_bar, 0));
          finish = false;
        } else if (ok) {
          ok = mbar_wait_cluster(parts_bar, 0, kF8WaitNs, abort_flag);
          const uint32_t src = smem_u32(s_swap + g * 128 + row);
          if (ok)
            add_parts(1, ranks - 1,
                      [&](uint32_t c, int j) { return ld_cluster_f32(map_to_rank(src, c) + j * (kRows * 4)); });
        }
      } else if (ok && (kb0 > 0 || kb1 < KB)) {
        // A cut unit: this CTA's sums, then whoever comes last adds all of them up.
        // Slot 1 of the first of its CTAs (which begins with the unit, or before it), slot 0 of the others.
        auto part_of = [&](uint32_t c, int slot) {
          return p.part + static_cast<size_t>(c * 2 + slot) * kTok * kRows + g * 128 + row;
        };
        float *dst = part_of(blockIdx.x, kb0 > 0 ? 0 : 1);
#pragma unroll
        for (int j = 0; j < kTok; j += 2) {
          const float2 v = unpack2(acc[j / 2]);
          if (j < t.ntok) __stcg(dst + j * kRows, v.x);
          if (j + 1 < t.ntok) __stcg(dst + (j + 1) * kRows, v.y);
        }
        __threadfence();
        ok = meet();
        if (ok && warp == 4 && lane == 0) {
          const long long i0 = static_cast<long long>(u) * KB;
          const uint32_t c0 = static_cast<uint32_t>(((i0 + 1) * n_cta - 1) / blocks);
          const uint32_t c1 = static_cast<uint32_t>(((i0 + KB) * n_cta - 1) / blocks);
          s_cut[0] = c0;
          s_cut[1] = c1;
          s_cut[2] = atomicAdd(p.cnt + c0, 1) == static_cast<int>(c1 - c0);
          __threadfence();
        }
        ok = ok && meet();
        finish = ok && s_cut[2] != 0;
        if (finish) {
          const uint32_t c_first = s_cut[0];
#pragma unroll
          for (int j = 0; j < kTok / 2; ++j) acc[j] = 0ull;
          add_parts(c_first, s_cut[1],
                    [&](uint32_t c, int j) { return __ldcg(part_of(c, c == c_first ? 1 : 0) + j * kRows); });
        }
      }
      if (ok && finish && kGlu) {
        constexpr int kHalf = kTok / 2;
        // The up rows of tokens 0 .. kHalf - 1 to the gate's warpgroup, the gate rows of the others to the up's.
        float *swap = s_swap + (g == 1 ? 0 : kHalf * 128) + row;
#pragma unroll
        for (int j = 0; j < kHalf; j += 2) {
          const float2 v = unpack2(g == 1 ? acc[j / 2] : acc[(kHalf + j) / 2]);
          swap[j * 128] = v.x;
          swap[(j + 1) * 128] = v.y;
        }
        ok = meet();
        const float *other = s_swap + (g == 1 ? kHalf * 128 : 0) + row;
        float h[kHalf], m = 0.f;
#pragma unroll
        for (int j = 0; j < kHalf; j += 2) {
          const float2 own = unpack2(g == 1 ? acc[(kHalf + j) / 2] : acc[j / 2]);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float mine = k == 0 ? own.x : own.y, o = other[(j + k) * 128];
            const float gate = g == 0 ? mine : o, up = g == 0 ? o : mine;
            h[j + k] = f8_silu(gate) * up;
            // Magnitudes are ordered as their bits; a NaN counts as 0.
            const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fabsf(h[j + k]), 0.f)));
            if (lane == j + k) m = __uint_as_float(top);
          }
        }
        // Lane l of warp q: the maximum of token l (of this half) over the warp's hidden units.
        if (lane < kHalf) s_max[(warp - 4) * kHalf + lane] = m;
        ok = ok && meet();
        if (lane < kHalf)
#pragma unroll
          for (int w = 0; w < 4; ++w) m = fmaxf(m, s_max[(4 * g + w) * kHalf + lane]);
        const float s = f8_scale(m), r = 1.f / s;
        const int tok0 = g * kHalf;
        if (ok) {
          uint8_t *dst = p.hq + static_cast<size_t>(t.row0 + tok0) * p.N + t.cb * 128 + row;
          // Every token has a scale of its own, in lane j.
          auto quantise = [&](auto quotients) {
#pragma unroll
            for (int j = 0; j < kHalf; j += 2) {
              if (tok0 + j >= t.ntok) break;
              auto of = [&](float v, int k) { return __shfl_sync(0xffffffffu, v, k); };
              const F8Divider div(of(s, j), of(s, j + 1), of(r, j), of(r, j + 1));
              const uint32_t two = f8_pack2(quotients(div, h[j], h[j + 1]));
              dst[static_cast<size_t>(j) * p.N] = static_cast<uint8_t>(two);
              if (tok0 + j + 1 < t.ntok) dst[static_cast<size_t>(j + 1) * p.N] = static_cast<uint8_t>(two >> 8);
            }
          };
          // (Tokens that the tile does not have have the smallest scale, which counts for nothing.)
          if (__any_sync(0xffffffffu, lane < kHalf && tok0 + lane < t.ntok && F8Divider(s, r).plain))
            quantise([](const F8Divider &div, float a, float b) { return div.slow(a, b); });
          else
            quantise([](const F8Divider &div, float a, float b) { return div(a, b); });
          if (q == 0 && lane < kHalf && tok0 + lane < t.ntok)
            p.hs[static_cast<size_t>(t.row0 + tok0 + lane) * p.NB + t.cb] = s;
        }
      } else if (ok && finish) {
        const int n = t.cb * kRows + g * 128 + row;
        if (n < p.N) {
          T *dst = static_cast<T *>(p.y) + static_cast<size_t>(t.row0) * p.N + n;
#pragma unroll
          for (int j = 0; j < kTok; j += 2) {
            const float2 v = unpack2(acc[j / 2]);
            if (j < t.ntok) convert(v.x, dst + static_cast<size_t>(j) * p.N);
            if (j + 1 < t.ntok) convert(v.y, dst + static_cast<size_t>(j + 1) * p.N);
          }
        }
      }
      if (!ok) {
        if (lane == 0) fail();
        break;
      }
      u += unit_step;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // Copies may be in flight whose barrier nobody has waited for (the producer's last ones are the MMA
    // issuer's to wait for): they land in microseconds; stay for two milliseconds.
    const uint64_t t_end = globaltimer() + 2000000ull;
    while (globaltimer() < t_end) __nanosleep(1000);
    if (warp >= 4) give_nan<kTok, kGlu, T>(p, tmem_slot + 5);
  }
  if (kSplit) cluster_sync();   // none leaves while another may still read its sums or signal it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kBufs * 2 * kTok);
  }
}

// ---------------------------------------------------------------- host side

// Row-major [outer, K] bytes, boxes of `rows` x 128, 128-byte swizzle.
bool make_map(CUtensorMap *m, const void *base, uint64_t K, uint64_t outer, uint32_t rows) {
  return encode_tmap_2d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, K, outer, kBK, rows,
                        CU_TENSOR_MAP_SWIZZLE_128B);
}

void launch_config(cudaLaunchConfig_t *cfg, cudaLaunchAttribute *attr, unsigned ctas, int cluster, int smem,
                   cudaStream_t s) {
  cfg->gridDim = dim3(ctas);
  cfg->blockDim = dim3(kThreads);
  cfg->dynamicSmemBytes = smem;
  cfg->stream = s;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg->attrs = attr;
  cfg->numAttrs = cluster > 1 ? 2 : 1;
}

template <int kTok, bool kGlu, class T, bool kSplit>
cudaError_t launch(const F8Args &a, cudaStream_t s) {
  constexpr int kSmemBytes = Shape<kTok, kSplit>::kSmemBytes;
  FewParams p;
  memset(&p, 0, sizeof(p));
  for (int i = 0; i < kBoxes && (16 << i) <= kTok; ++i)
    if (!make_map(&p.tmX[i], a.a, a.K, a.rows, 16u << i)) return cudaErrorInvalidValue;
  const uint64_t wrows = static_cast<uint64_t>(a.E) * a.N;
  if (!make_map(&p.tmW[0], a.b0, a.K, wrows, 128) || (kGlu && !make_map(&p.tmW[1], a.b1, a.K, wrows, 128)))
    return cudaErrorInvalidValue;
  p.edge = edge_rows(a.N);
  if (p.edge < 128 && !make_map(&p.tmW[2], a.b0, a.K, wrows, p.edge)) return cudaErrorInvalidValue;
  p.sa = a.sa;
  p.sb0 = a.sb0;
  p.sb1 = a.sb1;
  p.tiles = a.tiles;
  p.meta = a.meta;
  p.stats = a.stats;
  p.y = a.y;
  p.hq = a.hq;
  p.hs = a.hs;
  p.part = a.part;
  p.cnt = a.cnt;
  p.rows = a.rows;
  p.N = a.N;
  p.KB = (a.K + kBK - 1) / kBK;
  p.NB = (a.N + 127) / 128;
  p.early = a.early;
  p.hold = a.hold;
  p.wait_ns = a.wait_ns;
  const long long tiles = a.tiles != nullptr ? a.max_tiles : (a.rows + kTok - 1) / kTok;
  const long long units = tiles * (kGlu ? p.NB : (a.N + kRows - 1) / kRows);
  const int sms = a.n_sms < kF8Ctas ? a.n_sms : kF8Ctas;
  const void *kernel = reinterpret_cast<const void *>(f8_few_kernel<kTok, kGlu, T, kSplit>);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  static std::atomic<bool> seen{false};
  if (e == cudaSuccess) e = check_registers(kernel, &seen);
  if (e != cudaSuccess) return e;
  const long long most = (units * p.KB + kMinBlocks - 1) / kMinBlocks;
  const long long ctas = kSplit ? units * a.split : most < sms ? most : sms;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  launch_config(&cfg, attr, static_cast<unsigned>(ctas), kSplit ? a.split : 1, kSmemBytes, s);
  return cudaLaunchKernelEx(&cfg, f8_few_kernel<kTok, kGlu, T, kSplit>, p);
}

template <int kTok, bool kSplit>
cudaError_t launch_type(const F8Args &a, cudaStream_t s) {
  if (a.b1 != nullptr) return launch<kTok, true, float, kSplit>(a, s);
  if (a.y_dtype == XS_BF16) return launch<kTok, false, __nv_bfloat16, kSplit>(a, s);
  if (a.y_dtype == XS_F16) return launch<kTok, false, __half, kSplit>(a, s);
  return launch<kTok, false, float, kSplit>(a, s);
}

// Clusters of `size` CTAs that the current device runs at once, 0 if that cannot be found out
// (cached per device; host threads that race on it store the same value).
constexpr int kMostSplit = 8;
int resident_clusters(int size) {
  constexpr int kDevs = 64;
  static std::atomic<int> cache[kDevs][kMostSplit + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevs) return 0;
  int n = cache[dev][size].load(std::memory_order_relaxed);
  if (n > 0) return n;
  constexpr int kSmemBytes = Shape<32, true>::kSmemBytes;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  launch_config(&cfg, attr, size, size, kSmemBytes, nullptr);
  cfg.attrs = attr + 1;   // the cluster alone
  cfg.numAttrs = 1;
  // The query wants the shared-memory limit of the form it asks about.
  if (cudaFuncSetAttribute(reinterpret_cast<const void *>(f8_few_kernel<32, false, float, true>),
                           cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, f8_few_kernel<32, false, float, true>, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();  // a failed query leaves no sticky error
    return 0;
  }
  cache[dev][size].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace

int f8_split(int tile_tok, long long units, int K) {
  if (tile_tok != 32) return 1;
  const int KB = (K + kBK - 1) / kBK;
  for (int s = kMostSplit; s > 1; --s)
    if (KB / s >= kMinBlocks && units * s <= kF8Ctas && units <= resident_clusters(s)) return s;
  return 1;
}

cudaError_t launch_f8_few(const F8Args &a, cudaStream_t s) {
  if (a.tile_tok == 32) return a.split > 1 ? launch_type<32, true>(a, s) : launch_type<32, false>(a, s);
  return launch_type<64, false>(a, s);
}

size_t f8_part_bytes() { return static_cast<size_t>(kF8Ctas) * 2 * 64 * kRows * sizeof(float); }

}  // namespace xs
