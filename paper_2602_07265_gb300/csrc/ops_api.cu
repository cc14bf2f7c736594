// C ABI of the operators of xshare_ops.h: argument checks, workspace plans and
// launch sequences.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "ops_internal.cuh"

namespace xs {
namespace {

constexpr size_t kAlign = 256;
constexpr int kLeastTile = 32;   // rows of the smallest tile of the products
constexpr int kMaxDim = 1 << 20;
constexpr int kMaxMatrices = 1024;
constexpr long long kMaxWeightRows = 0x7fffffffll - 511;

// The current device's SM count, or a negative XS_ERR code (per device, filled
// on first use; host threads that race on it store the same value).
int ops_device_sms() {
  static std::atomic<int> cache[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return XS_ERR_CUDA;
  int v = cache[dev].load(std::memory_order_relaxed);
  if (v == 0) {
    int major = 0, minor = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return XS_ERR_CUDA;
    v = (major == 10 && minor == 3 && sms > 0) ? sms : XS_ERR_DEVICE;
    cache[dev].store(v, std::memory_order_relaxed);
  }
  return v;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <class... P>
bool all_aligned(const P *...p) {
  return (aligned16(p) && ...);
}
bool type_ok(int t) { return t == XS_F32 || t == XS_BF16 || t == XS_F16; }
int rc_of(cudaError_t e) { return e == cudaSuccess ? XS_OK : XS_ERR_CUDA; }
bool workspace_ok(const void *ws) { return ws != nullptr && reinterpret_cast<uintptr_t>(ws) % kAlign == 0; }

template <class T>
T *at(void *ws, size_t off) {
  return reinterpret_cast<T *>(static_cast<char *>(ws) + off);
}

struct Taker {
  size_t o = 0;
  size_t operator()(size_t bytes) {
    const size_t r = o;
    o = (o + bytes + kAlign - 1) / kAlign * kAlign;
    return r;
  }
};

// Tiles of `rows` rows over E experts at most.
int tiles_at_most(int rows, int E, int tile) {
  return E == 1 ? (rows + tile - 1) / tile : rows / tile + (E < rows ? E : rows);
}

// Where the permutation of P pairs over N experts keeps its parts.
struct PermPlan {
  size_t pos, cnt, first, meta, tiles;
  int max_tiles;
};
PermPlan perm_plan(Taker &take, int P, int N, bool with_tiles) {
  PermPlan pl;
  const size_t chunk_words = perm_chunks(P) > 1 ? static_cast<size_t>(perm_chunks(P)) * N : 0;
  pl.pos = take(static_cast<size_t>(P) * 4);
  pl.cnt = take(chunk_words * 4);
  pl.first = take(chunk_words * 4);
  pl.meta = take(sizeof(PermMeta));
  pl.max_tiles = with_tiles ? tiles_at_most(P, N, kLeastTile) : 0;
  pl.tiles = take(static_cast<size_t>(pl.max_tiles) * sizeof(Tile));
  return pl;
}
PermArgs perm_args(const PermPlan &pl, void *ws, const int32_t *ids, int P, int N) {
  PermArgs p;
  std::memset(&p, 0, sizeof(p));
  p.ids = ids;
  p.P = P;
  p.N = N;
  p.tile_tok = kLeastTile;
  p.pos = at<int32_t>(ws, pl.pos);
  p.cnt = at<int32_t>(ws, pl.cnt);
  p.first = at<int32_t>(ws, pl.first);
  p.meta = at<PermMeta>(ws, pl.meta);
  p.tiles = pl.max_tiles > 0 ? at<Tile>(ws, pl.tiles) : nullptr;
  return p;
}

int check_gate_shape(int B, int N, int k) {
  return B < 1 || B > kMaxB || N < 1 || N > kMaxN || k < 1 || k > kMaxK || k > N ? XS_ERR_SHAPE : XS_OK;
}

// The form of a float8 product for `rows` rows over several matrices, by rows per matrix: what
// the form for few reads of the weights again for every 32 or 64 rows, and what CTA pairs
// lose on tiles that are not full.  Tiles of 32 | 64 | pairs, us:
// (All slots count as rows and all experts as matrices, since the host knows no more.  Where the ids keep to a
// selection of the experts, the rows of a used one are more than this says: 512 tokens of 8 in 44 of 256
// experts have 93 each and take tiles of 32, by the lines below 1.6 times the best.  On a rank that holds some of the
// experts they are fewer.)
//   experts d = 2048, F = 768, 128 experts: 16 rows each 121 | 122 | 180, 32 147 | 133 | 185,
//   48 208 | 143 | 190, 64 228 | 195 | 192, 96 330 | 262 | 201;
//   experts d = 2048, F = 1024, 64 experts: 8 88 | 89 | 120, 32 110 | 107 | 125, 64 144 | 139 | 129;
//   64 products 2048 x 1024: 8 32 | 33 | 39, 32 37 | 41 | 41, 64 45 | 51 | 47, 100 70 | 50 | 54.
int tile_of(long long rows, int matrices) {
  if (rows > static_cast<long long>(matrices) * kF8FewTile) return kF8PairTile;
  return rows > static_cast<long long>(matrices) * 24 ? kF8FewTile : kLeastTile;
}

// The form of one float8 product, whose units may be fewer than the SMs: CTA pairs take
// whole units, the form for few shares a unit's K blocks in a cluster as long as all units
// find one at once, else among all CTAs, at a price for joining them.  In us, from these figures
// (few | pairs): clusters: N = 4096, K = 7168: M = 1 9.0 | 29, 32 12 | 29, 128 17 | 31; N = 7168, K = 2048:
// M = 1 7.2 | 11, 64 9.1 | 11; N = K = 1024: M = 32 7.5 | 7.0; N = 1024, K = 4096: M = 512 12 | 20;
// whole units: N = 4096, K = 7168: M = 256 31 | 31, 512 50 | 31; N = 7168, K = 2048: M = 128 12 | 12, 256 22 | 12;
// shared among all: N = 32768, K = 7168: M = 1 41 | 58, 32 44 | 59.
// Several matrices (tiles of 32 in clusters | of 64 | pairs): 2 of 1024 x 4096, 200 rows 12 | 25 | 21; 8 of 512 x
// 2048, 64 rows 9.3 | 11 | 13, 300 rows 11 | 17 | 13; where the units find no cluster tile_of() decides.
int tile_of_product(int M, int N, int K, int E) {
  const int KB = (K + 127) / 128;
  const long long columns = (N + 255) / 256, units = tiles_at_most(M, E, kLeastTile) * columns;
  const long long pair_units = tiles_at_most(M, E, kF8PairTile) * columns;
  const int split = f8_split(kLeastTile, units, K);
  if (split == 1 && E > 1) return tile_of(M, E);
  const double pairs = 3.5 + 0.46 * KB * static_cast<double>((pair_units + kF8Ctas / 2 - 1) / (kF8Ctas / 2));
  const double whole = static_cast<double>((units + kF8Ctas - 1) / kF8Ctas) * KB;
  const double share = std::max(2.0, static_cast<double>(units) * KB / kF8Ctas);
  const int part = (KB + split - 1) / split;
  const double few = split > 1 ? (M <= 8 * E ? 4.8 + 0.45 * part : 6.2 + 0.35 * (part + split))
                     : whole - share >= kF8CutBlocks ? 8.5 + 0.55 * share : 3.5 + 0.55 * whole;
  return few <= pairs ? kLeastTile : kF8PairTile;
}

struct MatmulPlan {
  size_t meta, tiles, cnt, part, total;
  int max_tiles;
};
int check_matmul_shape(int M, int N, int K, int E) {
  if (M < 1 || M > kMaxDim || N < 1 || N > kMaxDim || K < 16 || K > kMaxDim || K % 16 != 0 || E < 1 ||
      E > kMaxMatrices || static_cast<long long>(E) * N > kMaxWeightRows)
    return XS_ERR_SHAPE;
  return XS_OK;
}
MatmulPlan matmul_plan(int M, int E) {
  MatmulPlan pl;
  Taker take;
  // The parts of every form, so that a workspace serves fewer rows too.
  pl.max_tiles = tiles_at_most(M, E, kLeastTile);
  pl.meta = take(sizeof(PermMeta));
  pl.tiles = take(static_cast<size_t>(pl.max_tiles) * sizeof(Tile));
  pl.cnt = take(kF8Ctas * 4);
  pl.part = take(f8_part_bytes());
  pl.total = take.o;
  return pl;
}

struct ExpertsPlan {
  PermPlan perm;
  size_t cnt, part, rows, xq, xs, hq, hs, out, inv, total;
  int tile_tok;
};
int check_experts_shape(int B, int N, int k, int d, int F) {
  if (B < 1 || B > kMaxB || N < 1 || N > kMaxMatrices || k < 1 || k > kMaxSlots || d < 128 || d > kMaxDim ||
      d % 128 != 0 || F < 128 || F > kMaxDim || F % 128 != 0 ||
      static_cast<long long>(N) * (d > F ? d : F) > kMaxWeightRows)
    return XS_ERR_SHAPE;
  return XS_OK;
}
ExpertsPlan experts_plan(int B, int N, int k, int d, int F) {
  ExpertsPlan pl;
  Taker take;
  const size_t rows = static_cast<size_t>(B) * k;
  pl.tile_tok = tile_of(B * k, N);
  pl.perm = perm_plan(take, B * k, N, true);
  pl.cnt = take(2 * kF8Ctas * 4);   // the parts of every form, so that a workspace serves fewer tokens too
  pl.part = take(f8_part_bytes());
  pl.rows = take(rows * 4);
  pl.xq = take(rows * d);
  pl.xs = take(rows * (d / 128) * 4);
  pl.hq = take(rows * F);
  pl.hs = take(rows * (F / 128) * 4);
  // Expert outputs: fp32 in the form for few rows, fp16 and factors on pairs.
  const size_t few = static_cast<size_t>(N) * kF8FewTile;
  pl.out = take(std::max(rows * d * 2, std::min(rows, few) * d * 4));
  pl.inv = take(rows * (d / 64) * 4);
  pl.total = take.o;
  return pl;
}

}  // namespace
}  // namespace xs

using namespace xs;

extern "C" size_t xshare_gate_workspace_size(int B, int N, int k) {
  if (check_gate_shape(B, N, k) != XS_OK) return 0;
  Taker take;
  perm_plan(take, B * k, N, false);
  return take.o;
}

extern "C" int xshare_gate(const void *logits, int dtype, const float *bias, const uint8_t *expert_mask,
                           const uint8_t *token_mask, int B, int N, int k, const xs_gate_params *prm,
                           int32_t *topk_ids, float *topk_w, float *scores_out, int32_t *expert_counts,
                           int32_t *expert_offsets, int32_t *perm, void *workspace, size_t ws_bytes,
                           xs_stream_t stream) {
  if (prm == nullptr) return XS_ERR_NULL;
  const int rc = check_gate_shape(B, N, k);
  if (rc != XS_OK) return rc;
  if (!type_ok(dtype) || (prm->scoring != XS_SCORE_SOFTMAX && prm->scoring != XS_SCORE_SIGMOID) ||
      prm->n_groups < 1 || prm->n_groups > 32 || N % prm->n_groups != 0 || prm->top_groups < 1 ||
      prm->top_groups > prm->n_groups || (prm->group_top != 1 && prm->group_top != 2) ||
      (prm->renorm != 0 && prm->renorm != 1) || !std::isfinite(prm->scale))
    return XS_ERR_PARAM;
  if (!logits || !topk_ids || !topk_w) return XS_ERR_NULL;
  if (!all_aligned(logits, bias, expert_mask, token_mask, topk_ids, topk_w, scores_out, expert_counts,
                   expert_offsets, perm))
    return XS_ERR_ALIGN;
  const bool permute = expert_counts || expert_offsets || perm;
  if (permute && (!workspace_ok(workspace) || ws_bytes < xshare_gate_workspace_size(B, N, k)))
    return XS_ERR_WORKSPACE;
  const int sms = ops_device_sms();
  if (sms < 0) return sms;
  GateArgs a;
  a.logits = logits;
  a.bias = bias;
  a.expert_mask = expert_mask;
  a.token_mask = token_mask;
  a.B = B;
  a.N = N;
  a.k = k;
  a.prm = *prm;
  a.ids = topk_ids;
  a.w = topk_w;
  a.scores = scores_out;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (launch_gate(a, dtype, s) != cudaSuccess) return XS_ERR_CUDA;
  if (!permute) return XS_OK;
  Taker take;
  const PermPlan pl = perm_plan(take, B * k, N, false);
  PermArgs p = perm_args(pl, workspace, topk_ids, B * k, N);
  p.counts_out = expert_counts;
  p.offsets_out = expert_offsets;
  p.perm_out = perm;
  return rc_of(launch_permute(p, s));
}

extern "C" int xshare_quant_fp8_rows(const void *x, int dtype, int M, int K, uint8_t *q, float *scales,
                                     xs_stream_t stream) {
  if (M < 1 || M > kMaxDim || K < 1 || K > kMaxDim) return XS_ERR_SHAPE;
  if (!type_ok(dtype)) return XS_ERR_PARAM;
  if (!x || !q || !scales) return XS_ERR_NULL;
  if (!all_aligned(x, q, scales)) return XS_ERR_ALIGN;
  const int sms = ops_device_sms();
  if (sms < 0) return sms;
  return rc_of(launch_quant_rows(x, dtype, M, K, q, scales, reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" int xshare_quant_fp8_blocks(const void *x, int dtype, int n, int R, int K, uint8_t *q, float *scales,
                                       xs_stream_t stream) {
  if (n < 1 || n > kMaxMatrices || R < 1 || R > kMaxDim || K < 1 || K > kMaxDim ||
      static_cast<long long>(n) * ((R + 127) / 128) * ((K + 127) / 128) > kMaxWeightRows)
    return XS_ERR_SHAPE;
  if (!type_ok(dtype)) return XS_ERR_PARAM;
  if (!x || !q || !scales) return XS_ERR_NULL;
  if (!all_aligned(x, q, scales)) return XS_ERR_ALIGN;
  const int sms = ops_device_sms();
  if (sms < 0) return sms;
  return rc_of(launch_quant_blocks(x, dtype, n, R, K, q, scales, sms, reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" size_t xshare_matmul_fp8_workspace_size(int M, int N, int K, int E) {
  if (check_matmul_shape(M, N, K, E) != XS_OK) return 0;
  return matmul_plan(M, E).total;
}

extern "C" int xshare_matmul_fp8(const uint8_t *a, const float *a_scale, const uint8_t *b, const float *b_scale,
                                 const int32_t *offsets, int M, int N, int K, int E, void *y, int y_dtype,
                                 xs_stats *stats, void *workspace, size_t ws_bytes, xs_stream_t stream) {
  const int rc = check_matmul_shape(M, N, K, E);
  if (rc != XS_OK) return rc;
  if (offsets == nullptr && E != 1) return XS_ERR_NULL;
  if (!type_ok(y_dtype)) return XS_ERR_PARAM;
  if (!a || !a_scale || !b || !b_scale || !y) return XS_ERR_NULL;
  if (!all_aligned(a, a_scale, b, b_scale, offsets, y, stats)) return XS_ERR_ALIGN;
  const MatmulPlan pl = matmul_plan(M, E);
  if (!workspace_ok(workspace) || ws_bytes < pl.total) return XS_ERR_WORKSPACE;
  const int sms = ops_device_sms();
  if (sms < 0) return sms;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  F8Args f;
  std::memset(&f, 0, sizeof(f));
  f.a = a;
  f.sa = a_scale;
  f.b0 = b;
  f.sb0 = b_scale;
  f.rows = M;
  f.N = N;
  f.K = K;
  f.E = E;
  f.y = y;
  f.y_dtype = y_dtype;
  f.stats = stats;
  f.n_sms = sms;
  f.tile_tok = tile_of_product(M, N, K, E);
  f.split = f8_split(f.tile_tok, pl.max_tiles * ((N + 255ll) / 256), K);
  const bool joins = f.tile_tok != kF8PairTile && f.split == 1;
  f.cnt = joins ? at<int32_t>(workspace, pl.cnt) : nullptr;
  f.part = at<float>(workspace, pl.part);
  if (offsets != nullptr) {
    f.tiles = at<Tile>(workspace, pl.tiles);
    f.meta = at<PermMeta>(workspace, pl.meta);
    f.max_tiles = pl.max_tiles;
    if (launch_offset_tiles(offsets, E, M, f.tile_tok, at<Tile>(workspace, pl.tiles), f.meta, stats, f.cnt, kF8Ctas,
                            s) != cudaSuccess)
      return XS_ERR_CUDA;
  } else if (f.cnt != nullptr || stats != nullptr) {
    if (launch_zero(f.cnt, kF8Ctas, stats, s) != cudaSuccess) return XS_ERR_CUDA;
    f.early = true;   // the operands do not come from that kernel
  }
  return rc_of(launch_f8(f, s));
}

extern "C" size_t xshare_experts_fp8_workspace_size(int B, int N, int k, int d, int F) {
  if (check_experts_shape(B, N, k, d, F) != XS_OK) return 0;
  return experts_plan(B, N, k, d, F).total;
}

extern "C" int xshare_experts_fp8(const uint16_t *x, const int32_t *topk_ids, const float *topk_w,
                                  const xs_fp8_experts *experts, int B, int k, int d, int F, uint16_t *y,
                                  xs_stats *stats, void *workspace, size_t ws_bytes, xs_stream_t stream) {
  if (experts == nullptr) return XS_ERR_NULL;
  const int N = experts->n;
  const int rc = check_experts_shape(B, N, k, d, F);
  if (rc != XS_OK) return rc;
  if (!x || !topk_ids || !topk_w || !y || !experts->gate || !experts->up || !experts->down || !experts->gate_s ||
      !experts->up_s || !experts->down_s)
    return XS_ERR_NULL;
  if (!all_aligned(x, topk_ids, topk_w, y, stats, experts->gate, experts->up, experts->down, experts->gate_s,
                   experts->up_s, experts->down_s))
    return XS_ERR_ALIGN;
  const ExpertsPlan pl = experts_plan(B, N, k, d, F);
  if (!workspace_ok(workspace) || ws_bytes < pl.total) return XS_ERR_WORKSPACE;
  const int sms = ops_device_sms();
  if (sms < 0) return sms;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);

  PermArgs p = perm_args(pl.perm, workspace, topk_ids, B * k, N);
  p.stats = stats;
  p.tile_tok = pl.tile_tok;
  const bool few = pl.tile_tok != kF8PairTile;
  p.zero = few ? at<int32_t>(workspace, pl.cnt) : nullptr;
  p.zero_n = 2 * kF8Ctas;
  const bool one_kernel = perm_chunks(B * k) == 1;
  TokenArgs t;
  t.x = x;
  t.ids = topk_ids;
  t.pos = p.pos;
  t.first = p.first;
  t.rows = at<int32_t>(workspace, pl.rows);
  t.q = at<uint8_t>(workspace, pl.xq);
  t.scales = at<float>(workspace, pl.xs);
  t.B = B;
  t.k = k;
  t.d = d;
  t.N = N;
  if (one_kernel ? launch_quant_routed(t, p, s) != cudaSuccess
                 : launch_permute(p, s) != cudaSuccess || launch_quant_tokens(t, s) != cudaSuccess)
    return XS_ERR_CUDA;

  F8Args f;
  std::memset(&f, 0, sizeof(f));
  f.a = t.q;
  f.sa = t.scales;
  f.b0 = experts->gate;
  f.b1 = experts->up;
  f.sb0 = experts->gate_s;
  f.sb1 = experts->up_s;
  f.rows = B * k;
  f.N = F;
  f.K = d;
  f.E = N;
  f.tiles = p.tiles;
  f.meta = p.meta;
  f.max_tiles = pl.perm.max_tiles;
  f.early = !one_kernel;   // else the tiles come from the kernel before
  f.hq = at<uint8_t>(workspace, pl.hq);
  f.hs = at<float>(workspace, pl.hs);
  f.stats = stats;
  f.n_sms = sms;
  f.tile_tok = pl.tile_tok;
  f.split = f8_split(f.tile_tok, static_cast<long long>(pl.perm.max_tiles) * (F / 128), d);
  f.cnt = p.zero;
  f.part = at<float>(workspace, pl.part);
  if (launch_f8(f, s) != cudaSuccess) return XS_ERR_CUDA;
  f.a = f.hq;
  f.sa = f.hs;
  f.b0 = experts->down;
  f.b1 = nullptr;
  f.sb0 = experts->down_s;
  f.sb1 = nullptr;
  f.N = d;
  f.K = F;
  f.early = true;
  f.split = f8_split(f.tile_tok, static_cast<long long>(pl.perm.max_tiles) * ((d + 255) / 256), F);
  f.y = at<void>(workspace, pl.out);
  f.y_dtype = few ? XS_F32 : XS_F16;
  f.inv = few ? nullptr : at<float>(workspace, pl.inv);
  if (few) f.cnt = p.zero + kF8Ctas;
  if (launch_f8(f, s) != cudaSuccess) return XS_ERR_CUDA;

  CombineArgs c;
  c.out = at<void>(workspace, pl.out);
  c.inv = f.inv;
  c.rows = t.rows;
  c.w = topk_w;
  c.y = y;
  c.B = B;
  c.k = k;
  c.d = d;
  return rc_of(launch_combine_f8(c, s));
}
