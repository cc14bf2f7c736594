"""Float8 operators at the sizes they are made for: thousands of rows, experts of full size in a
selection, and more elements than 32 bits count.  Parts of the results are compared with the
plain 64-bit forms, within the bounds of test_gpu_fp8.py."""
import numpy as np
import pytest
import torch

import ops_reference as R
import test_gpu_fp8 as F8

pytestmark = pytest.mark.gpu
DEV = "cuda"
cpu = F8.cpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2602_07265_gb300 import _build
    _build.build()
    from paper_2602_07265_gb300 import ops
    return ops


def weights(n, r, K, seed):
    """Random e4m3 values (no NaN) and scales, made on the GPU: as many as the memory holds."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.empty(n, r, K, dtype=torch.uint8, device=DEV)
    for e in range(n):
        q[e].random_(0, 127, generator=g)
        q[e] += 128 * (q[e] & 1)   # signs
    s = (0.5 + torch.rand(n, -(-r // 128), -(-K // 128), generator=g, device=DEV)) * 2e-4
    return q.view(torch.float8_e4m3fn), s


def tokens(M, K, seed, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(M, K, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def check_rows(y, q, s, w, ws, rows, cols, dtype):
    """The listed rows of a product with one matrix, at the listed blocks of 128 columns."""
    c = torch.cat([torch.arange(128 * b, min(128 * b + 128, w.shape[0])) for b in cols])
    d = c.to(DEV)
    # Columns of a block keep their scale: a matrix of whole blocks, the last one perhaps shorter.
    ref, bound = F8.product_bound(cpu(q[rows]), cpu(s[rows]), cpu(w[d]), cpu(ws[torch.tensor(cols, device=DEV)]), dtype)
    got = cpu(y[rows][:, d])
    assert np.all(np.abs(got - ref) <= bound), (np.abs(got - ref) / bound).max()


@pytest.mark.parametrize("M,N,K,dtype", [(8192, 4096, 7168, torch.bfloat16), (5001, 1024, 2064, torch.float32),
                                         (1 << 20, 24, 16, torch.float32), (3, 1 << 20, 16, torch.float32),
                                         (2, 16, 1 << 20, torch.float32), (20011, 136, 272, torch.float16)])
def test_products_of_many(ops, M, N, K, dtype):
    q, s = F8.rows_of(ops, tokens(M, K, 1))
    (w, ws) = (t[0] for t in weights(1, N, K, 2))
    y = F8.matmul(ops, q, s, w, ws, dtype, fill=float("nan"))
    assert torch.isfinite(y).all()
    rows = torch.tensor(sorted({0, M // 3, M // 2, M - 2 if M > 1 else 0, M - 1}), device=DEV)
    NB = -(-N // 128)
    check_rows(y, q, s, w, ws, rows, sorted({0, NB // 2, NB - 1}), dtype)


def test_more_elements_than_32_bits_count(ops):
    """Rows, quantised rows and outputs beyond 2^31 elements each."""
    M, K, N = 300_000, 8192, 8192
    x = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    for i in range(0, M, 50_000):
        x[i:i + 50_000] = tokens(50_000, K, 10 + i)
    q, s = F8.rows_of(ops, x)
    rows = torch.tensor([0, 150_001, 262_143, 262_144, 262_145, M - 1], device=DEV)
    rq, rs = R.quant(cpu(x[rows]), 1)
    assert np.array_equal(cpu(s[rows]).astype(np.float32), rs) and np.array_equal(cpu(q[rows]), rq)
    wq, wqs = F8.blocks_of(ops, x)   # as one matrix
    for b in (0, 2047, M // 128):
        lo = 128 * b
        rq, rs = R.quant(cpu(x[lo:lo + 128]), 128)
        assert np.array_equal(cpu(wqs[b:b + 1]).astype(np.float32), rs) and np.array_equal(cpu(wq[lo:lo + 128]), rq)
    del x, wq, wqs
    w, ws = (t[0] for t in weights(1, N, K, 3))
    y = F8.matmul(ops, q, s, w, ws, torch.bfloat16, fill=float("nan"))
    check_rows(y, q, s, w, ws, rows, [0, 31, 63], torch.bfloat16)
    assert not torch.isnan(y[::997]).any()


@pytest.mark.parametrize("rows", [2, 90, 700])   # tiles of 32, of 64, CTA pairs
def test_weights_beyond_32_bits(ops, rows):
    """Products with the last of matrices that hold 2.7e9 elements together."""
    E, N, K = 40, 4096, 16384
    w, ws = weights(E, N, K, 4)
    used = (0, 20, 32, 38, 39)       # matrix 32 begins at 2^31
    count = np.zeros(E, np.int32)
    count[list(used)] = rows
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(count)]).astype(np.int32)).to(DEV)
    M = int(off[-1])
    q, s = F8.rows_of(ops, tokens(M, K, 5))
    y = F8.matmul(ops, q, s, w, ws, torch.float32, off, fill=float("nan"))
    assert torch.isfinite(y).all()
    for e in used:
        lo = int(off[e])
        check_rows(y, q, s, w[e], ws[e], torch.tensor([lo, lo + rows // 2, lo + rows - 1], device=DEV), [0, 17, 31],
                   torch.float32)


def test_the_most_weight_rows(ops):
    """1024 matrices of 2^20 rows."""
    E, N, K = 1024, 1 << 20, 16
    w, ws = weights(E, N, K, 6)
    off = torch.tensor([0] * 513 + [1] * 511 + [3], dtype=torch.int32, device=DEV)
    q, s = F8.rows_of(ops, tokens(3, K, 7))
    y = F8.matmul(ops, q, s, w, ws, torch.float32, off, fill=float("nan"))
    assert torch.isfinite(y).all()
    for r, e in ((0, 512), (1, 1023), (2, 1023)):
        check_rows(y, q, s, w[e], ws[e], torch.tensor([r], device=DEV), [0, 4095, 8191], torch.float32)


# Tokens, experts, slots, d, F.  The permutation kernels (more than 1024 pairs) with tiles of 32 and of 64
# and with pairs, up to the most tokens and slots.
@pytest.mark.parametrize("B,n,k,d,F,unused", [(256, 256, 8, 256, 128, 0), (256, 250, 8, 384, 256, 0.3), (1000, 300, 6, 128, 256, 0),
                                              (700, 120, 4, 256, 128, 0.1), (8192, 64, 8, 256, 128, 0.05),
                                              (8192, 1024, 3, 128, 128, 0), (2048, 40, 32, 128, 128, 0.2), (8192, 33, 32, 128, 128, 0.5)])
def test_experts_of_many_tokens(ops, B, n, k, d, F, unused):
    ex = F8.experts_of(ops, n, d, F, 30)
    x = F8.randn(B, d, seed=31, dtype=torch.bfloat16)
    ids, w = F8.routed(B, n, k, 32, unused)
    st = torch.full((8,), -1, dtype=torch.int32, device=DEV)
    y = F8.run_experts(ops, x, ids, w, ex, st)
    i = ids.cpu().numpy()
    ref, bound = F8.experts_bound(cpu(x), i, cpu(w), *F8.parts(ex))
    assert np.all(np.abs(cpu(y) - ref) <= bound)
    assert st.tolist() == [0, len(np.unique(i[i >= 0])), 0, 0, int((i >= 0).sum()), 0, 0, 0]


@pytest.mark.parametrize("B,live", [(256, 58), (512, 44)])
def test_a_selection_of_many_experts(ops, B, live):
    """Tokens that are routed inside a selection: most experts have no row, the others 35 and more."""
    n, k, d, F = 256, 8, 512, 256
    ex = F8.experts_of(ops, n, d, F, 40)
    x = F8.randn(B, d, seed=41, dtype=torch.bfloat16)
    inside = torch.randperm(n, generator=torch.Generator().manual_seed(42))[:live].int().to(DEV)
    ids, w = F8.routed(B, live, k, 43)
    ids = inside[ids.long()].contiguous()
    y = F8.run_experts(ops, x, ids, w, ex)
    ref, bound = F8.experts_bound(cpu(x), ids.cpu().numpy(), cpu(w), *F8.parts(ex))
    assert np.all(np.abs(cpu(y) - ref) <= bound)


@pytest.mark.parametrize("B,outside", [(64, 0.875), (2048, 0.875)])
def test_a_ranks_share(ops, B, outside):
    """Most ids outside the rank's experts: below 0, or from n on."""
    n, k, d, F = 32, 8, 256, 256
    ex = F8.experts_of(ops, n, d, F, 50)
    x = F8.randn(B, d, seed=51, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(52)
    ids, w = F8.routed(B, n, k, 53)
    gone = torch.rand(B, k, generator=g) < outside
    far = torch.randint(n, 256, (B, k), generator=g, dtype=torch.int32)
    far[::2] = -far[::2]
    ids = torch.where(gone.to(DEV), far.to(DEV), ids).contiguous()
    y = F8.run_experts(ops, x, ids, w, ex)
    i = ids.cpu().numpy()
    i = np.where((i >= 0) & (i < n), i, -1)
    ref, bound = F8.experts_bound(cpu(x), i, np.where(i >= 0, cpu(w), 0), *F8.parts(ex))
    assert np.all(np.abs(cpu(y) - ref) <= bound)


@pytest.mark.parametrize("B", [1, 9, 200])
def test_experts_of_full_size(ops, B):
    """256 experts of 7168 x 2048, 3.8e9 elements in each of the three matrices, tokens on the last ones; 200 tokens have
    the experts' 67 rows each and still tiles of 32."""
    n, k, d, F, used = 256, 1, 7168, 2048, (0, 254, 255)
    parts = []
    for i, (r, K) in enumerate(((F, d), (F, d), (d, F))):
        parts += weights(n, r, K, 60 + i)
    ex = ops.Fp8Experts(*parts)
    x = tokens(B, d, 63)
    ids = torch.tensor([used[t % 3] if B > 1 else 255 for t in range(B)], dtype=torch.int32, device=DEV).view(B, 1)
    w = torch.full((B, 1), 0.75, device=DEV)
    y = F8.run_experts(ops, x, ids, w, ex)
    few = torch.tensor([t for t in range(B) if t < 3 or t >= B - 3], device=DEV)
    pick = torch.tensor(used, device=DEV)
    sub = [(parts[2 * i].view(torch.uint8)[pick].view(torch.float8_e4m3fn), parts[2 * i + 1][pick]) for i in range(3)]
    local = np.array([used.index(e) for e in ids[few].view(-1).tolist()])[:, None]
    ref, bound = F8.experts_bound(cpu(x[few]), local, cpu(w[few]), *((cpu(q), cpu(s)) for q, s in sub))
    err = np.abs(cpu(y[few]) - ref)
    assert np.all(err <= bound), (err / bound).max()
    assert np.linalg.norm(cpu(y[few]) - ref) <= 1e-2 * np.linalg.norm(ref)
    assert torch.isfinite(y).all()
