"""Waits that run out inside the float8 products, without a GPU fault.

One CTA has a barrier that waits for one arrival too many; after a limit of 20 ms the kernel
gives up by its own way out.  The call has to report it, and the next call on
the same workspace has to be right.
"""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
WAIT_NS = 20_000_000
OK, TIMEOUT = 0, 1


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2602_07265_gb300 import _build
    _build.build()
    from paper_2602_07265_gb300 import ops
    ops.LIB.xshare_selftest_f8_hold.argtypes = [ctypes.c_int, ctypes.c_uint32, ctypes.c_uint64]
    return ops


def hold(ops, launches, block):
    assert ops.LIB.xshare_selftest_f8_hold(launches, block, WAIT_NS) == 0


def randn(*shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn(*shape, generator=g)).to(torch.bfloat16).to(DEV)


def rows_of(ops, x):
    q = torch.empty(x.shape, dtype=ops.FP8, device=DEV)
    s = torch.empty(x.shape[0], -(-x.shape[1] // 128), device=DEV)
    ops.xshare_quant_fp8_rows(x, q, s)
    return q, s


def blocks_of(ops, w):
    q = torch.empty(w.shape, dtype=ops.FP8, device=DEV)
    s = torch.empty(*w.shape[:-2], -(-w.shape[-2] // 128), -(-w.shape[-1] // 128), device=DEV)
    ops.xshare_quant_fp8_blocks(w, q, s)
    return q, s


# Rows, columns, K, matrices, and the K block of CTA 0 that never becomes full (one of the first
# that the ring holds: four with tiles of 64, else five or six).
PRODUCTS = [(3, 1000, 2048, 1, 0), (20, 512, 2048, 1, 1),          # a cluster for every unit
            (1, 32768, 7168, 1, 3), (8, 32768, 7168, 1, 4),       # units cut between CTAs
            (320, 4096, 512, 8, 0), (320, 4096, 640, 8, 3),        # whole units, tiles of 64
            (190, 9000, 256, 8, 1),                                # and of 32
            (600, 1000, 640, 1, 2), (300, 4096, 384, 1, 0), (1500, 1040, 512, 3, 3)]   # CTA pairs


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K,E,block", PRODUCTS)
def test_product_reports_and_the_next_is_right(ops, M, N, K, E, block, dtype):
    q, s = rows_of(ops, randn(M, K, seed=1))
    w, ws = blocks_of(ops, randn(E, N, K, seed=2, std=0.02))
    off = torch.linspace(0, M, E + 1).int().to(DEV) if E > 1 else None
    work = torch.empty(ops.xshare_matmul_fp8_workspace_size(M, N, K, E), dtype=torch.uint8, device=DEV)
    st = torch.full((8,), -1, dtype=torch.int32, device=DEV)
    want, y = torch.empty(M, N, dtype=dtype, device=DEV), torch.empty(M, N, dtype=dtype, device=DEV)
    ops.xshare_matmul_fp8(q, s, w, ws, want, work, offsets=off, stats=st)
    assert st[5].item() == OK
    hold(ops, 0, block)
    ops.xshare_matmul_fp8(q, s, w, ws, y, work, offsets=off, stats=st)
    assert st[5].item() == TIMEOUT
    ops.xshare_matmul_fp8(q, s, w, ws, y, work, offsets=off, stats=st)
    assert st[5].item() == OK and torch.equal(y, want)


# Tokens, experts, slots, d, F: tiles of 32 in clusters and cut, of 64, CTA pairs.
EXPERTS = [(1, 8, 2, 1024, 512), (4, 64, 8, 2048, 1024), (40, 4, 4, 256, 256), (200, 2, 2, 256, 256)]


@pytest.mark.parametrize("which", [0, 1])   # gate and up, down
@pytest.mark.parametrize("B,n,k,d,F", EXPERTS)
def test_experts_report_and_the_next_are_right(ops, B, n, k, d, F, which):
    ex = ops.Fp8Experts.quantise(randn(n, F, d, seed=3, std=0.05), randn(n, F, d, seed=4, std=0.05),
                                 randn(n, d, F, seed=5, std=0.05))
    x = randn(B, d, seed=6)
    ids = torch.rand(B, n, generator=torch.Generator().manual_seed(7)).argsort(1)[:, :k].int().contiguous().to(DEV)
    w = torch.full((B, k), 1.0 / k, device=DEV)
    work = torch.empty(ops.xshare_experts_fp8_workspace_size(B, n, k, d, F), dtype=torch.uint8, device=DEV)
    st = torch.full((8,), -1, dtype=torch.int32, device=DEV)
    want, y = torch.empty_like(x), torch.empty_like(x)
    ops.xshare_experts_fp8(x, ids, w, ex, want, work, stats=st)
    assert st[5].item() == OK
    hold(ops, which, 1)
    ops.xshare_experts_fp8(x, ids, w, ex, y, work, stats=st)
    assert st[5].item() == TIMEOUT
    ops.xshare_experts_fp8(x, ids, w, ex, y, work, stats=st)
    assert st[5].item() == OK and torch.equal(y, want)


def owed(y, want):
    """Elements that are NaN; all others have to be those of a whole call."""
    gone = torch.isnan(y)
    assert gone.any() and torch.equal(torch.where(gone, want, y), want)
    return gone


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("stats", [False, True])
@pytest.mark.parametrize("M,N,K,E,block", PRODUCTS)
def test_what_a_product_could_not_finish_is_nan(ops, M, N, K, E, block, stats, dtype):
    """With and without statistics: no element keeps what the buffer held before."""
    q, s = rows_of(ops, randn(M, K, seed=11))
    w, ws = blocks_of(ops, randn(E, N, K, seed=12, std=0.02))
    off = torch.linspace(0, M, E + 1).int().to(DEV) if E > 1 else None
    work = torch.empty(ops.xshare_matmul_fp8_workspace_size(M, N, K, E), dtype=torch.uint8, device=DEV)
    st = torch.zeros(8, dtype=torch.int32, device=DEV) if stats else None
    want, y = torch.empty(M, N, dtype=dtype, device=DEV), torch.full((M, N), 333.0, dtype=dtype, device=DEV)
    ops.xshare_matmul_fp8(q, s, w, ws, want, work, offsets=off, stats=st)
    assert not torch.isnan(want).any()
    hold(ops, 0, block)
    ops.xshare_matmul_fp8(q, s, w, ws, y, work, offsets=off, stats=st)
    owed(y, want)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("B,n,k,d,F", EXPERTS)
def test_what_the_experts_could_not_finish_is_nan(ops, B, n, k, d, F, which):
    ex = ops.Fp8Experts.quantise(randn(n, F, d, seed=13, std=0.05), randn(n, F, d, seed=14, std=0.05),
                                 randn(n, d, F, seed=15, std=0.05))
    x = randn(B, d, seed=16)
    ids = torch.rand(B, n, generator=torch.Generator().manual_seed(17)).argsort(1)[:, :k].int().contiguous().to(DEV)
    w = torch.full((B, k), 1.0 / k, device=DEV)
    work = torch.empty(ops.xshare_experts_fp8_workspace_size(B, n, k, d, F), dtype=torch.uint8, device=DEV)
    want, y = torch.empty_like(x), torch.full_like(x, 333.0)
    ops.xshare_experts_fp8(x, ids, w, ex, want, work)
    hold(ops, which, 1)
    ops.xshare_experts_fp8(x, ids, w, ex, y, work)
    gone = owed(y, want)
    if which == 0:   # an activation that is missing takes the token's whole row with it
        assert torch.equal(gone.any(1), gone.all(1))
