"""Float8 operators on inputs whose results are known to the bit."""
import numpy as np
import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2602_07265_gb300 import _build
    _build.build()
    from paper_2602_07265_gb300 import ops
    return ops


def fp8(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.float8_e4m3fn).to(DEV)


@pytest.mark.parametrize("B", [1, 3, 30, 60, 300])   # tiles of 32, of 64, CTA pairs
def test_activations_on_the_border_of_two_values(ops, B):
    """h = 64 u with whole u whose quotient by the block's scale is the middle of two e4m3
    values, for scales whose reciprocal is off enough that a product with it would fall
    on the other side.  All sums are exact: silu(64) = 64, e^-64 being below half an ulp of 1."""
    d, scales = 128, (7, 13, 15, 41, 47, 51, 55, 61)
    F = 128 * len(scales)
    mids = [2.0 ** e * (1 + (2 * i + 1) / 16) for e in range(2, 8) for i in range(8)]
    u = np.zeros(F)
    for b, t in enumerate(scales):   # the first hidden unit of a block has its largest value
        v = np.array([448] + [m for m in mids if m <= 440 and float(m * t).is_integer()]) * t
        u[128 * b:128 * b + len(v)] = v
    # u = sum over columns of 256 or powers of two in x and digits 0 .. 15 in the weights.
    x = np.zeros(d)
    x[0], x[1:13], x[13:21], x[21] = 448, 256, 2.0 ** np.arange(8), 64
    up, gate, down = np.zeros((F, d)), np.zeros((F, d)), np.zeros((d, F))
    high, low = (u // 256).astype(int), (u % 256).astype(int)
    for c in range(12):
        up[:, 1 + c] = np.clip(high - 15 * c, 0, 15)
    for c in range(8):
        up[:, 13 + c] = (low >> c) & 1
    gate[:, 21] = 1
    assert np.array_equal(up @ x, u) and (high <= 180).all()
    h = (64 * u).astype(np.float32)
    hq, hs = R.quant(h[None], 1)
    product = R.e4m3_round(h * np.repeat(np.float32(1) / hs[0], 128))
    assert np.sum(product != hq[0]) > 20   # the case means something
    one = lambda *s: torch.ones(1, *s, device=DEV)  # noqa: E731
    for n0 in range(0, F, d):   # output n reads hidden unit n0 + n
        down[:] = 0
        down[np.arange(d), n0 + np.arange(d)] = 1
        ex = ops.Fp8Experts(fp8(gate[None]), one(F // 128, 1), fp8(up[None]), one(F // 128, 1), fp8(down[None]),
                            one(1, F // 128))
        xs = torch.from_numpy(np.repeat(x[None], B, 0)).to(torch.bfloat16).to(DEV)
        ids, w = torch.zeros(B, 1, dtype=torch.int32, device=DEV), torch.ones(B, 1, device=DEV)
        y = torch.empty(B, d, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(ops.xshare_experts_fp8_workspace_size(B, 1, 1, d, F), dtype=torch.uint8, device=DEV)
        ops.xshare_experts_fp8(xs, ids, w, ex, y, ws)
        want = torch.from_numpy(hq[0, n0:n0 + d] * float(hs[0, n0 // 128])).to(torch.bfloat16).to(DEV)
        assert torch.equal(y, want.expand(B, d))


def bytes_of(x, rows):
    """The quantised bytes by their definition: the quotient rounded to 32 bits, then to e4m3."""
    s = R.quant(x, rows)[1]
    big = np.repeat(np.repeat(s, rows, 0)[:x.shape[0]], 128, 1)[:, :x.shape[1]]
    q = (x.astype(np.float64) / big.astype(np.float64)).astype(np.float32)
    return torch.from_numpy(q).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


@pytest.mark.parametrize("dtype,amax", [(t, a) for t in (torch.float32, torch.bfloat16, torch.float16)
                                        for a in (3.0, 1e-30, 1e30)      # both ways to divide
                                        if a == 3.0 or t is not torch.float16])
@pytest.mark.parametrize("K", [128, 130, 133, 132, 144, 1000])   # every width of access
def test_signs_of_zeros(ops, dtype, K, amax):
    """-0, and values so small that they round to a zero, keep their sign, whatever the scale."""
    g = torch.Generator().manual_seed(K)
    x = torch.randn(200, K, generator=g) * amax
    x[torch.rand(200, K, generator=g) < 0.3] = 0.0
    x[torch.rand(200, K, generator=g) < 0.2] *= 1e-6
    x = torch.where(torch.rand(200, K, generator=g) < 0.5, -x, x).to(dtype)
    assert ((x == 0) & torch.signbit(x)).any()
    d = x.to(DEV)
    for rows, call in ((1, ops.xshare_quant_fp8_rows), (128, ops.xshare_quant_fp8_blocks)):
        q = torch.empty(200, K, dtype=ops.FP8, device=DEV)
        s = torch.empty(-(-200 // rows), -(-K // 128), device=DEV)
        call(d, q, s)
        assert np.array_equal(q.view(torch.uint8).cpu().numpy(), bytes_of(x.float().numpy(), rows))
