"""xshare_gate's order of choice values against the plain 64-bit form, where fp32 misleads."""
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


def ids_of(ops, logits, k, scoring, bias=None, **kw):
    B = logits.shape[0]
    ids, w = torch.full((B, k), 77, dtype=torch.int32, device=DEV), torch.empty(B, k, device=DEV)
    ops.xshare_gate(logits.to(DEV), k, ops.gate_params(scoring, **kw), ids, w, bias=None if bias is None else bias.to(DEV))
    return ids.cpu().numpy()


def check(ops, logits, k, scoring, bias=None, **kw):
    want = R.gate(logits.numpy(), k, scoring, bias=None if bias is None else bias.numpy(), **kw)[0]
    got = ids_of(ops, logits, k, scoring, bias, **kw)
    assert np.array_equal(got, want), (int((got != want).any(1).sum()), "rows differ")


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,size,top", [(3, 2, 2), (8, 8, 3), (5, 7, 2), (32, 3, 9), (4, 64, 3)])
def test_groups_whose_values_cancel(ops, scoring, G, size, top):
    """One group holds a large positive and a large negative bias: fp32 knows its worth to 2^-14
    or so, wherever among the groups it comes out, while the others' worths lie 2^-12 apart."""
    g = torch.Generator().manual_seed(G)
    B, N = 4000, G * size
    bias = torch.zeros(G, size)
    bias[:, 2:] = -0.9             # the first two experts make a group's worth
    at = G // 2
    # The group's third value must not come near: far below in the group with the large pair.
    bias[at] = -3000.0
    bias[at, 0], bias[at, 1] = 1000.0, -1000.0
    l = torch.full((B, G, size), 0.5)
    spread = 2e-4 if scoring == "sigmoid" else 2e-4 * N / 4
    l[:, :, :2] += spread * torch.randn(B, G, 2, generator=g)
    check(ops, l.reshape(B, N).contiguous(), min(top * size, 16) if size < 8 else 8, scoring, bias.reshape(N).contiguous(),
          n_groups=G, top_groups=top, group_top=2)


def logit(s):
    return torch.log(s / (1 - s))


@pytest.mark.parametrize("k,copies", [(1, 1), (1, 2), (3, 1), (3, 5), (8, 30)])
@pytest.mark.parametrize("G", [1, 2])
def test_equal_experts_before_one_that_is_near(ops, k, copies, G):
    """The last winner has equals of a higher index, and behind them an expert whose real choice value is
    larger or smaller by less than fp32 resolves: it wins or loses against all of them."""
    g = torch.Generator().manual_seed(k + copies)
    B, N, b0, b1 = 2000, 64, torch.tensor(0.1), torch.tensor(0.3)
    base = torch.empty(B, dtype=torch.float32).uniform_(0.0, 2.0, generator=g)
    l = torch.full((B, N), -5.0)
    l[:, :k - 1] = 4 + torch.rand(B, k - 1, generator=g)     # winners before
    l[:, k - 1:k + copies] = base[:, None]
    s = torch.sigmoid(base.double()) + b0.double() - b1.double()
    x = N // G - 1                                            # in the first group
    l[:, x] = logit(s).float()
    bias = torch.full((N,), 0.1)
    bias[x] = 0.3
    c = torch.sigmoid(l.double()) + bias.double()
    gap = c[:, x] - c[:, k - 1]
    keep = gap.abs() > 2.0 ** -36                             # what 40 bits tell for certain
    assert keep.sum() > 1900 and 0.4 < (gap[keep] > 0).double().mean() < 0.6
    check(ops, l[keep].contiguous(), k, "sigmoid", bias, n_groups=G, top_groups=1)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_scores_below_the_range_of_fp32(ops, scoring):
    """e^-100 and less: the choice values differ by orders of magnitude, and a bias of zeros changes nothing."""
    for rows, k in (([[-130.0, -120, -110], [-105, -101, -104], [0, -120, -110], [-99, -100.5, -101.5], [-90, -95, -89]], 3),
                    ([[-87.5, -88.0, -103.9, -150, -149, -600, -599, -400]], 5)):
        l = torch.tensor(rows)
        for n in range(1, k + 1):
            check(ops, l, n, scoring, torch.zeros(l.shape[1]))
            check(ops, l, n, scoring)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,k", [(20, 6), (64, 16), (256, 8), (1000, 16)])
@pytest.mark.parametrize("lo,hi", [(-300, -90), (-200, 5), (30, 250), (-1e30, -1e29), (-20, 20), (-1e-20, 1e-20)])
def test_a_bias_of_zeros_changes_nothing(ops, scoring, N, k, lo, hi):
    """Scores that underflow, saturate or agree in all the bits that are looked at: equal biases leave the order to the
    logits, for few such experts and for more than are kept as candidates."""
    g = torch.Generator().manual_seed(N)
    l = torch.empty(60, N).uniform_(lo, hi, generator=g)
    want = R.gate(l.numpy(), k, scoring)[0]
    assert np.array_equal(ids_of(ops, l, k, scoring, torch.zeros(N)), want)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,size,top", [(4, 2, 2), (8, 8, 3), (5, 7, 2), (32, 3, 9), (4, 64, 3), (8, 1, 5)])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("lo,hi", [(-140, -110), (-115, -80), (-400, -70), (-90, -60), (-300, 0)])
def test_groups_of_scores_below_the_range_of_fp32(ops, scoring, G, size, top, group_top, lo, hi):
    """Groups whose worth underflows keep the order of the real sums, without a bias and with one of zeros
    (a softmax has them below its largest score)."""
    g = torch.Generator().manual_seed(G + size)
    l = torch.empty(100, G * size).uniform_(lo, hi, generator=g)
    if scoring == "softmax":
        l[:, 0] = 2.0
    k = min(top * size, 8)
    kw = dict(n_groups=G, top_groups=top, group_top=group_top)
    check(ops, l, k, scoring, **kw)
    # The reference takes groups by logits where there is no bias, which is the order of the scores too.
    want = R.gate(l.numpy(), k, scoring, **kw)[0]
    assert np.array_equal(ids_of(ops, l, k, scoring, torch.zeros(G * size), **kw), want)
