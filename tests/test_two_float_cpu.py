"""The pair arithmetic of two_float.cuh (compiled for the host) against decimal arithmetic."""
import ctypes
import os
import subprocess
from decimal import Decimal, getcontext

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_07265_gb300", "csrc")
SOURCE = r"""
#include "two_float.cuh"
extern "C" {
void run_exp(const float *x, double *y, int n) {
  for (int i = 0; i < n; ++i) { xs::Two t = xs::two_exp(x[i]); y[i] = (double)t.hi + t.lo; }
}
void run_sigmoid(const float *x, double *y, int n) {
  for (int i = 0; i < n; ++i) { xs::Two t = xs::two_sigmoid(x[i]); y[i] = (double)t.hi + t.lo; }
}
void run_add(const float *a, const float *b, double *y, int n) {
  for (int i = 0; i < n; ++i) {
    xs::Two t = xs::two_sigmoid(a[i]) + b[i];
    y[i] = (double)t.hi + t.lo;
    float s = t.hi + t.lo;
    if (s != t.hi) y[i] = NAN;   // not normalised
  }
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("two")
    src, out = d / "two.cpp", d / "two.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-I", CSRC, "-x", "c++", str(src),
                    "-o", str(out)], check=True, capture_output=True, text=True)
    return ctypes.CDLL(str(out))


def run(fn, *args):
    y = np.empty(len(args[0]), np.float64)
    ptr = lambda a: a.ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    fn(*(ptr(a) for a in args), ptr(y), ctypes.c_int(len(y)))
    return y


def points(lo, hi):
    rng = np.random.default_rng(1)
    edge = (np.arange(-115, 1)[:, None] * np.log(2) / 2 + np.array([-1e-6, 0, 1e-6])).ravel()   # where the reduction steps
    x = np.concatenate([rng.uniform(lo, hi, 3000), -np.exp(rng.uniform(-40, 4, 500)), edge, [0.0, -0.0]])
    return x[(x >= lo) & (x <= hi)].astype(np.float32)


def test_exp(lib):
    getcontext().prec = 40
    x = points(-40.0, 0.0)
    want = np.array([float(Decimal(float(v)).exp()) for v in x])
    assert np.all(np.abs(run(lib.run_exp, x) - want) <= 2.0 ** -40 * want)
    assert np.all(run(lib.run_exp, np.array([-100.5, -1e30, -np.inf], np.float32)) == 0)


def test_sigmoid(lib):
    getcontext().prec = 40
    x = points(-40.0, 0.0)
    x = np.concatenate([x, -x])
    want = np.array([float(1 / (1 + (-Decimal(float(v))).exp())) for v in x])
    assert np.all(np.abs(run(lib.run_sigmoid, x) - want) <= 2.0 ** -38 * want)


def test_sums_are_normalised(lib):
    getcontext().prec = 40
    x = points(-12.0, 0.0)
    b = np.random.default_rng(2).uniform(-1, 1, len(x)).astype(np.float32)
    got = run(lib.run_add, x, b)
    want = np.array([float(1 / (1 + (-Decimal(float(v))).exp()) + Decimal(float(u))) for v, u in zip(x, b)])
    assert np.all(np.abs(got - want) <= 2.0 ** -38 + 2.0 ** -46 * np.abs(want))


def test_small_values(lib):
    """Down to the smallest numbers, whose last bit is 2^-149 whatever the value."""
    getcontext().prec = 60
    x = points(-100.0, 0.0)
    want = np.array([float(Decimal(float(v)).exp()) for v in x])
    assert np.all(np.abs(run(lib.run_exp, x) - want) <= 2.0 ** -40 * want + 2.0 ** -148)
    want = np.array([float(1 / (1 + (-Decimal(float(v))).exp())) for v in x])
    assert np.all(np.abs(run(lib.run_sigmoid, x) - want) <= 2.0 ** -38 * want + 2.0 ** -147)
    assert np.all(np.abs(run(lib.run_sigmoid, -x) - 1 + want) <= 2.0 ** -38)


def test_the_order_is_kept(lib):
    """Larger arguments never give smaller values, into the subnormal numbers."""
    x = np.sort(points(-110.0, 0.0))
    for fn in (lib.run_exp, lib.run_sigmoid):
        assert np.all(np.diff(run(fn, x)) >= 0)


DIFF = r"""
#include "two_float.cuh"
extern "C" void run_exp_diff(const float *l, const float *m, double *y, int n) {
  for (int i = 0; i < n; ++i) { xs::Two t = xs::two_exp_diff(l[i], m[i]); y[i] = (double)t.hi + t.lo; }
}
"""


def test_exp_of_a_difference(tmp_path):
    """Logits whose difference fp32 does not hold, far apart: the rounding of l - m is made good."""
    getcontext().prec = 60
    src, out = tmp_path / "diff.cpp", tmp_path / "diff.so"
    src.write_text(DIFF)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-I", CSRC, "-x", "c++", str(src),
                    "-o", str(out)], check=True, capture_output=True, text=True)
    lib = ctypes.CDLL(str(out))
    rng = np.random.default_rng(3)
    m = rng.uniform(-3, 40, 4000).astype(np.float32)
    l = (m.astype(np.float64) - rng.uniform(0, 75, 4000)).astype(np.float32)
    l = np.minimum(l, m)
    got = run(lib.run_exp_diff, l, m)
    want = np.array([float((Decimal(float(a)) - Decimal(float(b))).exp()) for a, b in zip(l, m)])
    assert np.all(np.abs(got - want) <= 1.5 * 2.0 ** -40 * want + 2.0 ** -148), (np.abs(got - want) / want).max()
