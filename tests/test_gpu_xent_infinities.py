"""Logits that pass float32's range in the cross entropy: -infinity is a probability of 0, +infinity
a NaN, each in its own rows. The first hidden column is 2^100 in some rows and 0 in the others, and
the weight's first column +-2^100 in one vocabulary entry: in bfloat16 both are exact."""

import math

import numpy as np
import pytest

from oracle import xent as ox
from tests import _harness as H
from tests.test_gpu_xent import _bf16, _dev, _ids, _np

pytestmark = pytest.mark.gpu

BIG = 2.0 ** 100


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _problem(T, V, at, sign, rows, seed=0):
    rng = np.random.default_rng(seed + T + V)
    h, w = _bf16(rng.normal(size=(T, 64))), _bf16(rng.normal(size=(V, 64)) * 0.3)
    h[:, 0], w[:, 0] = 0.0, 0.0
    h[rows, 0], w[at, 0] = BIG, sign * BIG
    y = rng.integers(0, V, T)
    y[y == at] = (at + 1) % V
    return h, w, y


# heights of 64 and 256 rows; the entry in the middle, first, last and alone in its unit of 64
@pytest.mark.parametrize("T,V,at", [(5, 300, 77), (70, 257, 256), (70, 1000, 0), (400, 40001, 40000)])
@pytest.mark.parametrize("lam", [0.0, 1e-3])
def test_minus_infinity_off_the_target(T, V, at, lam):
    """The row is as if the entry did not exist."""
    dart = _dart()
    rows = np.arange(0, T, 3)
    h, w, y = _problem(T, V, at, -1.0, rows)
    args = _dev(h), _dev(w), _ids(y)
    h0, kept = h.copy(), np.delete(np.arange(V), at)
    h0[:, 0] = 0.0
    ref = ox.xent(h0[rows], w[kept], np.searchsorted(kept, y[rows]), 0.0, lam)
    slack = H.LOGP_TOL * (1.0 + 2.0 * lam * np.abs(ref["lse"]).max()) + 2.0 ** -24 * ref["tok"].max()
    loss, tok, n, dh, dw = dart.dart_lmhead_xent_fwd_bwd(*args, z_loss=lam)
    for got, total in ((tok, loss), dart.dart_lmhead_xent_fwd(*args, z_loss=lam)[1::-1]):
        assert np.abs(_np(got)[rows] - ref["tok"]).max() <= slack
        assert math.isfinite(float(total))
    assert int(n) == T and np.isfinite(_np(dh)).all() and np.isfinite(_np(dw)).all()
    # the entry's own gradient: nothing from those rows (their first hidden value is 2^100)
    assert _np(dw)[at, 0] == 0.0


@pytest.mark.parametrize("eps,hit", [(0.0, True), (0.1, False), (0.1, True)])
def test_minus_infinity_that_is_to_be_learnt(eps, hit):
    dart = _dart()
    rows = np.array([1, 8])
    h, w, y = _problem(12, 300, 130, -1.0, rows)
    if hit:
        y[rows] = 130
    args = _dev(h), _dev(w), _ids(y)
    loss, tok, _, dh, dw = dart.dart_lmhead_xent_fwd_bwd(*args, label_smoothing=eps)
    for total, got in ((loss, tok), dart.dart_lmhead_xent_fwd(*args, label_smoothing=eps)[:2]):
        assert np.flatnonzero(np.isposinf(_np(got))).tolist() == rows.tolist()
        assert np.isfinite(np.delete(_np(got), rows)).all() and float(total) == math.inf
    # the gradient is p less the learnt distribution all the same
    assert np.isfinite(_np(dh)).all() and np.isfinite(_np(dw)).all()
    share = (1.0 - eps if hit else 0.0) + eps / 300
    want = -share * len(rows) / 12 * BIG
    # 2^-8 of dz's rounding, as much of the result's, 2^-11 of the division's by 1 - eps
    assert abs(_np(dw)[130, 0] - want) <= (2 * 2.0 ** -8 + 2.0 ** -11) * abs(want)


@pytest.mark.parametrize("V,at", [(300, 77), (257, 256), (1000, 0)])
@pytest.mark.parametrize("hit", [False, True])
@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_plus_infinity_and_nothing_but_minus_infinity(V, at, hit, eps):
    dart = _dart()
    rows = np.array([2, 3, 9])
    h, w, y = _problem(12, V, at, 1.0, rows)
    if hit:
        y[rows] = at
    _nan_rows(dart, h, w, y, rows, eps)
    w[:, 0] = -BIG
    _nan_rows(dart, h, w, y, rows, eps)


def _nan_rows(dart, h, w, y, rows, eps):
    args = _dev(h), _dev(w), _ids(y)
    loss, tok, _, dh, _ = dart.dart_lmhead_xent_fwd_bwd(*args, label_smoothing=eps)
    for total, got in ((loss, tok), dart.dart_lmhead_xent_fwd(*args, label_smoothing=eps)[:2]):
        assert np.flatnonzero(np.isnan(_np(got))).tolist() == rows.tolist() and math.isnan(float(total))
    bad = np.isnan(_np(dh)).all(1)
    assert np.flatnonzero(bad).tolist() == rows.tolist() and np.isfinite(_np(dh)[~bad]).all()
