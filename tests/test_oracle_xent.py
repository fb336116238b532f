"""Pins of the cross-entropy oracle: closed forms, torch's float64 loss and its autograd, finite
differences, and the rows that do not count."""

import math

import numpy as np
import pytest
import torch

from oracle import xent as ox


def _problem(T, d, V, seed=0):
    rng = np.random.default_rng(seed)
    return rng.normal(size=(T, d)), rng.normal(size=(V, d)), rng.integers(0, V, T)


def test_flat_rows():
    h, w, y = np.zeros((3, 4)), np.ones((7, 4)), np.array([0, 3, 6])
    r = ox.xent(h, w, y, eps=0.3, lam=0.5)
    assert np.allclose(r["tok"], math.log(7) + 0.5 * math.log(7) ** 2)
    r = ox.xent(h, w, y, reduction="sum")
    assert np.isclose(r["loss"], 3 * math.log(7))
    assert np.allclose(r["dz"].sum(1), 0)
    assert np.isclose(r["dz"][1, 3], 1 / 7 - 1) and np.isclose(r["dz"][1, 0], 1 / 7)


@pytest.mark.parametrize("reduction", ["mean", "sum"])
@pytest.mark.parametrize("eps", [0.0, 0.1, 0.9])
@pytest.mark.parametrize("lam", [0.0, 0.01])
def test_against_torch(eps, lam, reduction):
    h, w, y = _problem(9, 5, 11)
    y[[2, 5]] = -100
    r = ox.xent(h, w, y, eps, lam, reduction)
    th, tw = (torch.tensor(a, requires_grad=True) for a in (h, w))
    z = th @ tw.t()
    loss = torch.nn.functional.cross_entropy(z, torch.tensor(y), ignore_index=-100, label_smoothing=eps,
                                             reduction=reduction)
    keep = torch.tensor(y >= 0)
    extra = lam * torch.logsumexp(z, 1).square()[keep].sum()
    loss = loss + (extra / 7 if reduction == "mean" else extra)
    loss.backward()
    assert np.isclose(r["loss"], loss.item()) and r["n"] == 7
    assert np.allclose(r["dh"], th.grad.numpy()) and np.allclose(r["dw"], tw.grad.numpy())
    assert (r["dh"][[2, 5]] == 0).all() and (r["tok"][[2, 5]] == 0).all()


def test_finite_differences():
    h, w, y = _problem(4, 3, 6, seed=3)
    y[1] = -1
    r = ox.xent(h, w, y, 0.2, 0.03)
    step = 1e-6
    for a, grad in ((h, r["dh"]), (w, r["dw"])):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + step
            up = ox.xent(h, w, y, 0.2, 0.03)["loss"]
            a[i] = keep - step
            down = ox.xent(h, w, y, 0.2, 0.03)["loss"]
            a[i] = keep
            assert abs((up - down) / (2 * step) - grad[i]) <= 1e-8


def test_rows_that_do_not_count():
    h, w, y = _problem(5, 3, 4)
    y[:] = [-1, 4, 2, 100, -100]
    clean = ox.xent(h[2:3], w, y[2:3], 0.1)
    h[[0, 1, 3, 4]] = np.nan
    r = ox.xent(h, w, y, 0.1)
    assert r["n"] == 1 and np.isclose(r["loss"], clean["loss"])
    assert np.allclose(r["dw"], clean["dw"]) and np.allclose(r["dh"][2], clean["dh"][0])
    none = ox.xent(h, w, np.full(5, -100), 0.1)
    assert none["n"] == 0 and none["loss"] == 0 and not none["dw"].any()
