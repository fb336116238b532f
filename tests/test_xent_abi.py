"""Host-side rules of the cross-entropy entry points: refusals (no case enqueues any work),
workspace sizes and the plan of its chunks."""

import ctypes

import pytest

import paper_2509_23866_amd as dart

P = 4096  # never dereferenced
INV, UNS = dart.DART_ERR_INVALID_ARG, dart.DART_ERR_UNSUPPORTED
BIG = 2 ** 31 - 1


def _gpu_visible():
    import torch

    return torch.cuda.device_count() > 0


no_gpu = pytest.mark.skipif("_gpu_visible()")


def _config(eps=0.0, lam=0.0, reduction=0):
    return ctypes.byref(dart.dart_xent_config_t(eps, lam, reduction))


BAD = [dict(h=0), dict(w=0), dict(y=0), dict(config=None), dict(loss=0), dict(tok=0), dict(n=0),
       dict(ws=0), dict(ws=P + 8), dict(T=0), dict(V=0), dict(d=4), dict(d=12), dict(ldh=8), dict(ldw=8),
       dict(ldh=20), dict(ldw=20), dict(h=P + 8), dict(w=P + 8), dict(T=BIG + 1), dict(V=BIG + 1),
       dict(nws=15)] + [
    dict(config=_config(*c)) for c in ((-0.1, 0.0, 0), (1.0, 0.0, 0), (float("nan"), 0.0, 0),
                                       (0.0, -1.0, 0), (0.0, float("inf"), 0), (0.0, float("nan"), 0),
                                       (0.0, 0.0, 2), (0.0, 0.0, -1))]


@no_gpu
@pytest.mark.parametrize("kw", BAD + [dict(rc=UNS, T=BIG, V=BIG), dict(rc=UNS, ldh=2 ** 22 + 8),
                                      dict(rc=UNS, ldw=2 ** 22 + 8), dict(rc=UNS, T=2 ** 23)])
def test_fwd_rejects(kw):
    kw = dict(kw)
    rc = kw.pop("rc", INV)
    a = dict(h=P, T=4, d=16, ldh=16, w=P, V=32, ldw=16, y=P, config=_config(), loss=P, tok=P, n=P, ws=P,
             nws=1 << 30)
    a.update(kw)
    assert dart.load_library().dart_lmhead_xent_fwd(*a.values(), None) == rc


@no_gpu
@pytest.mark.parametrize("kw", BAD + [
    dict(dh=0, dw=0), dict(lddh=15), dict(lddw=15), dict(chunk=0), dict(chunk=-1), dict(dh=P + 1),
    dict(dw=P + 1), dict(rc=UNS, T=BIG, V=BIG, chunk=BIG), dict(rc=UNS, ldh=2 ** 22 + 8),
    dict(rc=UNS, V=2 ** 22 + 1), dict(rc=UNS, lddh=2 ** 22 + 1), dict(rc=UNS, lddw=2 ** 22 + 1)])
def test_fwd_bwd_rejects(kw):
    kw = dict(kw)
    rc = kw.pop("rc", INV)
    a = dict(h=P, T=4, d=16, ldh=16, w=P, V=32, ldw=16, y=P, config=_config(), loss=P, tok=P, n=P, dh=P,
             lddh=16, dw=P, lddw=16, chunk=4, ws=P, nws=1 << 30)
    a.update(kw)
    assert dart.load_library().dart_lmhead_xent_fwd_bwd(*a.values(), None) == rc


@no_gpu
@pytest.mark.parametrize("kw", [dict(x=0), dict(f=0), dict(rows=0), dict(cols=0), dict(ld=7), dict(dtype=3),
                                dict(x=P + 1), dict(f=P + 2), dict(dtype=0, x=P + 2), dict(rows=BIG + 1)])
def test_grad_scale_rejects(kw):
    a = dict(x=P, dtype=1, rows=4, cols=8, ld=8, f=P)
    a.update(kw)
    assert dart.load_library().dart_grad_scale(*a.values(), None) == INV


def test_workspace_sizes():
    for f in (dart.dart_lmhead_xent_fwd_workspace_bytes,
              lambda *a: dart.dart_lmhead_xent_workspace_bytes(*a, 4)):
        for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (BIG + 1, 8, 8)):
            assert f(*bad) == 0
    assert dart.dart_lmhead_xent_workspace_bytes(8, 8, 8, 0) == 0
    T, d, V = 1000, 64, 5000
    fwd = dart.dart_lmhead_xent_fwd_workspace_bytes(T, d, V)
    assert fwd >= T * 20 * 16 + T * (2 * d + 8)
    one = dart.dart_lmhead_xent_workspace_bytes(T, d, V, T)
    assert one >= fwd + T * V * 2
    assert dart.dart_lmhead_xent_workspace_bytes(T, d, V, 10 * T) == one
    cut = dart.dart_lmhead_xent_workspace_bytes(T, d, V, 256)
    assert cut >= 256 * V * 2 + V * d * 4 and cut < one


def test_plan():
    assert dart.lmhead_xent_plan(4096, 152064) == 4096
    for T, V, budget in ((152569, 152064, 2 << 30), (10000, 50257, 1 << 28), (600, 152064, 1)):
        rows = dart.lmhead_xent_plan(T, V, budget)
        most = max(budget // (2 * ((V + 7) // 8 * 8)), 256)
        assert rows % 256 == 0 and rows <= most
        assert -(-T // rows) == -(-T // (most // 256 * 256))  # no more chunks than must be
