"""Host-side refusals of the four-bit entry points: no case enqueues any work."""

import pytest

import paper_2509_23866_amd as dart

P = 4096  # never dereferenced
INV, UNS = dart.DART_ERR_INVALID_ARG, dart.DART_ERR_UNSUPPORTED
BIG = 2 ** 31 - 1


def _gpu_visible():
    import torch

    return torch.cuda.device_count() > 0


pytestmark = pytest.mark.skipif("_gpu_visible()")


def test_sizes():
    assert dart.dart_mxfp4_bytes(1, 1) == dart.dart_mxfp4_bytes(32, 256) == 4352
    assert dart.dart_mxfp4_bytes(33, 513) == 2 * 3 * 4352
    assert dart.dart_mxfp4_bytes(BIG, BIG) == 2 ** 26 * 2 ** 23 * 4352
    for R, K in ((0, 1), (1, 0), (-1, 5), (5, -1), (BIG + 1, 1), (1, BIG + 1)):
        assert dart.dart_mxfp4_bytes(R, K) == 0
        assert dart.dart_lmhead_mxfp4_stats_workspace_bytes(R, K) == 0
    assert dart.dart_lmhead_mxfp4_stats_workspace_bytes(4, 129) == 4 * 2 * 16 + 16


@pytest.mark.parametrize("kw,rc", [
    (dict(x=0), INV), (dict(q=0), INV), (dict(R=0), INV), (dict(K=0), INV), (dict(ld=63), INV),
    (dict(dtype=2), INV), (dict(R=BIG + 1), INV), (dict(x=P + 1), INV), (dict(q=P + 8), INV),
    (dict(dtype=0, x=P + 2), INV), (dict(R=BIG, K=2 ** 20, ld=2 ** 20), UNS),
])
def test_quantize_rejects(kw, rc):
    a = dict(x=P, dtype=1, R=4, K=64, ld=64, q=P)
    a.update(kw)
    assert dart.load_library().dart_mxfp4_quantize(*a.values(), None) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(q=0), INV), (dict(out=0), INV), (dict(R=0), INV), (dict(K=-1), INV), (dict(ld=63), INV),
    (dict(dtype=9), INV), (dict(q=P + 1), INV), (dict(out=P + 1), INV),
    (dict(R=BIG, K=2 ** 20, ld=2 ** 20), UNS),
])
def test_dequantize_rejects(kw, rc):
    a = dict(q=P, R=4, K=64, dtype=1, out=P, ld=64)
    a.update(kw)
    assert dart.load_library().dart_mxfp4_dequantize(*a.values(), None) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(a=0), INV), (dict(b=0), INV), (dict(out=0), INV), (dict(M=0), INV), (dict(N=0), INV),
    (dict(K=0), INV), (dict(M=BIG + 1), INV), (dict(ld=31), INV), (dict(dtype=5), INV),
    (dict(a=P + 8), INV), (dict(b=P + 8), INV), (dict(out=P + 1), INV), (dict(K=2 ** 24 + 1), UNS),
    (dict(M=BIG, N=BIG, ld=BIG), UNS), (dict(N=2 ** 30, ld=2 ** 30), UNS),
])
def test_matmul_rejects(kw, rc):
    a = dict(a=P, M=4, b=P, N=32, K=64, dtype=1, out=P, ld=32)
    a.update(kw)
    assert dart.load_library().dart_mxfp4_matmul(*a.values(), None) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(h=0), INV), (dict(w=0), INV), (dict(y=0), INV), (dict(logp=0), INV), (dict(ent=0), INV),
    (dict(lse=0), INV), (dict(ws=0), INV), (dict(T=0), INV), (dict(V=0), INV), (dict(d=0), INV),
    (dict(temp=0.0), INV), (dict(temp=float("nan")), INV), (dict(temp=float("inf")), INV),
    (dict(nws=4 * 16 + 4 * 4 - 1), INV), (dict(ws=P + 8), INV), (dict(w=P + 4), INV),
    (dict(d=2 ** 24 + 1), UNS), (dict(T=BIG, V=BIG, nws=2 ** 63), UNS),
])
def test_tok_stats_rejects(kw, rc):
    a = dict(h=P, T=4, w=P, V=32, d=64, y=P, temp=1.0, logp=P, ent=P, lse=P, ws=P, nws=4 * 16 + 4 * 4)
    a.update(kw)
    assert dart.load_library().dart_lmhead_mxfp4_tok_stats(*a.values(), None) == rc
