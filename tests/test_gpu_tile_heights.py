"""Every height of the cross entropy's and the four-bit tile, chosen by size as the library chooses
(each test states the height that its sizes take): the 256-row ones with several rounds of the
ring, their last height with 1 to 255 rows (up to 128 it is formed as a short one), and rows whose
bits are the same in calls of different heights. References in float64 on the GPU, tolerances those
of the operators' own tests."""

import numpy as np
import pytest

from tests import _harness as H
from tests import _heights

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _gen(seed):
    import torch

    return torch.Generator(device="cuda").manual_seed(seed)


def _stats(z, y):
    import torch

    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    return lp.gather(1, y.long()[:, None])[:, 0], -(lp.exp() * lp).sum(1), lse


# rows, vocabulary and hidden size (a panel's K slice has 256 columns: 4, 5 and 8 of them; a ring 3),
# the height
FOUR_BIT = [(600, 50257, 776, 256), (640, 40000, 1100, 256), (900, 40000, 1100, 256), (1152, 20000, 776, 256),
            (513, 40000, 1793, 256), (512, 30000, 1100, 256), (700, 20000, 776, 256), (640, 40000, 520, 256),
            (257, 40000, 1100, 128), (384, 33000, 1793, 128), (600, 20000, 776, 128), (513, 20000, 1100, 128),
            (129, 20000, 1100, 64), (200, 4099, 1793, 64)]


@pytest.mark.parametrize("M,N,K,height", FOUR_BIT)
def test_four_bit_product_and_statistics(M, N, K, height):
    import torch

    dart = _dart()
    assert _heights.mxfp4(M, N) == height
    g = _gen(M + N + K)
    qh = dart.dart_mxfp4_quantize(torch.randn((M, K), generator=g, device="cuda"))
    qw = dart.dart_mxfp4_quantize(torch.randn((N, K), generator=g, device="cuda") * (3.0 / K ** 0.5))
    y = torch.randint(0, N, (M,), generator=g, device="cuda", dtype=torch.int32)
    h, w = (dart.dart_mxfp4_dequantize(q, dtype=torch.float32).double() for q in (qh, qw))
    z = h @ w.t()
    tol = K * 2.0 ** -23 * (h.abs() @ w.abs().t())
    out = dart.dart_mxfp4_matmul(qh, qw, dtype=torch.float32)
    assert bool(((out.double() - z).abs() <= tol).all())
    out = dart.dart_mxfp4_matmul(qh, qw)
    assert bool(((out.double() - z).abs() <= tol + U * z.abs()).all())
    for got, ref in zip(dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y), _stats(z, y)):
        assert float((got.double() - ref).abs().max()) <= H.LOGP_TOL


def _xent_problem(T, d, V, left_out, seed=0):
    import torch

    g = _gen(T + V + d + seed)
    w = (torch.randn((V, d), generator=g, device="cuda") * (3.0 / d ** 0.5)).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    wy = w[y.long()].float()
    up = torch.rand((T, 1), generator=g, device="cuda") * 25.0 / wy.square().sum(1, keepdim=True).clamp(min=1e-3)
    h = (torch.randn((T, d), generator=g, device="cuda") + up * wy).to(torch.bfloat16)
    drop = torch.rand(T, generator=g, device="cuda") < left_out
    return h, w, torch.where(drop, torch.full_like(y, -100), y)


def check_xent(got, h, w, y, eps, lam):
    """(loss, tok, n, dh, dw) of a mean against float64 sums over the labelled rows, 1500 at a time."""
    import torch

    loss, tok, n, dh, dw = got
    V, rows = w.shape[0], torch.nonzero(y >= 0)[:, 0]
    N = rows.numel()
    assert int(n) == N
    w = w.double()
    rdw, mdw = torch.zeros_like(w), torch.zeros_like(w)
    hsum = torch.zeros(w.shape[1], dtype=torch.float64, device=w.device)
    ref = torch.zeros(y.numel(), dtype=torch.float64, device=w.device)
    each, least, top = U + 2.0 ** -11 + 2.0 ** -13, 2.0 ** -39 / max(N, 1), 0.0
    for r in rows.split(1500):
        x, at = h[r].double(), y[r].long()
        z = x @ w.t()
        lse = torch.logsumexp(z, 1)
        want = torch.full_like(z, eps / V)
        want.scatter_add_(1, at[:, None], torch.full_like(z[:, :1], 1.0 - eps))
        ref[r] = (want * (lse[:, None] - z)).sum(1) + lam * lse ** 2
        p = (z - lse[:, None]).exp() * (1.0 + 2.0 * lam * lse)[:, None]
        dz, mag = (p - want) / N, (p.abs() + want) / N
        rdh, mdh = dz @ w, mag @ w.abs()
        tol = each * mdh + least * w.abs().sum(0) + V * 2.0 ** -24 * mdh + U * rdh.abs()
        assert bool(((dh[r].double() - rdh).abs() <= tol).all())
        rdw += dz.t() @ x
        mdw += mag.t() @ x.abs()
        hsum += x.abs().sum(0)
        top = max(top, float(lse.abs().max()))
    tol = each * mdw + least * hsum + y.numel() * 2.0 ** -24 * mdw + U * rdw.abs()
    assert bool(((dw.double() - rdw).abs() <= tol).all())
    assert not bool(dh[y < 0].any()) and not bool(tok[y < 0].any())
    slack = H.LOGP_TOL * (1.0 + 2.0 * lam * top)
    assert float((tok.double() - ref).abs().max()) <= slack + 2.0 ** -24 * float(ref.abs().max())
    mean = float(ref.sum()) / max(N, 1)
    assert abs(float(loss) - mean) <= slack + 2.0 ** -23 * abs(mean)


# a K slice has 64 columns
XENT = [(640, 264, 40000, 256), (900, 520, 40000, 256), (513, 264, 40000, 256), (512, 200, 30000, 256),
        (1152, 264, 20000, 256), (700, 136, 20000, 256), (600, 520, 20000, 256), (384, 264, 33000, 128),
        (257, 520, 40000, 128), (700, 264, 4099, 128), (129, 520, 20000, 64), (600, 264, 2000, 64)]


@pytest.mark.parametrize("T,d,V,height", XENT)
@pytest.mark.parametrize("left_out", [0.0, 0.4])
def test_cross_entropy(T, d, V, height, left_out):
    import torch

    dart = _dart()
    assert _heights.xent(T, V) == height
    h, w, y = _xent_problem(T, d, V, left_out)
    for eps, lam in ((0.0, 0.0), (0.1, 1e-3)):
        got = dart.dart_lmhead_xent_fwd_bwd(h, w, y, eps, lam)
        check_xent(got, h, w, y, eps, lam)
        loss, tok, n = dart.dart_lmhead_xent_fwd(h, w, y, eps, lam)
        check_xent((loss, tok, n, *got[3:]), h, w, y, eps, lam)
    torch.cuda.synchronize()


PARTS = [slice(0, 1), slice(5, 134), slice(100, 357), slice(1, 513), slice(0, 700)]


def test_rows_of_the_four_bit_statistics_in_every_height():
    import torch

    dart = _dart()
    T, d, V = 700, 520, 20000
    assert {_heights.mxfp4(len(range(T)[p]), V) for p in PARTS} == {64, 128, 256}
    g = _gen(3)
    h = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    qw = dart.dart_mxfp4_quantize(torch.randn((V, d), generator=g, device="cuda") * 0.1)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    whole = dart.dart_lmhead_mxfp4_tok_stats(h, qw, y)
    for rows in PARTS:
        for a, b in zip(whole, dart.dart_lmhead_mxfp4_tok_stats(h[rows], qw, y[rows])):
            assert torch.equal(a[rows], b)


def test_rows_of_the_cross_entropy_in_every_height():
    import torch

    dart = _dart()
    T, d, V = 700, 264, 20000
    assert {_heights.xent(len(range(T)[p]), V) for p in PARTS} == {64, 128, 256}
    h, w, y = _xent_problem(T, d, V, 0.1)
    whole, both = dart.dart_lmhead_xent_fwd(h, w, y, 0.1)[1], dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1)[1]
    for rows in PARTS:
        assert torch.equal(dart.dart_lmhead_xent_fwd(h[rows], w, y[rows], 0.1)[1], whole[rows])
        assert torch.equal(dart.dart_lmhead_xent_fwd_bwd(h[rows], w, y[rows], 0.1)[1], both[rows])


def test_rows_of_the_four_bit_product_in_every_height():
    import torch

    dart = _dart()
    M, K, N = 700, 776, 20000
    parts = [p for p in PARTS if len(range(M)[p]) > 32]  # up to 32 rows sum in another order
    assert {_heights.mxfp4(len(range(M)[p]), N) for p in parts} == {64, 128, 256}
    g = _gen(4)
    h = torch.randn((M, K), generator=g, device="cuda")
    qw = dart.dart_mxfp4_quantize(torch.randn((N, K), generator=g, device="cuda"))
    whole = dart.dart_mxfp4_matmul(h, qw, dtype=torch.float32)
    for rows in parts:
        assert torch.equal(dart.dart_mxfp4_matmul(h[rows], qw, dtype=torch.float32), whole[rows])
