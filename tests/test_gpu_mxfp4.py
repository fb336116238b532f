"""GPU tests of the four-bit operators against the float64 oracle: quantisation bit for bit
(values, codes, scales and the buffer's padding), its inverse, the product and the token
statistics of a four-bit head.

Tolerances. Quantised values are exact. A product's terms are exact in float32 (four-bit sizes
and powers of two), its sum of K terms is off by at most K half-steps of the sum of sizes, taken
twice as wide (2^-23) for a sum that cuts off instead of rounding: K 2^-23 sum |a b|; bfloat16
adds half a step, 2^-8 of the value. Statistics: those of the LM head (2e-4), whose inputs are
the logits of such a product."""

import math

import numpy as np
import pytest

import oracle
from oracle import mxfp4 as mx
from tests import _harness as H

pytestmark = pytest.mark.gpu


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _bf16(x):
    """float32 values of x rounded to bfloat16."""
    return oracle.bf16_bits_to_f64(H.rne_bf16_bits(np.asarray(x, np.float32))).astype(np.float32)


def _cuda(x, dtype="f32"):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _values(rng, R, K):
    """Rows of different size with a few far values, a row and a block of zeros."""
    x = rng.normal(size=(R, K)) * 2.0 ** rng.integers(-20, 20, (R, 1))
    x *= np.where(rng.random((R, K)) < 0.02, 50.0, 1.0)
    x[R // 2] = 0.0
    x[0, :32] = -0.0
    return _bf16(x)


def _same(q, x):
    """An Mxfp4 against the oracle's, byte for byte."""
    import torch

    torch.cuda.synchronize()
    _, code, scale = mx.quantize(x)
    assert np.array_equal(q.data.cpu().numpy(), mx.buffer_bytes(code, scale))


SHAPES = [(1, 1), (1, 31), (3, 32), (33, 33), (31, 255), (64, 256), (65, 257), (7, 1000), (200, 520),
          (5, 3584)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,K", SHAPES)
def test_quantize_shapes(R, K, dtype):
    dart = _dart()
    x = _values(np.random.default_rng(R * 7919 + K), R, K)
    if dtype == "f32":
        x = (x * np.float32(1.0 + 2.0 ** -12)).astype(np.float32)  # not bfloat16 numbers
    q = dart.dart_mxfp4_quantize(_cuda(x, dtype))
    assert (q.rows, q.cols) == (R, K)
    _same(q, x)
    import torch

    for out in (torch.bfloat16, torch.float32):
        v = dart.dart_mxfp4_dequantize(q, dtype=out)
        assert np.array_equal(v.float().cpu().numpy().astype(np.float64), mx.quantize(x)[0])


def test_quantize_every_bf16_number():
    """Every bfloat16 number, subnormals among them, beside each of several largest sizes: the
    rounding at every tie, saturation, and blocks that end at the smallest scale."""
    dart = _dart()
    every = (np.arange(1 << 16, dtype=np.uint32) << 16).view(np.float32)
    every = every[np.isfinite(every)]
    rows = []
    for top in (2.0 ** -126, 2.0 ** -122, 1.0, 1.5, 1.9921875, 3.0e38):
        some = every[np.abs(every) <= top]
        some = np.concatenate([some, np.zeros(-len(some) % 31, np.float32)]).reshape(-1, 31)
        rows.append(np.concatenate([some, np.full((len(some), 1), top, np.float32)], 1))
    x = np.concatenate(rows)[::3]
    x = x[: len(x) // 8 * 8].reshape(-1, 256)
    _same(dart.dart_mxfp4_quantize(_cuda(x)), x)
    x = _bf16(x)
    _same(dart.dart_mxfp4_quantize(_cuda(x, "bf16")), x)


def test_quantize_float32_next_to_ties():
    """float32 numbers one step either side of every tie, and on it."""
    dart = _dart()
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    near = np.concatenate([ties, np.nextafter(ties, np.float32(0)), np.nextafter(ties, np.float32(9))])
    row = np.concatenate([near, -near])[:42]
    x = np.stack([np.concatenate([[s * 7.0], row[i:i + 31] * s]) for s in 2.0 ** np.arange(-30.0, 31.0, 10)
                  for i in (0, 11)]).astype(np.float32)
    _same(dart.dart_mxfp4_quantize(_cuda(x)), x)


def test_blocks_that_are_not_finite():
    import torch

    dart = _dart()
    rng = np.random.default_rng(3)
    x = rng.normal(size=(40, 300)).astype(np.float32)
    x[3, 40], x[9, 299], x[20, 0], x[39, 256] = np.inf, np.nan, -np.inf, np.nan
    for dtype in ("f32", "bf16"):
        xx = _bf16(x) if dtype == "bf16" else x
        q = dart.dart_mxfp4_quantize(_cuda(xx, dtype))
        _same(q, xx)
        want = mx.quantize(xx)[0]
        got = dart.dart_mxfp4_dequantize(q, dtype=torch.float32).cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        # a product is NaN for just the rows that hold such a block
        b = dart.dart_mxfp4_quantize(_cuda(rng.normal(size=(37, 300)).astype(np.float32)))
        for out in (dart.dart_mxfp4_matmul(q, b, dtype=torch.float32),
                    dart.dart_mxfp4_matmul(b, q, dtype=torch.float32).t()):
            nan = np.isnan(out.cpu().numpy())
            rows = np.isnan(want).any(1)
            assert nan[rows].all() and not nan[~rows].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_and_dequantize_strided_rows(dtype):
    """Rows of a wider matrix, every second row, a base that is no multiple of 16 bytes; written
    rows leave the columns around them alone."""
    import torch

    dart = _dart()
    rng = np.random.default_rng(5)
    wide = _values(rng, 90, 413)
    t = _cuda(wide, dtype)
    for view, ref in ((t[:, 8:400], wide[:, 8:400]), (t[1::2, 3:410], wide[1::2, 3:410]),
                      (t[5:6, 1:], wide[5:6, 1:]), (t[:, 7:8], wide[:, 7:8])):
        q = dart.dart_mxfp4_quantize(view)
        _same(q, ref)
        R, K = ref.shape
        for at, pad in ((0, 0), (3, 5), (8, 8)):
            big = torch.full((R, at + K + pad), 7.0, dtype=t.dtype, device="cuda")
            dart.dart_mxfp4_dequantize(q, out=big[:, at:at + K])
            got = big.float().cpu().numpy().astype(np.float64)
            assert np.array_equal(got[:, at:at + K], mx.quantize(ref)[0])
            assert (got[:, :at] == 7).all() and (got[:, at + K:] == 7).all()


def _product(rng, M, N, K):
    a, b = _values(rng, M, K), _values(rng, N, K)
    va, vb = mx.quantize(a)[0], mx.quantize(b)[0]
    return a, b, va @ vb.T, np.abs(va) @ np.abs(vb).T


# few rows, the tiles of 64, 128 and 256 rows and their edges, inner sizes inside a block, a slice
# and up to several rounds of the ring
PRODUCTS = [(1, 1, 1), (1, 40, 4600), (32, 97, 1300), (3, 64, 2304), (1, 300, 64), (2, 257, 255), (15, 33, 256), (16, 1000, 513), (17, 255, 1000),
            (33, 256, 320), (64, 1025, 776), (65, 129, 2048), (128, 511, 264), (129, 700, 96),
            (257, 130, 512), (300, 2050, 40), (700, 300, 1024),
            (40, 260, 1536), (100, 130, 1793), (300, 129, 1281), (257, 500, 4600), (65, 300, 3600)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_matmul_shapes(M, N, K, out):
    import torch

    dart = _dart()
    a, b, ref, size = _product(np.random.default_rng(M * 31 + N * 7 + K), M, N, K)
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    qb = dart.dart_mxfp4_quantize(_cuda(b))
    got = dart.dart_mxfp4_matmul(dart.dart_mxfp4_quantize(_cuda(a)), qb, dtype=dtype)
    assert tuple(got.shape) == (M, N) and got.dtype == dtype
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = K * 2.0 ** -23 * size + (2.0 ** -8 * np.abs(ref) if out == "bf16" else 0.0)
    assert np.all(err <= tol), float((err - tol).max())
    # an operand that is not yet quantised, and the same bits again
    again = dart.dart_mxfp4_matmul(_cuda(a, "bf16"), qb, dtype=dtype)
    assert torch.equal(again.view(torch.int16), got.view(torch.int16))


@pytest.mark.parametrize("M,N", [(5, 301), (70, 301), (260, 515)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_matmul_into_a_wider_matrix(M, N, out):
    """Any row stride and alignment of the result; the columns and rows around it stay."""
    import torch

    dart = _dart()
    a, b, ref, size = _product(np.random.default_rng(M), M, N, 200)
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    qa, qb = dart.dart_mxfp4_quantize(_cuda(a)), dart.dart_mxfp4_quantize(_cuda(b))
    want = dart.dart_mxfp4_matmul(qa, qb, dtype=dtype)
    for at, pad in ((1, 2), (8, 3), (3, 0)):
        big = torch.full((M + 2, at + N + pad), 7.0, dtype=dtype, device="cuda")
        dart.dart_mxfp4_matmul(qa, qb, out=big[1:M + 1, at:at + N])
        assert torch.equal(big[1:M + 1, at:at + N], want)
        big[1:M + 1, at:at + N] = 7.0
        assert bool((big == 7.0).all())


STATS = [(1, 8, 1), (64, 1100, 130), (130, 2100, 400), (1, 300, 1000), (3, 40, 5), (16, 256, 700), (64, 512, 4099), (129, 200, 513),
         (257, 776, 1300), (600, 128, 2000)]


def _stats_ref(z, y):
    m = z.max(1, keepdims=True)
    e = np.exp(z - m)
    s = e.sum(1)
    lse = m[:, 0] + np.log(s)
    lp = z - lse[:, None]
    return z[np.arange(len(y)), y] - lse, -(e / s[:, None] * lp).sum(1), lse


@pytest.mark.parametrize("inv_temp", [1.0, 0.7])
@pytest.mark.parametrize("T,d,V", STATS)
def test_tok_stats_shapes(T, d, V, inv_temp):
    dart = _dart()
    rng = np.random.default_rng(T + 5 * V + d)
    h = _bf16(rng.normal(size=(T, d)))
    w = _bf16(rng.normal(size=(V, d)) * 3.0 / math.sqrt(d))
    y = rng.integers(0, V, T).astype(np.int32)
    z = mx.quantize(h)[0] @ mx.quantize(w)[0].T * np.float64(np.float32(inv_temp))
    ref = _stats_ref(z, y)
    qw = dart.dart_mxfp4_quantize(_cuda(w, "bf16"))
    got = dart.dart_lmhead_mxfp4_tok_stats(_cuda(h, "bf16"), qw, _cuda(y), inv_temp=inv_temp)
    for name, g, r in zip(("logp", "entropy", "lse"), got, ref):
        err = np.abs(g.cpu().numpy().astype(np.float64) - r).max()
        H.log(f"mxfp4 stats T={T} d={d} V={V}: {name} {err:.1e}")
        assert err <= H.LOGP_TOL
    # hidden states quantised by the caller: the same bits
    again = dart.dart_lmhead_mxfp4_tok_stats(dart.dart_mxfp4_quantize(_cuda(h, "bf16")), qw, _cuda(y),
                                             inv_temp=inv_temp)
    for g, a in zip(got, again):
        assert np.array_equal(g.cpu().numpy(), a.cpu().numpy())


# heights of 256 rows, the last of which has 1, 44, 88, 128 or 129 of them (up to 128 it is formed
# as a short one), from one to several rounds of the ring; the values from the inverse
@pytest.mark.parametrize("T,d,V", [(257, 1100, 40000), (300, 64, 30000), (600, 776, 20000),
                                   (384, 40, 33000), (385, 300, 33000)])
def test_heights_of_256_rows(T, d, V):
    import torch

    dart = _dart()
    rng = np.random.default_rng(T + d + V)
    qh = dart.dart_mxfp4_quantize(_cuda(rng.normal(size=(T, d)).astype(np.float32)))
    qw = dart.dart_mxfp4_quantize(_cuda((rng.normal(size=(V, d)) * 3.0 / math.sqrt(d)).astype(np.float32)))
    y = rng.integers(0, V, T).astype(np.int32)
    h, w = (dart.dart_mxfp4_dequantize(q, dtype=torch.float32).double().cpu().numpy() for q in (qh, qw))
    z = h @ w.T
    tol = d * 2.0 ** -23 * (np.abs(h) @ np.abs(w).T)
    out = dart.dart_mxfp4_matmul(qh, qw, dtype=torch.float32).double().cpu().numpy()
    assert np.all(np.abs(out - z) <= tol)
    out = dart.dart_mxfp4_matmul(qh, qw).double().cpu().numpy()
    assert np.all(np.abs(out - z) <= tol + 2.0 ** -8 * np.abs(z))
    for g, r in zip(dart.dart_lmhead_mxfp4_tok_stats(qh, qw, _cuda(y)), _stats_ref(z, y)):
        assert np.abs(g.cpu().numpy().astype(np.float64) - r).max() <= H.LOGP_TOL


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_product_of_more_than_32_bits_of_elements(out):
    """16500 x 152064 results (2.5e9): rows on both sides of 2^31 elements, every column."""
    import torch

    dart = _dart()
    g = torch.Generator(device="cuda").manual_seed(9)
    M, N, K = 16500, 152064, 72
    qa = dart.dart_mxfp4_quantize(torch.randn((M, K), generator=g, device="cuda"))
    qb = dart.dart_mxfp4_quantize(torch.randn((N, K), generator=g, device="cuda"))
    a, b = (dart.dart_mxfp4_dequantize(q, dtype=torch.float32).double() for q in (qa, qb))
    got = dart.dart_mxfp4_matmul(qa, qb, dtype=torch.bfloat16 if out == "bf16" else torch.float32)
    for rows in (slice(0, 64), slice(7000, 7100), slice(14100, 14150), slice(16400, 16500)):
        z, size = a[rows] @ b.t(), a[rows].abs() @ b.abs().t()
        tol = K * 2.0 ** -23 * size + (2.0 ** -8 * z.abs() if out == "bf16" else 0.0)
        assert bool(((got[rows].double() - z).abs() <= tol).all())


def test_tok_stats_of_blocks_that_are_not_finite():
    """A NaN block of a hidden row shows in that row alone, one of a weight row in every row."""
    import torch

    dart = _dart()
    rng = np.random.default_rng(11)
    h, w = rng.normal(size=(70, 96)), rng.normal(size=(400, 96))
    y = _cuda(rng.integers(0, 399, 70).astype(np.int32))
    qw = dart.dart_mxfp4_quantize(_cuda(w.astype(np.float32)))
    h[5, 40] = np.nan
    got = dart.dart_lmhead_mxfp4_tok_stats(_cuda(h.astype(np.float32)), qw, y)
    for g in got:
        assert torch.nonzero(g.isnan())[:, 0].tolist() == [5]
    h[5, 40], w[399, 3] = 0.0, np.inf
    qw = dart.dart_mxfp4_quantize(_cuda(w.astype(np.float32)))
    for g in dart.dart_lmhead_mxfp4_tok_stats(_cuda(h.astype(np.float32)), qw, y):
        assert bool(g.isnan().all())


def test_tok_stats_do_not_depend_on_the_batch():
    """A row's statistics are the same bits alone, in a small and in a large call."""
    import torch

    dart = _dart()
    g = torch.Generator(device="cuda").manual_seed(7)
    T, d, V = 700, 520, 3000
    h = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    qw = dart.dart_mxfp4_quantize(torch.randn((V, d), generator=g, device="cuda").mul_(0.1))
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    whole = dart.dart_lmhead_mxfp4_tok_stats(h, qw, y)
    for rows in (slice(0, 1), slice(690, 700), slice(100, 230), slice(3, 590)):
        part = dart.dart_lmhead_mxfp4_tok_stats(h[rows], qw, y[rows])
        for a, b in zip(whole, part):
            assert torch.equal(a[rows], b)


def test_seven_b_head():
    """The 7B policy's head (V = 152064, d = 3584): the product of 1 and 300 tokens on sampled
    columns and their statistics against a float64 product on the GPU of the values."""
    import torch

    dart = _dart()
    g = torch.Generator(device="cuda").manual_seed(1)
    V, d = 152064, 3584
    w = (torch.randn((V, d), generator=g, device="cuda") * 0.05).to(torch.bfloat16)
    qw = dart.dart_mxfp4_quantize(w)
    vw = dart.dart_mxfp4_dequantize(qw, dtype=torch.float32)
    rows = torch.randint(0, V, (64,), generator=g, device="cuda")
    assert np.array_equal(vw[rows].cpu().numpy(), mx.quantize(w[rows].float().cpu().numpy())[0])
    for T in (1, 300):
        h = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
        y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        vh = mx.quantize(h.float().cpu().numpy())[0]
        z = torch.cat([torch.from_numpy(vh).cuda() @ part.double().t() for part in vw.split(16384)], 1)
        out = dart.dart_mxfp4_matmul(h, qw, dtype=torch.float32)
        bound = d * 2.0 ** -23 * float(torch.linalg.vector_norm(torch.from_numpy(vh), dim=1).max()
                                       * torch.linalg.vector_norm(vw, dim=1).max())
        assert float((out.double() - z).abs().max()) <= bound
        logp, ent, lse = dart.dart_lmhead_mxfp4_tok_stats(h, qw, y)
        rlse = torch.logsumexp(z, 1)
        lp = z - rlse[:, None]
        assert float((lse - rlse).abs().max()) <= H.LOGP_TOL
        assert float((logp - lp.gather(1, y.long()[:, None])[:, 0]).abs().max()) <= H.LOGP_TOL
        assert float((ent + (lp.exp() * lp).sum(1)).abs().max()) <= H.H_TOL


def test_captured_and_on_another_stream():
    """Quantise, multiply and score in one HIP graph, replayed on new inputs between eager calls;
    and the same on a stream of the caller's."""
    import torch

    dart = _dart()
    g = torch.Generator(device="cuda").manual_seed(2)
    T, d, V = 70, 300, 900
    w = torch.randn((V, d), generator=g, device="cuda") * 0.2
    h = torch.randn((T, d), generator=g, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)

    def run(stream=None):
        q = dart.dart_mxfp4_quantize(w, stream=stream)
        return (dart.dart_mxfp4_dequantize(q, stream=stream), dart.dart_mxfp4_matmul(h, q, stream=stream),
                *dart.dart_lmhead_mxfp4_tok_stats(h, q, y, stream=stream))

    run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for k in range(3):
        h.copy_(torch.randn((T, d), generator=g, device="cuda"))
        w.mul_(-1.5)
        want = [t.clone() for t in run()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k
    side.wait_stream(torch.cuda.current_stream())
    other = run(stream=side)
    side.synchronize()
    for a, b in zip(other, want):
        assert torch.equal(a, b)


def test_refusals_with_tensors():
    import torch

    dart = _dart()
    x = torch.randn((40, 64), device="cuda")
    q = dart.dart_mxfp4_quantize(x)
    y = torch.zeros(40, dtype=torch.int32, device="cuda")
    for bad in (x.half(), x.double(), "x"):
        with pytest.raises(TypeError):
            dart.dart_mxfp4_quantize(bad)
    for bad in (x.cpu(), x.t(), x[0], x[:, :0], x[:0], x[:, ::2], x[:1].expand(40, 64)):
        with pytest.raises(ValueError):
            dart.dart_mxfp4_quantize(bad)
    with pytest.raises(ValueError):
        dart.dart_mxfp4_quantize(x[:, :63], out=q)
    with pytest.raises(TypeError):
        dart.dart_mxfp4_dequantize(q, dtype=torch.float16)
    with pytest.raises(TypeError):
        dart.dart_mxfp4_dequantize(x)
    with pytest.raises(ValueError):
        dart.dart_mxfp4_dequantize(q, out=torch.empty((40, 63), device="cuda"))
    with pytest.raises(ValueError):
        dart.dart_mxfp4_dequantize(q._replace(rows=80))
    with pytest.raises(ValueError):
        dart.dart_mxfp4_dequantize(q._replace(data=q.data[1:]))
    with pytest.raises(ValueError):
        dart.dart_mxfp4_matmul(x[:, :32].contiguous(), q)
    for bad in ((q, x), ("x", q), (None, q)):
        with pytest.raises(TypeError):
            dart.dart_mxfp4_matmul(*bad)
    with pytest.raises(ValueError):
        dart.dart_mxfp4_matmul(x.cpu(), q)
    with pytest.raises(TypeError):
        dart.dart_mxfp4_matmul(q, q, dtype=torch.float16)
    with pytest.raises(ValueError):
        dart.dart_mxfp4_matmul(q, q, out=torch.empty((40, 80), device="cuda")[:, ::2])
    with pytest.raises(ValueError):
        dart.dart_lmhead_mxfp4_tok_stats(q, q, y[:39])
    for temp in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(dart.DartError):
            dart.dart_lmhead_mxfp4_tok_stats(q, q, y, inv_temp=temp)
    with pytest.raises(dart.DartError):  # too small a workspace
        dart.dart_lmhead_mxfp4_tok_stats(q, q, y, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


def test_results_apart_from_the_inputs():
    import torch

    dart = _dart()
    x = torch.randn((64, 512), device="cuda")
    q = dart.dart_mxfp4_quantize(x)
    room = x.view(torch.uint8).reshape(-1)
    inside = dart.Mxfp4(room[:q.data.numel()], 64, 512)
    for call in (lambda: dart.dart_mxfp4_quantize(x, out=inside),
                 lambda: dart.dart_mxfp4_dequantize(inside, out=x),
                 lambda: dart.dart_mxfp4_matmul(inside, q, out=x[:, :64]),
                 lambda: dart.dart_mxfp4_matmul(q, inside, out=x[:, :64]),
                 lambda: dart.dart_mxfp4_matmul(x, q, out=x[:, :64])):
        with pytest.raises(ValueError, match="overlap"):
            call()
