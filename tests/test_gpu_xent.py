"""GPU tests of the LM head's cross entropy and its gradients against the float64 oracle.

Tolerances. Losses: those of the LM head's statistics (2e-4, the logits' error in float32), times
1 + 2 lambda |lse| for the z-loss. Gradients: with U = 2^-8 (half a bfloat16 step), an element of
dz is off by its roundings to float16 (2^-11) and bfloat16 (U) and the error of its exponential
(2^-13, as for the LM head's dlogits), all of the sum of its terms' sizes, and by what a
float16 below its normal range loses (2^-39 of the row's weight); a product of K terms adds
K 2^-24 of the terms' sizes, and the result's rounding U of itself."""

import math

import numpy as np
import pytest

import oracle
from oracle import xent as ox
from tests import _harness as H

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _bf16(x):
    return oracle.bf16_bits_to_f64(H.rne_bf16_bits(np.asarray(x, np.float32)))


def _dev(x, pad=0, rows=0):
    """x as a bfloat16 GPU matrix whose rows are `pad` elements apart, NaNs between and after."""
    import torch

    t = torch.full((x.shape[0] + rows, x.shape[1] + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    t[:x.shape[0], :x.shape[1]] = torch.from_numpy(np.asarray(x, np.float32)).cuda()
    return t[:x.shape[0], :x.shape[1]]


def _ids(y):
    import torch

    return torch.from_numpy(np.asarray(y, np.int32)).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _problem(T, d, V, left_out=0.3, seed=None):
    """Logits of standard deviation 3, targets from unlikely to almost sure, some rows left out."""
    rng = np.random.default_rng(T * 131 + d * 7 + V if seed is None else seed)
    w = _bf16(rng.normal(size=(V, d)) * 3.0 / math.sqrt(d))
    y = rng.integers(0, V, T)
    wy = w[y]
    up = rng.uniform(0, 25, (T, 1)) / np.maximum((wy ** 2).sum(1, keepdims=True), 1e-3)
    h = _bf16(rng.normal(size=(T, d)) + up * wy)
    y[rng.random(T) < left_out] = -100
    return h, w, y


def _check_loss(got, ref, lam=0.0, reduction="mean"):
    loss, tok, n = got
    slack = 1.0 + 2.0 * lam * np.abs(ref["lse"]).max(initial=0.0)
    assert int(n.item()) == ref["n"]
    err = np.abs(_np(tok) - ref["tok"]).max()
    assert err <= H.LOGP_TOL * slack + 2.0 ** -24 * np.abs(ref["tok"]).max(), err
    # a mean is off by no more than its terms, a sum by all of theirs
    terms = max(ref["n"], 1) if reduction == "sum" else 1
    assert abs(float(loss.item()) - ref["loss"]) <= H.LOGP_TOL * slack * terms + 2.0 ** -23 * abs(ref["loss"])


def _tolerance(ref, weight, a, b, K, out):
    """Of out = a' b with a the sizes of dz's terms, b those of the other operand."""
    elem = (U + 2.0 ** -11 + 2.0 ** -13) * a + 2.0 ** -39 * weight * (a > 0)
    return elem @ b + K * 2.0 ** -24 * (a @ b) + U * np.abs(out) + 1e-30


def _check_grads(dh, dw, ref, h, w, y, reduction="mean"):
    T, V = ref["mag"].shape
    weight = 1.0 if reduction == "sum" else 1.0 / max(ref["n"], 1)
    rows = (np.asarray(y) >= 0) & (np.asarray(y) < V)
    h0 = np.where(rows[:, None], h, 0.0)
    if dh is not None:
        err = np.abs(_np(dh) - ref["dh"])
        tol = _tolerance(ref, weight, ref["mag"], np.abs(w), V, ref["dh"])
        assert np.all(err <= tol), float((err / tol).max())
        assert not _np(dh)[~rows].any()
    if dw is not None:
        err = np.abs(_np(dw) - ref["dw"])
        tol = _tolerance(ref, weight, ref["mag"].T, np.abs(h0), T, ref["dw"])
        assert np.all(err <= tol), float((err / tol).max())


# tiles of 64, 128 and 256 rows, their edges, vocabularies and hidden sizes that end inside tiles
SHAPES = [(1, 8, 1), (1, 64, 300), (3, 8, 5), (48, 512, 4000), (64, 256, 257), (129, 72, 513),
          (200, 136, 255), (257, 264, 1030), (300, 200, 2001), (700, 136, 1000), (1030, 64, 700)]


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("eps,lam,reduction", [(0.0, 0.0, "mean"), (0.1, 1e-3, "mean"), (0.0, 1e-2, "sum")])
def test_shapes(T, d, V, eps, lam, reduction):
    dart = _dart()
    h, w, y = _problem(T, d, V)
    ref = ox.xent(h, w, y, eps, lam, reduction)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    kw = dict(label_smoothing=eps, z_loss=lam, reduction=reduction)
    _check_loss(dart.dart_lmhead_xent_fwd(hd, wd, yd, **kw), ref, lam, reduction)
    *got, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, **kw)
    _check_loss(got, ref, lam, reduction)
    _check_grads(dh, dw, ref, h, w, y, reduction)


# heights of 256 rows, the last of which has 1, 44, 88, 128 or 129 of them (up to 128 it is formed
# as a short one), from one to several rounds of the ring
@pytest.mark.parametrize("T,d,V", [(257, 264, 40000), (300, 64, 30000), (600, 520, 20000), (384, 8, 33000),
                                   (385, 72, 33000)])
def test_heights_of_256_rows(T, d, V):
    dart = _dart()
    h, w, y = _problem(T, d, V, left_out=0.0)
    ref = ox.xent(h, w, y, 0.1, 1e-3)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    _check_loss(dart.dart_lmhead_xent_fwd(hd, wd, yd, 0.1, 1e-3), ref, 1e-3)
    *got, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, 0.1, 1e-3)
    _check_loss(got, ref, 1e-3)
    _check_grads(dh, dw, ref, h, w, y)


# the gradient's products in large and in small tiles (rows, d, V on both sides of the rule), rows and
# columns that end inside them, blocks of rows, results in wider matrices of odd row lengths
@pytest.mark.parametrize("T,d,V,chunk,pad", [(321, 136, 15000, 321, 0), (320, 136, 15000, 320, 0),
                                             (700, 136, 14000, 400, 3), (400, 264, 13569, 400, 1),
                                             (500, 3584, 1300, 500, 0), (400, 128, 15000, 400, 3),
                                             (1100, 264, 6700, 350, 0)])
def test_tiles_of_the_gradient_products(T, d, V, chunk, pad):
    import torch

    dart = _dart()
    h, w, y = _problem(T, d, V)
    ref = ox.xent(h, w, y, 0.1, 1e-3)
    dh = torch.full((T, d + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((V, d + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    *got, _, _ = dart.dart_lmhead_xent_fwd_bwd(_dev(h), _dev(w), _ids(y), 0.1, 1e-3, chunk_rows=chunk,
                                               dhidden=dh[:, :d], dweight=dw[:, :d])
    _check_loss(got, ref, 1e-3)
    _check_grads(dh[:, :d], dw[:, :d], ref, h, w, y)
    assert bool((dh[:, d:] == 7.0).all()) and bool((dw[:, d:] == 7.0).all())


@pytest.mark.parametrize("chunk", [1, 100, 256, 300, 512])
def test_chunks(chunk):
    """dweight summed over chunks of rows, also where the last ones hold no labelled row."""
    import torch

    dart = _dart()
    T, d, V = (40, 72, 300) if chunk == 1 else (700, 72, 900)
    h, w, y = _problem(T, d, V, left_out=0.4)
    ref = ox.xent(h, w, y, 0.05, 1e-3)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    kw = dict(label_smoothing=0.05, z_loss=1e-3)
    *got, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, chunk_rows=chunk, **kw)
    _check_loss(got, ref, 1e-3)
    _check_grads(dh, dw, ref, h, w, y)
    *_, dh1, _ = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, chunk_rows=chunk, want=(True, False), **kw)
    *_, none, dw1 = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, chunk_rows=chunk, want=(False, True), **kw)
    assert none is None and torch.equal(dh1, dh) and torch.equal(dw1, dw)


@pytest.mark.parametrize("T", [5, 300])
def test_no_labels_one_label_and_ids_past_the_vocabulary(T):
    import torch

    dart = _dart()
    h, w, y = _problem(T, 64, 500, left_out=0.0)
    hd, wd = _dev(h), _dev(w)
    for labels in (np.full(T, -100), np.where(np.arange(T) == T - 1, y, -1), np.where(np.arange(T) == 0, y, 500),
                   np.where(np.arange(T) % 2 == 0, y, 2 ** 31 - 1), np.full(T, -2 ** 31)):
        for reduction in ("mean", "sum"):
            ref = ox.xent(h, w, labels, 0.1, 1e-3, reduction)
            kw = dict(label_smoothing=0.1, z_loss=1e-3, reduction=reduction)
            _check_loss(dart.dart_lmhead_xent_fwd(hd, wd, _ids(labels), **kw), ref, 1e-3, reduction)
            for chunk in (T, 2):
                *got, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd, wd, _ids(labels), chunk_rows=chunk, **kw)
                _check_loss(got, ref, 1e-3, reduction)
                _check_grads(dh, dw, ref, h, w, labels, reduction)
                if ref["n"] == 0:
                    assert float(got[0]) == 0.0 and not bool(dw.any()) and not bool(dh.any())
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 300])
def test_the_sum_of_the_rows_losses(T):
    """The loss is the float64 sum of tok_loss, rounded once (where its order may change no more
    than the last bit), the same bits every time, also over a workspace that held anything."""
    import torch

    dart = _dart()
    h, w, y = _problem(T, 72, 700, left_out=0.4, seed=T)
    y[T // 2] = 5
    hd, wd = _dev(h), _dev(w)
    n = dart.dart_lmhead_xent_fwd_workspace_bytes(T, 72, 700)
    for labels in (y, np.where(np.arange(T) == T - 1, 3, -100), np.full(T, -100)):
        yd = _ids(labels)
        for reduction in ("mean", "sum"):
            first = None
            for fill in (0, 255, 1, 77, 255, 0):
                ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
                loss, tok, _ = dart.dart_lmhead_xent_fwd(hd, wd, yd, reduction=reduction, workspace=ws)
                want = _np(tok).sum() / (max((labels >= 0).sum(), 1) if reduction == "mean" else 1)
                assert abs(float(loss) - want) <= 2.0 ** -23 * abs(want)
                first = loss if first is None else first
                assert torch.equal(loss, first)


def test_rows_left_out_may_hold_anything():
    """NaNs and infinities in the hidden states of rows without a label reach nothing, and the
    same rows' outputs are zeros."""
    import torch

    dart = _dart()
    h, w, y = _problem(300, 64, 700, left_out=0.5)
    ref = ox.xent(h, w, y, 0.1)
    hd = _dev(h)
    rows = torch.from_numpy(y < 0).cuda()
    hd[rows] = torch.tensor([float("nan"), float("inf")] * 32, dtype=torch.bfloat16, device="cuda")
    *got, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd, _dev(w), _ids(y), label_smoothing=0.1)
    _check_loss(got, ref)
    _check_grads(dh, dw, ref, h, w, y)
    _check_loss(dart.dart_lmhead_xent_fwd(hd, _dev(w), _ids(y), label_smoothing=0.1), ref)


def test_a_nan_shows_in_its_row_alone():
    dart = _dart()
    h, w, y = _problem(70, 64, 300, left_out=0.0)
    hd = _dev(h)
    hd[7, 3] = float("nan")
    loss, tok, _, dh, _ = dart.dart_lmhead_xent_fwd_bwd(hd, _dev(w), _ids(y))
    bad = np.isnan(_np(tok))
    assert bad[7] and bad.sum() == 1 and math.isnan(float(loss))
    assert np.isnan(_np(dh)[7]).all() and np.isfinite(np.delete(_np(dh), 7, 0)).all()
    assert np.isnan(_np(dart.dart_lmhead_xent_fwd(hd, _dev(w), _ids(y))[1])).sum() == 1


def test_far_apart_logits():
    """Rows whose logits span hundreds, in one tile and across tiles: probabilities down to 0,
    a target that is the only likely one and one that is hopeless."""
    dart = _dart()
    rng = np.random.default_rng(4)
    T, d, V = 64, 32, 1500
    w = _bf16(rng.normal(size=(V, d)))
    h = _bf16(rng.normal(size=(T, d)) * 10.0 ** rng.uniform(-2, 2, (T, 1)))
    z = h @ w.T
    y = np.where(np.arange(T) % 3 == 0, z.argmax(1), np.where(np.arange(T) % 3 == 1, z.argmin(1),
                                                                rng.integers(0, V, T)))
    size = np.abs(h) @ np.abs(w).T  # the logits' error is relative to this
    for eps in (0.0, 0.2):
        ref = ox.xent(h, w, y, eps)
        loss, tok, n, dh, dw = dart.dart_lmhead_xent_fwd_bwd(_dev(h), _dev(w), _ids(y), label_smoothing=eps)
        slack = 4.0 * d * 2.0 ** -24 * size.max(1)  # of two logits and lse, twice over
        assert np.all(np.abs(_np(tok) - ref["tok"]) <= H.LOGP_TOL + slack)
        # an exponential's relative error is the logits' absolute one
        mag = ref["mag"] * (1.0 + 2.0 ** 8 * slack[:, None])
        _check_grads(dh, dw, {**ref, "mag": mag}, h, w, y)


@pytest.mark.parametrize("pad", [0, 8, 24])
def test_rows_apart_and_results_in_wider_matrices(pad):
    import torch

    dart = _dart()
    T, d, V = 130, 72, 301
    h, w, y = _problem(T, d, V)
    ref = ox.xent(h, w, y, 0.1)
    want = dart.dart_lmhead_xent_fwd_bwd(_dev(h), _dev(w), _ids(y), label_smoothing=0.1)
    for at in (0, 1, 8):
        big_h = torch.full((T + 1, d + at + 3), 7.0, dtype=torch.bfloat16, device="cuda")
        big_w = torch.full((V + 1, d + at + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        got = dart.dart_lmhead_xent_fwd_bwd(_dev(h, pad, 1), _dev(w, pad, 1), _ids(y), label_smoothing=0.1,
                                            dhidden=big_h[:T, at:at + d], dweight=big_w[:V, at:at + d])
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        _check_grads(got[3], got[4], ref, h, w, y)
        big_h[:T, at:at + d] = 7.0
        big_w[:V, at:at + d] = 7.0
        assert bool((big_h == 7.0).all()) and bool((big_w == 7.0).all())


def test_rows_do_not_depend_on_each_other():
    """A token's loss is the same bits in any batch that takes the same call, and twice."""
    import torch

    dart = _dart()
    h, w, y = _problem(600, 136, 2000, left_out=0.1)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    whole = dart.dart_lmhead_xent_fwd(hd, wd, yd)[1]
    both = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd)
    for a, b in zip(both, dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd)):
        assert torch.equal(a, b)
    for rows in (slice(0, 1), slice(5, 70), slice(100, 399)):
        assert torch.equal(dart.dart_lmhead_xent_fwd(hd[rows], wd, yd[rows])[1], whole[rows])
        part = dart.dart_lmhead_xent_fwd_bwd(hd[rows], wd, yd[rows])
        assert torch.equal(part[1], both[1][rows])


def test_autograd():
    """The loss as a function: only the wanted gradients, an incoming gradient, a second backward,
    no gradients under no_grad, and a sum of two losses."""
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    dart = _dart()
    h, w, y = _problem(130, 72, 900)
    yd = _ids(y)
    hd, wd = _dev(h).requires_grad_(), _dev(w).requires_grad_()
    loss0, _, _, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd.detach(), wd.detach(), yd, 0.1, 1e-3)
    loss = dart_lmhead_xent_loss(hd, wd, yd, 0.1, 1e-3)
    assert loss.shape == () and torch.equal(loss, loss0[0])
    loss.backward(retain_graph=True)
    assert torch.equal(hd.grad, dh) and torch.equal(wd.grad, dw)
    g = torch.autograd.grad(loss, (hd, wd), grad_outputs=torch.tensor(0.5, device="cuda"))
    assert torch.equal(g[0], dh * 0.5) and torch.equal(g[1], dw * 0.5)
    assert torch.equal(hd.grad, dh)
    only = torch.autograd.grad(dart_lmhead_xent_loss(hd, wd.detach(), yd, 0.1, 1e-3) * 3.0, hd)[0]
    assert torch.equal(only, (dh.float() * 3.0).to(torch.bfloat16))
    with torch.no_grad():
        assert not dart_lmhead_xent_loss(hd, wd, yd).requires_grad
    assert not dart_lmhead_xent_loss(hd.detach(), wd.detach(), yd).requires_grad
    two = dart_lmhead_xent_loss(hd, wd, yd) + dart_lmhead_xent_loss(hd, wd, yd, reduction="sum")
    a, b = torch.autograd.grad(two, (hd, wd))
    assert bool(torch.isfinite(a).all()) and bool(torch.isfinite(b).all())


def test_gradients_against_differences():
    """Directional derivatives of the float64 loss at the bfloat16 inputs."""
    dart = _dart()
    T, d, V = 40, 64, 400
    h, w, y = _problem(T, d, V)
    *_, dh, dw = dart.dart_lmhead_xent_fwd_bwd(_dev(h), _dev(w), _ids(y), label_smoothing=0.1, z_loss=1e-3)
    rng = np.random.default_rng(0)
    for _ in range(4):
        a, b = rng.normal(size=h.shape), rng.normal(size=w.shape)
        s = 1e-5
        up = ox.xent(h + s * a, w + s * b, y, 0.1, 1e-3)["loss"]
        down = ox.xent(h - s * a, w - s * b, y, 0.1, 1e-3)["loss"]
        got = float((_np(dh) * a).sum() + (_np(dw) * b).sum())
        ref = ox.xent(h, w, y, 0.1, 1e-3)
        tol = (_tolerance(ref, 1.0 / ref["n"], ref["mag"], np.abs(w), V, ref["dh"]) * np.abs(a)).sum() \
            + (_tolerance(ref, 1.0 / ref["n"], ref["mag"].T, np.abs(h), T, ref["dw"]) * np.abs(b)).sum()
        assert abs(got - (up - down) / (2 * s)) <= tol + 1e-7


def test_grad_scale():
    import torch

    dart = _dart()
    g = torch.Generator(device="cuda").manual_seed(1)
    for dtype in (torch.bfloat16, torch.float32):
        for shape, cut in (((1, 1), 0), ((7, 64), 0), ((300, 1000), 0), ((5, 77), 3), ((65, 40), 8)):
            big = torch.randn((shape[0], shape[1] + cut), generator=g, device="cuda").to(dtype)
            x = big[:, cut:]
            for f in (1.0, 0.3, -2.0, 0.0):
                want = (x.float() * torch.tensor(f, device="cuda")).to(dtype)
                keep = big[:, :cut].clone()
                assert dart.dart_grad_scale(x, torch.tensor([f], device="cuda")) is x
                assert torch.equal(x, want) and torch.equal(big[:, :cut], keep)
    bad = torch.full((2, 8), float("nan"), device="cuda")
    dart.dart_grad_scale(bad, torch.ones(1, device="cuda"))
    assert bool(bad.isnan().all())


def test_captured_and_on_another_stream():
    """Loss and gradients in one HIP graph, replayed with other targets (other counts of labelled
    rows) between eager calls; two calls at once on two streams."""
    import torch

    dart = _dart()
    h, w, y = _problem(300, 72, 1100)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    hold = torch.Generator(device="cuda").manual_seed(3)

    def run(stream=None):
        return (*dart.dart_lmhead_xent_fwd(hd, wd, yd, 0.1, stream=stream),
                *dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, 0.1, chunk_rows=256, stream=stream))

    run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for k, left_out in enumerate((0.0, 0.5, 1.0, 0.2)):
        new = torch.randint(0, 1100, (300,), generator=hold, device="cuda", dtype=torch.int32)
        drop = torch.rand(300, generator=hold, device="cuda") < left_out
        yd.copy_(torch.where(drop, torch.full_like(new, -100), new))
        want = [t.clone() for t in run()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k
    side.wait_stream(torch.cuda.current_stream())
    first, second = run(stream=side), run()
    side.synchronize()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, want):
        assert torch.equal(a, c) and torch.equal(b, c)


def test_captured_backward():
    """A training step of the loss captured and replayed. While an eager loss of the same leaves
    is alive the captured one is refused (its backward would end the process)."""
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    h, w, y = _problem(60, 64, 300)
    hd, wd, yd = _dev(h).requires_grad_(), _dev(w).requires_grad_(), _ids(y)
    alive = dart_lmhead_xent_loss(hd, wd, yd)
    refused = torch.cuda.CUDAGraph()
    with torch.cuda.graph(refused):
        kept = yd + 1
        with pytest.raises(RuntimeError, match="still alive"):
            dart_lmhead_xent_loss(hd, wd, yd)
    refused.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, yd + 1)
    want = (alive.detach().clone(), *torch.autograd.grad(alive, (hd, wd)))
    del alive

    def step():
        loss = dart_lmhead_xent_loss(hd, wd, yd)
        return (loss.detach(), *torch.autograd.grad(loss, (hd, wd)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(got, step(), want):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_capture_is_refused_beside_any_graph_of_a_leaf():
    """Whatever made the leaf's accumulator on another stream; one made by the same capture is
    no reason."""
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    h, w, y = _problem(40, 64, 300)
    hd, wd, yd = _dev(h), _dev(w).requires_grad_(), _ids(y)
    alive = (wd.float() ** 2).sum()
    refused = torch.cuda.CUDAGraph()
    with torch.cuda.graph(refused):
        kept = yd + 1
        with pytest.raises(RuntimeError, match="still alive"):
            dart_lmhead_xent_loss(hd, wd, yd)
    refused.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, yd + 1)
    del alive
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = dart_lmhead_xent_loss(hd, wd, yd)
        second = dart_lmhead_xent_loss(hd, wd, yd, 0.1)
        got = (first.detach(), second.detach(), torch.autograd.grad(first + second, wd)[0])
    del first, second
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        a, b = dart_lmhead_xent_loss(hd, wd, yd), dart_lmhead_xent_loss(hd, wd, yd, 0.1)
        want = (a.detach(), b.detach(), torch.autograd.grad(a + b, wd)[0])
        del a, b
        for x, z in zip(got, want):
            assert torch.equal(x, z)


def test_offsets_past_32_bits():
    """16500 rows of V = 152064 in one block: 5 GB of exponentials, and results of rows and entries
    on both sides of 2^31 elements against a float64 sum on the GPU."""
    import torch

    dart = _dart()
    T, d, V = 16500, 64, 152064
    g = torch.Generator(device="cuda").manual_seed(5)
    hd = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    wd = (torch.randn((V, d), generator=g, device="cuda") * 0.4).to(torch.bfloat16)
    yd = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    loss, tok, n, dh, dw = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, chunk_rows=T, reduction="sum")
    h, w, y = hd.double(), wd.double(), yd.long()
    rdh, mdh = torch.empty_like(h), torch.empty_like(h)
    rdw, mdw = torch.zeros_like(w), torch.zeros_like(w)
    ref = torch.empty(T, dtype=torch.float64, device="cuda")
    for r in range(0, T, 1500):
        s = slice(r, min(r + 1500, T))
        z = h[s] @ w.t()
        lse = torch.logsumexp(z, 1)
        at = y[s][:, None]
        ref[s] = lse - z.gather(1, at)[:, 0]
        p = (z - lse[:, None]).exp_()
        mdh[s] = p @ w.abs() + w.abs()[y[s]]
        mdw += p.t() @ h[s].abs()
        mdw.index_add_(0, y[s], h[s].abs())
        p.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float64))
        rdh[s] = p @ w
        rdw += p.t() @ h[s]
    assert int(n) == T and float((tok.double() - ref).abs().max()) <= H.LOGP_TOL + 2.0 ** -24 * float(ref.max())
    assert abs(float(loss) - float(ref.sum())) <= H.LOGP_TOL * T + 2.0 ** -23 * float(ref.sum())
    each = U + 2.0 ** -11 + 2.0 ** -13
    least = 2.0 ** -39
    tol = each * mdh + least * w.abs().sum(0) + V * 2.0 ** -24 * mdh + U * rdh.abs()
    assert bool(((dh.double() - rdh).abs() <= tol).all())
    tol = each * mdw + least * h.abs().sum(0) + T * 2.0 ** -24 * mdw + U * rdw.abs()
    assert bool(((dw.double() - rdw).abs() <= tol).all())


def test_checks_report_ids_past_the_vocabulary(monkeypatch):
    dart = _dart()
    h, w, y = _problem(20, 16, 50)
    hd, wd = _dev(h), _dev(w)
    want = dart.dart_lmhead_xent_fwd_bwd(hd, wd, _ids(y))
    monkeypatch.setenv("DART_CHECK", "1")
    for a, b in zip(dart.dart_lmhead_xent_fwd_bwd(hd, wd, _ids(y)), want):
        assert bool((a == b).all())
    y[3] = 50
    for call in (dart.dart_lmhead_xent_fwd, dart.dart_lmhead_xent_fwd_bwd):
        with pytest.raises(dart.DartError):
            call(hd, wd, _ids(y))


def test_refusals_with_tensors():
    import torch

    dart = _dart()
    h, w, y = _problem(20, 16, 50)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    for call in (dart.dart_lmhead_xent_fwd, dart.dart_lmhead_xent_fwd_bwd):
        for bad in ((hd.float(), wd, yd), (hd, wd.half(), yd), (hd[0], wd, yd)):
            with pytest.raises(TypeError):
                call(*bad)
        for bad in ((hd.cpu(), wd, yd), (hd, wd[:, :8], yd), (hd, wd, yd[:19]), (hd, wd, yd.long()),
                    (hd.t(), wd, yd), (hd[:, 1:9], wd[:, :8], yd)):
            with pytest.raises(ValueError):
                call(*bad)
        for kw in (dict(label_smoothing=1.0), dict(label_smoothing=-0.1), dict(z_loss=-1.0),
                   dict(z_loss=float("nan")), dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
            with pytest.raises(dart.DartError):
                call(hd, wd, yd, **kw)
        with pytest.raises(ValueError):
            call(hd, wd, yd, reduction="none")
    for kw in (dict(want=(False, False)), dict(dhidden=torch.empty((20, 15), device="cuda")),
               dict(dweight=torch.empty((50, 16), device="cuda")), dict(workspace="none")):
        with pytest.raises(ValueError):
            dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, **kw)
    with pytest.raises(ValueError):
        dart.dart_grad_scale(hd, torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        dart.dart_grad_scale(hd, 2.0)


def test_results_apart_from_the_inputs():
    import torch

    dart = _dart()
    h, w, y = _problem(20, 16, 50)
    hd, wd, yd = _dev(h), _dev(w), _ids(y)
    both = torch.empty((69, 16), dtype=torch.bfloat16, device="cuda")
    for kw in (dict(dhidden=hd), dict(dweight=wd), dict(dhidden=both[:20], dweight=both[19:])):
        with pytest.raises(ValueError, match="overlap"):
            dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, **kw)
    both = torch.empty((70, 16), dtype=torch.bfloat16, device="cuda")
    got = dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd, dhidden=both[:20], dweight=both[20:])
    for a, b in zip(got, dart.dart_lmhead_xent_fwd_bwd(hd, wd, yd)):
        assert torch.equal(a, b)
