"""The cross entropy of more than 4096 rows, where the labelled ones are found by a kernel of their
own (1024 rows at a time) and gathered by another: rows left out at random, in runs, at the ends
and nearly all of them, in one chunk and in several of which the last hold no labelled row."""

import numpy as np
import pytest

from tests.test_gpu_tile_heights import _xent_problem, check_xent

pytestmark = pytest.mark.gpu


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _labels(y, kind, T):
    """Some of y's rows left out: True where one is kept."""
    import torch

    t = torch.arange(T, device=y.device)
    rng = np.random.default_rng(T)
    keep = {"some": torch.from_numpy(rng.random(T) < 0.6).cuda(), "few": torch.from_numpy(rng.random(T) < 0.03).cuda(),
            "runs": t // 700 % 2 == 0, "episodes": t % 1200 > 900, "first": t < 1024, "last": t >= T - 1,
            "middle": (t >= 1000) & (t < 2100), "all": t >= 0, "even": t % 2 == 0}[kind]
    return torch.where(keep, y, torch.full_like(y, -100))


@pytest.mark.parametrize("T,d,V", [(4096, 72, 700), (4097, 72, 700), (5120, 136, 1001), (9001, 64, 513)])
@pytest.mark.parametrize("kind", ["some", "few", "runs", "episodes", "first", "last", "middle", "all", "even"])
def test_left_out_rows(T, d, V, kind):
    dart = _dart()
    h, w, y = _xent_problem(T, d, V, 0.0)
    y = _labels(y, kind, T)
    h[y < 0] = float("nan")  # reaches nothing
    for eps, lam, chunk in ((0.0, 0.0, None), (0.1, 1e-3, 1500)):
        got = dart.dart_lmhead_xent_fwd_bwd(h, w, y, eps, lam, chunk_rows=chunk)
        check_xent(got, h, w, y, eps, lam)
        loss = dart.dart_lmhead_xent_fwd(h, w, y, eps, lam)
        check_xent((*loss, *got[3:]), h, w, y, eps, lam)


@pytest.mark.parametrize("want", [(True, False), (False, True)])
@pytest.mark.parametrize("chunk", [100, 2048, 4999])
def test_one_gradient_and_chunks(want, chunk):
    import torch

    dart = _dart()
    h, w, y = _xent_problem(5000, 72, 600, 0.0)
    y = _labels(y, "episodes", 5000)
    both = dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1, 1e-3, chunk_rows=chunk)
    check_xent(both, h, w, y, 0.1, 1e-3)
    one = dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1, 1e-3, chunk_rows=chunk, want=want)
    for a, b in zip(one, both):
        assert a is None or torch.equal(a, b)
    assert [g is None for g in one[3:]] == [not x for x in want]


def test_no_labels():
    import torch

    dart = _dart()
    h, w, y = _xent_problem(6000, 72, 600, 0.0)
    y.fill_(-1)
    for chunk in (None, 1000):
        loss, tok, n, dh, dw = dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1, 1e-3, chunk_rows=chunk)
        assert float(loss) == 0.0 and int(n) == 0
        assert not any(bool(t.any()) for t in (tok, dh, dw))
    torch.cuda.synchronize()


def test_rows_on_both_sides_of_the_two_forms():
    """4096 rows take one kernel, 4097 two: the rows that both calls hold have the same bits."""
    import torch

    dart = _dart()
    h, w, y = _xent_problem(4097, 136, 900, 0.5)
    more, less = (dart.dart_lmhead_xent_fwd(h[:T], w, y[:T], 0.1) for T in (4097, 4096))
    assert torch.equal(more[1][:4096], less[1])
    more, less = (dart.dart_lmhead_xent_fwd_bwd(h[:T], w, y[:T], 0.1, reduction="sum") for T in (4097, 4096))
    assert torch.equal(more[1][:4096], less[1])


def test_captured_with_other_labels_on_replay():
    import torch

    dart = _dart()
    h, w, y = _xent_problem(5000, 72, 600, 0.0)
    full = y.clone()

    def run():
        return (*dart.dart_lmhead_xent_fwd(h, w, y, 0.1), *dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1, chunk_rows=2048))

    run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for kind in ("few", "all", "last", "runs"):
        y.copy_(_labels(full, kind, 5000))
        want = [t.clone() for t in run()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), kind
