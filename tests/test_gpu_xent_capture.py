"""The captured cross entropy of hidden states that are no leaf: a graph made elsewhere that the
backward pass would run into, through them or through a leaf behind them, is refused (its backward
would end the process; only the refusal is run); one made wholly in the capture is not."""

import pytest

from tests.test_gpu_xent import _dev, _ids, _problem

pytestmark = pytest.mark.gpu


def _inputs():
    h, w, y = _problem(40, 64, 300)
    return _dev(h).requires_grad_(), _dev(w).requires_grad_(), _ids(y)


def _refused(yd, call):
    """call is refused in a capture, which goes on: its graph replays."""
    import torch

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = yd + 1
        with pytest.raises(RuntimeError, match="still alive"):
            call()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, yd + 1)


def test_an_eager_graph_of_a_leaf_behind_the_hidden_states():
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    x, w, y = _inputs()
    x.data, w.data = x.data.contiguous(), w.data.contiguous()
    alive = x * 3.0
    _refused(y, lambda: dart_lmhead_xent_loss(x * 2.0, w, y))
    _refused(y, lambda: dart_lmhead_xent_loss(x * 2.0, w.detach(), y))
    del alive
    torch.cuda.synchronize()


def test_hidden_states_made_before_the_capture():
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    x, w, y = _inputs()
    before = x * 2.0
    _refused(y, lambda: dart_lmhead_xent_loss(before, w, y))
    torch.cuda.synchronize()
    # nothing to learn from them: no reason
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = dart_lmhead_xent_loss(before.detach(), w.detach(), y)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, dart_lmhead_xent_loss(before.detach(), w.detach(), y))


def test_a_graph_of_a_third_stream():
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    x, w, y = _inputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        alive = w * 3.0
    torch.cuda.synchronize()
    _refused(y, lambda: dart_lmhead_xent_loss(x.detach() * 2.0, w, y))
    del alive
    torch.cuda.synchronize()


def test_hidden_states_made_in_the_capture():
    """Loss and gradients of the leaves behind them, replayed between eager steps."""
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    x, w, y = _inputs()

    def step():
        loss = dart_lmhead_xent_loss(x * 2.0, w, y, 0.1, 1e-3)
        return (loss.detach(), *torch.autograd.grad(loss, (x, w)))

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
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_hidden_states_of_a_stream_that_joined_the_capture():
    """Not refused: a stream that the capture forked off is being captured too (the loss alone)."""
    import torch

    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    x, w, y = _inputs()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            hidden = x * 2.0
        here.wait_stream(side)
        loss = dart_lmhead_xent_loss(hidden, w.detach(), y).detach()
        del hidden
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, dart_lmhead_xent_loss(x.detach() * 2.0, w.detach(), y))
