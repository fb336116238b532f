"""Which tensors of a call may not share memory: what it writes, with each other and with what it
reads (tensors on the CPU; no call is made)."""

import pytest
import torch

import paper_2509_23866_amd as dart

BUF = torch.zeros((8, 12))
LINE = BUF.view(-1)


@pytest.mark.parametrize("writes,reads,names", [
    (dict(x=LINE[:10]), dict(y=LINE[9:20]), ("x", "y")),
    (dict(x=LINE[10:20]), dict(y=LINE[:11]), ("x", "y")),
    (dict(x=BUF[:4]), dict(y=BUF[3, :1]), ("x", "y")),
    (dict(x=BUF[2:6, 3:7]), dict(y=LINE[2 * 12 + 5: 2 * 12 + 6]), ("x", "y")),
    (dict(x=LINE[:4], y=LINE[3:5]), {}, ("y", "x")),
    (dict(x=None, y=LINE[:4], z=LINE[2:]), dict(r=None), ("z", "y")),
    (dict(w=LINE.view(torch.uint8)[:16]), dict(y=LINE[3:4]), ("w", "y")),
    (dict(x=LINE[5:6]), dict(y=LINE[:48].view(2, 4, 6)), ("x", "y")),
    # columns of one matrix that meet, also around a row's end
    (dict(x=BUF[:4, :7]), dict(y=BUF[2:6, 6:]), ("x", "y")),
    (dict(x=LINE[6:].as_strided((4, 9), (12, 1))), dict(y=BUF[1:4, :3]), ("x", "y")),
    (dict(x=BUF[:4, :6]), dict(y=BUF[::2, 6:]), ("x", "y")),
])
def test_refused(writes, reads, names):
    with pytest.raises(ValueError, match="the memory of {} and {} must not overlap".format(*names)):
        dart._check_apart(writes, reads)


@pytest.mark.parametrize("writes,reads", [
    (dict(x=LINE[:10]), dict(y=LINE[10:20])),
    (dict(x=BUF[:4]), dict(y=BUF[4:], z=None)),
    (dict(x=BUF[:1, 6:]), dict(y=BUF[:1, :6])),
    (dict(x=None), dict(y=LINE)),
    (dict(x=BUF[:, :6]), dict(y=BUF[:, 6:])),
    (dict(x=BUF[2:6, 8:11]), dict(y=BUF[:, 3:8], z=BUF[:5, 11:])),
    (dict(x=LINE[:4], y=LINE[4:8], z=LINE.view(torch.uint8)[32:40]), dict(r=LINE[10:], s=LINE[10:])),
])
def test_allowed(writes, reads):
    dart._check_apart(writes, reads)


def test_every_pair_of_small_matrices():
    """Against the sets of elements that two matrices of rows equally far apart hold."""
    line = torch.zeros(64)
    views = [line[at:].as_strided((r, c), (5, 1)) for at in (0, 2, 3, 5, 9, 14) for r in (1, 2, 4)
             for c in (1, 2, 4, 5)]
    sets = [{(v[i, j].data_ptr()) for i in range(v.shape[0]) for j in range(v.shape[1])} for v in views]
    for x, sx in zip(views, sets):
        for y, sy in zip(views, sets):
            if sx & sy:
                assert dart._share_memory(x, y)
            elif min(x.shape[0], y.shape[0]) > 1:
                spans = dart._span(x), dart._span(y)
                apart = spans[0][0] >= spans[1][1] or spans[1][0] >= spans[0][1]
                assert apart or not dart._share_memory(x, y)
