"""A NaN among the logits of a four-bit head (and of the bfloat16 one, whose epilogue it shares) shows in every result of the row, wherever in the
vocabulary it is: alone in the last unit of 64 columns, filling a unit, or filling the columns of a
unit that one lane holds (those with the same bit 2), so that no finite value stands beside it."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _problem(T, d, V, bad, seed):
    """Quantised hidden states and head, rows `bad` of which hold a NaN, and targets elsewhere."""
    import torch

    dart = _dart()
    rng = np.random.default_rng(seed)
    w = rng.normal(size=(V, d)).astype(np.float32)
    w[bad, rng.integers(0, d, len(bad))] = np.nan
    good = np.setdiff1d(np.arange(V), bad)
    y = torch.from_numpy(rng.choice(good, T).astype(np.int32)).cuda()
    h = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).cuda()
    return dart.dart_mxfp4_quantize(h), dart.dart_mxfp4_quantize(torch.from_numpy(w).cuda()), y


UNIT = np.arange(64)
# vocabulary, rows with a NaN: the last row alone in its unit, a whole unit (in a tile of its own
# half, and the last), one lane's columns of a unit, every row but a few
CASES = [(65, [64]), (385, [384]), (40001, [40000]), (400, 64 + UNIT), (400, 128 + UNIT),
         (448, 384 + UNIT), (300, UNIT[UNIT & 4 == 0]), (300, 64 + UNIT[UNIT & 4 != 0]),
         (321, np.arange(3, 321))]


@pytest.mark.parametrize("T", [1, 70, 300])
@pytest.mark.parametrize("V,bad", CASES)
def test_nan_logits_show_wherever_they_are(T, V, bad):
    dart = _dart()
    qh, qw, y = _problem(T, 96, V, np.asarray(bad), T + V)
    logits = dart.dart_mxfp4_matmul(qh, qw)
    assert logits.isnan().sum(1).tolist() == [len(bad)] * T
    for temp in (1.0, 0.5):
        for got in dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y, inv_temp=temp):
            assert bool(got.isnan().all())


@pytest.mark.parametrize("T,V", [(1, 65), (70, 400), (300, 40001)])
def test_a_nan_target_shows(T, V):
    """The target's own logit alone is a NaN."""
    dart = _dart()
    qh, qw, y = _problem(T, 96, V, np.asarray([V - 1]), T + V)
    y.fill_(V - 1)
    for got in dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y):
        assert bool(got.isnan().all())


@pytest.mark.parametrize("T", [1, 70, 300])
@pytest.mark.parametrize("V,bad", CASES)
def test_bfloat16_head(T, V, bad):
    import torch

    dart = _dart()
    g = torch.Generator(device="cuda").manual_seed(T + V)
    h = torch.randn((T, 64), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn((V, 64), generator=g, device="cuda").to(torch.bfloat16)
    w[torch.as_tensor(np.asarray(bad), device="cuda"), 5] = float("nan")
    y = torch.from_numpy(np.random.default_rng(V).choice(np.setdiff1d(np.arange(V), bad), T).astype(np.int32)).cuda()
    for got in dart.dart_lmhead_tok_stats(h, w, y):
        assert bool(got.isnan().all())
