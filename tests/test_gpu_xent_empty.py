"""No rows or no vocabulary entries: refused the same way with and without gradients."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V", [(0, 50), (20, 0), (0, 0)])
def test_empty_calls_are_refused(T, V):
    import torch

    import paper_2509_23866_amd as dart
    from paper_2509_23866_amd.autograd import dart_lmhead_xent_loss

    h = torch.zeros((T, 16), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((V, 16), dtype=torch.bfloat16, device="cuda").requires_grad_()
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    for kw in ({}, dict(stream=side)):
        for call in (dart.dart_lmhead_xent_fwd, dart.dart_lmhead_xent_fwd_bwd):
            with pytest.raises(dart.DartError, match="INVALID_ARG"):
                call(h, w.detach(), y, **kw)
    with pytest.raises(dart.DartError, match="INVALID_ARG"):
        dart_lmhead_xent_loss(h, w, y)
