"""The cross entropy's and the four-bit operators' refusals of memory that a call would write while
it reads it, or write twice: results, workspaces, a factor inside what it scales."""

import pytest

pytestmark = pytest.mark.gpu


def _dart():
    import paper_2509_23866_amd as dart

    return dart


def _case():
    import torch

    g = torch.Generator(device="cuda").manual_seed(8)
    h = torch.randn((40, 64), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn((300, 64), generator=g, device="cuda").to(torch.bfloat16)
    return h, w, torch.randint(0, 300, (40,), generator=g, device="cuda", dtype=torch.int32)


def _bytes(t):
    import torch

    return t.view(-1).view(torch.uint8)


def _inside(big, n):
    """A workspace of n bytes over the start of the tensor's memory (which holds as many)."""
    return _bytes(big)[:n]


def test_workspaces_of_the_cross_entropy():
    import torch

    dart = _dart()
    h, w, y = _case()
    n = dart.dart_lmhead_xent_fwd_workspace_bytes(40, 64, 300)
    m = dart.dart_lmhead_xent_workspace_bytes(40, 64, 300, 40)
    room = torch.zeros(max(n, m), dtype=torch.uint8, device="cuda")
    hr = room[:h.numel() * 2].view(torch.bfloat16).view(40, 64).copy_(h)
    wr = room[:w.numel() * 2].view(torch.bfloat16).view(300, 64)
    yr = room[n - 160 - n % 4: n - n % 4].view(torch.int32)
    with pytest.raises(ValueError, match="workspace and hidden must not overlap"):
        dart.dart_lmhead_xent_fwd(hr, w, y, workspace=room)
    with pytest.raises(ValueError, match="workspace and weight must not overlap"):
        dart.dart_lmhead_xent_fwd(h, wr, y, workspace=room)
    with pytest.raises(ValueError, match="workspace and target must not overlap"):
        dart.dart_lmhead_xent_fwd(h, w, yr, workspace=room)
    for kw, names in ((dict(dhidden=hr), "workspace and dhidden"), (dict(dweight=wr), "workspace and dweight")):
        with pytest.raises(ValueError, match=names + " must not overlap"):
            dart.dart_lmhead_xent_fwd_bwd(h, w, y, workspace=room, **kw)
    with pytest.raises(ValueError, match="workspace and hidden must not overlap"):
        dart.dart_lmhead_xent_fwd_bwd(hr, w, y, workspace=room)
    for a, b in zip(dart.dart_lmhead_xent_fwd_bwd(h, w, y, workspace=room), dart.dart_lmhead_xent_fwd_bwd(h, w, y)):
        assert torch.equal(a, b)


def test_results_and_workspace_of_the_four_bit_statistics():
    import torch

    dart = _dart()
    h, w, y = _case()
    qh, qw = dart.dart_mxfp4_quantize(h), dart.dart_mxfp4_quantize(w)
    want = dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y)
    n = dart.dart_lmhead_mxfp4_stats_workspace_bytes(40, 300)
    f32 = lambda t: _bytes(t)[:160].view(torch.float32)  # noqa: E731
    three = torch.zeros(118, device="cuda")
    for kw, names in ((dict(logp=f32(y)), "logp and target"), (dict(entropy=f32(qh.data)), "entropy and hidden"),
                      (dict(lse=f32(qw.data)), "lse and weight"),
                      (dict(logp=three[:40], entropy=three[39:79]), "entropy and logp"),
                      (dict(logp=three[:40], entropy=three[40:80], lse=three[78:]), "lse and entropy"),
                      (dict(workspace=_inside(qw.data, n)), "workspace and weight"),
                      (dict(workspace=_inside(qh.data, n)), "workspace and hidden")):
        with pytest.raises(ValueError, match=names + " must not overlap"):
            dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y, **kw)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="workspace and lse must not overlap"):
        dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y, lse=f32(ws), workspace=ws)
    with pytest.raises(ValueError, match="logp and hidden must not overlap"):
        dart.dart_lmhead_mxfp4_tok_stats(h, qw, y, logp=f32(h))
    got = dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y, logp=three[:40], entropy=three[78:], lse=f32(ws[:160].clone()),
                                           workspace=ws)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_a_factor_inside_what_it_scales():
    import torch

    dart = _dart()
    x = torch.full((3, 5), 2.0, device="cuda")
    for factor in (x[0, 0], x[1, 2:3], x[2:, 4:]):
        with pytest.raises(ValueError, match="x and factor must not overlap"):
            dart.dart_grad_scale(x, factor)
    assert bool((x == 2.0).all())
    dart.dart_grad_scale(x[:2], x[2:, 4:])
    assert bool((x[:2] == 4.0).all())
