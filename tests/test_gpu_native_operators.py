"""The two host paths of the cross entropy and of the four-bit operators: a call that leaves its
outputs to the library (marshalled natively) gives the bits of the same call with its stream given
(marshalled in Python), and what the native path does not take ends as the Python path ends it."""

import pytest

from tests.test_gpu_native_calls import native  # noqa: F401  (the fixture that records the path)

pytestmark = pytest.mark.gpu


def _case():
    import torch

    g = torch.Generator(device="cuda").manual_seed(5)
    h = torch.randn((70, 64), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn((300, 64), generator=g, device="cuda").to(torch.bfloat16)
    y = torch.randint(0, 300, (70,), generator=g, device="cuda", dtype=torch.int32)
    return h, w, torch.where(y % 5 == 0, torch.full_like(y, -100), y)


def _calls(h, w, y):
    import torch

    import paper_2509_23866_amd as dart

    qh, qw = dart.dart_mxfp4_quantize(h), dart.dart_mxfp4_quantize(w)
    y0 = y.clamp(min=0)
    return dict(
        fwd=lambda **k: dart.dart_lmhead_xent_fwd(h, w, y, 0.1, 1e-3, "sum", **k),
        fwd_bwd=lambda **k: dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1, 1e-3, chunk_rows=32, **k),
        only_h=lambda **k: dart.dart_lmhead_xent_fwd_bwd(h, w, y, want=(True, False), **k),
        quantize=lambda **k: dart.dart_mxfp4_quantize(w.float(), **k),
        quantize_strided=lambda **k: dart.dart_mxfp4_quantize(w[::2, 3:], **k),
        dequantize=lambda **k: dart.dart_mxfp4_dequantize(qw, **k),
        dequantize_f32=lambda **k: dart.dart_mxfp4_dequantize(qw, dtype=torch.float32, **k),
        matmul=lambda **k: dart.dart_mxfp4_matmul(qh, qw, **k),
        matmul_raw=lambda **k: dart.dart_mxfp4_matmul(h[:3], qw, dtype=torch.float32, **k),
        stats=lambda **k: dart.dart_lmhead_mxfp4_tok_stats(h, qw, y0, inv_temp=0.7, **k),
        stats_quantised=lambda **k: dart.dart_lmhead_mxfp4_tok_stats(qh, qw, y0, **k))


def _flat(out):
    import torch

    return [t for t in (out if isinstance(out, tuple) else (out,)) if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("name", ["fwd", "fwd_bwd", "only_h", "quantize", "quantize_strided", "dequantize",
                                  "dequantize_f32", "matmul", "matmul_raw", "stats", "stats_quantised"])
def test_both_paths_agree(name, native):  # noqa: F811
    import torch

    call = _calls(*_case())[name]
    del native.taken[:]
    got = call()
    assert native.taken == [True]
    del native.taken[:]
    want = call(stream=torch.cuda.current_stream())
    assert native.taken == []
    assert type(got) is type(want) and len(_flat(got)) == len(_flat(want)) > 0
    for a, b in zip(_flat(got), _flat(want)):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_what_the_native_path_leaves(native):  # noqa: F811
    """Refused with the Python path's exceptions, a failed C call by its name."""
    import torch

    import paper_2509_23866_amd as dart

    h, w, y = _case()
    qw = dart.dart_mxfp4_quantize(w)
    del native.taken[:]
    for error, call in ((TypeError, lambda: dart.dart_lmhead_xent_fwd(h.float(), w, y)),
                        (ValueError, lambda: dart.dart_lmhead_xent_fwd_bwd(h, w, y.long())),
                        (ValueError, lambda: dart.dart_lmhead_xent_fwd(h, w, y, reduction="none")),
                        (TypeError, lambda: dart.dart_mxfp4_quantize(h.half())),
                        (ValueError, lambda: dart.dart_mxfp4_quantize(h.t())),
                        (TypeError, lambda: dart.dart_mxfp4_dequantize((qw.data, 300, 64))),
                        (ValueError, lambda: dart.dart_mxfp4_dequantize(qw._replace(rows=400))),
                        (TypeError, lambda: dart.dart_mxfp4_matmul(h, qw, dtype=torch.float16)),
                        (ValueError, lambda: dart.dart_mxfp4_matmul(h[:, :32], qw)),
                        (ValueError, lambda: dart.dart_lmhead_mxfp4_tok_stats(h, qw, y[:5]))):
        with pytest.raises(error):
            call()
    assert not any(native.taken)
    for name, call in (("dart_lmhead_xent_fwd", lambda: dart.dart_lmhead_xent_fwd(h, w, y, 1.5)),
                       ("dart_lmhead_xent_fwd_bwd", lambda: dart.dart_lmhead_xent_fwd_bwd(h, w, y, -0.5)),
                       ("dart_lmhead_mxfp4_tok_stats",
                        lambda: dart.dart_lmhead_mxfp4_tok_stats(h, qw, y.clamp(min=0), inv_temp=0.0))):
        with pytest.raises(dart.DartError, match=name + " failed"):
            call()
