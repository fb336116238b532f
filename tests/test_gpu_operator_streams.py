"""The cross entropy's and the four-bit operators' ``stream`` argument: what a call allocates
(workspace, a quantised operand, results) is the memory of the stream that its kernels run on, so
that calls in flight on several streams share none of it, whatever came before on the current one."""

import pytest

pytestmark = pytest.mark.gpu

NAMES = ["fwd", "fwd_bwd", "quantize", "dequantize", "matmul", "stats"]


def _case(seed, T=700, V=20000, d=512):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((V, d), generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    return h, w, y


def _call(name, h, w, y, q, **k):
    import torch

    import paper_2509_23866_amd as dart

    out = dict(fwd=lambda: dart.dart_lmhead_xent_fwd(h, w, y, 0.1, **k),
               fwd_bwd=lambda: dart.dart_lmhead_xent_fwd_bwd(h, w, y, 0.1, chunk_rows=256, **k),
               quantize=lambda: dart.dart_mxfp4_quantize(w, **k).data,
               dequantize=lambda: dart.dart_mxfp4_dequantize(q, **k),
               matmul=lambda: dart.dart_mxfp4_matmul(h, q, **k),
               stats=lambda: dart.dart_lmhead_mxfp4_tok_stats(h, q, y, **k))[name]()
    return [out] if isinstance(out, torch.Tensor) else list(out)


def _problems():
    import paper_2509_23866_amd as dart

    out = []
    for seed in (1, 2):
        h, w, y = _case(seed)
        out.append((h, w, y, dart.dart_mxfp4_quantize(w)))
    return out


@pytest.mark.parametrize("name", NAMES)
def test_allocations_are_the_streams(name, monkeypatch):
    """Every allocation is made with the call's stream current: a stream, its handle, and the null
    stream's handle."""
    import torch

    one, _ = _problems()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    here = torch.cuda.current_stream()
    made, empty = [], torch.empty

    def recorded(*a, **k):
        made.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **k)

    for stream, handle in ((side, side.cuda_stream), (side.cuda_stream, side.cuda_stream),
                           (0, torch.cuda.default_stream().cuda_stream)):
        del made[:]
        with monkeypatch.context() as m:
            m.setattr(torch, "empty", recorded)
            got = _call(name, *one, stream=stream)
        assert made and set(made) == {handle}
        assert torch.cuda.current_stream() == here
        torch.cuda.synchronize()
        for a, b in zip(got, _call(name, *one)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_a_call_on_an_idle_stream_right_after_one_on_the_current(name, raw):
    """The first call's workspace is free again on the host while its kernels run; the second, on a
    stream that waits for nothing, must not be given it."""
    import torch

    one, two = _problems()
    want = [_call(name, *p) for p in (one, two)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        first = _call(name, *one)
        second = _call(name, *two, stream=side.cuda_stream if raw else side)
        torch.cuda.synchronize()
        for got, ref in zip((first, second), want):
            for a, b in zip(got, ref):
                assert torch.equal(a, b)
        del first, second


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_memory_of_a_call_on_another_stream_is_not_reused_before_it_ends(name, raw):
    """Allocations on the current stream right after the call, of every size that it made, are
    written at once; the call's results stand."""
    import torch

    one, _ = _problems()
    want = _call(name, *one)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = _call(name, *one, stream=side.cuda_stream if raw else side)
        fills = [torch.full((n << 20,), 255, dtype=torch.uint8, device="cuda")
                 for n in (1, 2, 4, 8, 16, 32, 64, 128)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del fills, got
