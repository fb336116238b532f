"""The cross entropy's workspaces are the parts that include/dart.h names, each at a multiple of 256
bytes; with chunks of a few rows too."""

import pytest

import paper_2509_23866_amd as dart


def _up(a, b):
    return -(-a // b)


def _parts(T, d, V, R):
    """Bytes that every call of R rows at a time has, and those of one with gradients."""
    both = [R * 4, R * _up(V, 128) * 16, R * _up(V, 128) * 4, T * 4, T * 4,
            _up(T, R) * _up(R, 32) * _up(d, 64) * 4096]
    return both, both + [R * _up(V, 8) * 16, T * d * 2] + ([V * d * 4] if R < T else [])


SIZES = [(1, 8, 1), (48, 512, 4000), (1000, 72, 4999), (4096, 3584, 152064), (5000, 200, 32003)]


@pytest.mark.parametrize("T,d,V", SIZES)
def test_forward(T, d, V):
    need = sum(_parts(T, d, V, T)[0])
    assert need <= dart.dart_lmhead_xent_fwd_workspace_bytes(T, d, V) <= need + 256 * 8


@pytest.mark.parametrize("T,d,V", SIZES)
def test_with_gradients(T, d, V):
    for chunk in (1, 2, 31, 32, 33, 100, 256, 257, 1024, T - 1, T, T + 1):
        R = min(chunk, T)
        if R < 1:
            continue
        need = sum(_parts(T, d, V, R)[1])
        got = dart.dart_lmhead_xent_workspace_bytes(T, d, V, chunk)
        assert need <= got <= need + 256 * 12 + (64 << 20)  # and dh in parts


def test_few_rows_a_chunk_take_more():
    """The panels at T = 4096, d = 3584: 28 MiB in chunks of 256 rows, 896 MiB in chunks of one."""
    of = lambda R: _parts(4096, 3584, 1, R)[0][-1] >> 20  # noqa: E731
    assert (of(256), of(32), of(8), of(1)) == (28, 28, 112, 896)
    size = lambda R: dart.dart_lmhead_xent_workspace_bytes(4096, 3584, 1, R)  # noqa: E731
    assert size(1) - size(32) > 800 << 20
