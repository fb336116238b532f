"""The height of a call's tile, as the tests work it out, against sizes that were measured."""

from tests import _heights


def test_heights_of_known_calls():
    assert [_heights.mxfp4(M, 152064) for M in (64, 128, 1000, 4096)] == [64, 128, 256, 256]
    assert [_heights.xent(T, V) for T, V in ((48, 4000), (1000, 152064), (4096, 152064), (2000, 50257))] \
        == [64, 256, 256, 256]
    assert _heights.mxfp4(48, 32003) == 64
