"""The plan of the cross entropy's chunks for sizes that the call refuses: the refusal is the call's,
as without gradients."""

import paper_2509_23866_amd as dart


def test_plan_of_an_empty_call():
    assert dart.lmhead_xent_plan(5, 0) == 5
    assert dart.lmhead_xent_plan(0, 5) == 0
    assert dart.lmhead_xent_plan(0, 0) == 0
