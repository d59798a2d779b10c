"""Host side of the constraints on logits (no GPU): an empty list has no address (a tensor of no numbers has none), and what goes with it may still be there."""
import ctypes as C

import pytest

from paper_2503_08524_b200 import binding as B
from test_block8_host import logits_args


@pytest.mark.parametrize("history", [None, "there"])
def test_an_empty_history_may_have_companions(history):
    kw = dict(n_rows=0, n_history=0)                     # (no rows: nothing is enqueued)
    if history is None:
        kw["history_dev"] = None
    assert B.LIB.d3_constrain_logits(C.byref(logits_args(**kw)), None) == B.OK


def test_an_empty_list_of_biases_has_no_address():
    assert B.LIB.d3_constrain_logits(C.byref(logits_args(n_rows=0, n_bias=0, bias_ids_dev=None, bias_dev=None)), None) == B.OK
    assert B.LIB.d3_constrain_logits(C.byref(logits_args(n_bias=4, bias_ids_dev=None)), None) == B.EINVAL


def test_a_history_with_entries_needs_its_address():
    assert B.LIB.d3_constrain_logits(C.byref(logits_args(history_dev=None)), None) == B.EINVAL
