"""Calls of linear attention, layer norm and clipping that their documentation allows: sizes, places and values that other tests do not have."""
import ctypes as C
import itertools

import pytest
import torch

from paper_2202_13638_amd import binding
from test_more_operators import _attention_struct

gpu = pytest.mark.gpu


# segments are a number of chunks of rows that depends on the type: of eight and of four chunks, 16 bits keep what 32 bits make odd
@pytest.mark.parametrize("heads,states", [(8, 8), (16, 8), (4, 1), (8, 2), (1, 1)])
def test_work_spaces_are_for_every_type(heads, states):
    """What bagel_linear_attention_workspace says without a type is enough for each.  (The calls are refused, for the place of the work space, before anything is launched.)"""
    for rows, sequences, grad in itertools.product(list(range(1000, 70000, 1777)) + [15000, 30000, 31000, 32000], [1, 2, 50], [False, True]):
        size = binding.bagel_linear_attention_workspace(rows, sequences, heads, states, 64, 64, grad)
        for dtype, offsets in itertools.product([0, 1, 2], [None, 0x10000]):
            if offsets is None and rows % sequences:
                continue
            a = _attention_struct(rows=rows, sequences=sequences, heads=heads, states=states, key_width=64, value_width=64, dtype=dtype, offsets=offsets,
                                  workspace=0x10004, workspace_bytes=size)
            for k in ("query", "key", "value", "out", "d_out", "d_query", "d_key", "d_value"):
                setattr(a, k + "_head", 64)
                setattr(a, k + "_stride", 64 * heads)
            lib = binding.load()
            assert (lib.bagel_linear_attention_grad if grad else lib.bagel_linear_attention)(C.byref(a), None) == binding.EINVAL
            assert b"16 bytes" in lib.bagel_last_error(None), (rows, sequences, dtype, offsets, lib.bagel_last_error(None))
