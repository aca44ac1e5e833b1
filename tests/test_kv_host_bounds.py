"""Sizes of the key/value cache's calls whose products do not fit in 64 bits.  No GPU."""
import ctypes

import pytest

import paper_2606_21023_amd as heal
from test_kv_host import FAKE, INVALID, _append, _attention, _batch, _cache


@pytest.mark.parametrize("n_sel", [1 << 25, 1 << 57, 1 << 58, (1 << 58) + 1, (1 << 60) + 2, (1 << 63) - 1])
def test_a_list_longer_than_any_sequence_is_refused(n_sel):
    """n_sel blocks of 64 tokens are 2^31 or more, or their number wraps to 0, 64 or 128."""
    assert _attention(sel=FAKE, n_sel=n_sel) == INVALID
    c, b = ctypes.byref(_cache()), ctypes.byref(_batch())
    assert heal.lib().heal_kv_attention_workspace(c, b, 4, 0, n_sel, 0) == -1
    assert heal.lib().heal_kv_attention_tile(c, b, 4, 0, n_sel, 0) == 0


@pytest.mark.parametrize("call", ["attention", "append"])
def test_outputs_that_overlap_at_far_strides_are_refused(call):
    """Two heads of 2^30 tokens, one stride for both: (2^30 - 1) 2^34 wraps to -2^34."""
    batch, s = _batch(tokens=1 << 30, table_cols=1, table_ld=1), 1 << 34
    if call == "attention":
        assert _attention(batch=batch, heads_q=2, out_token=s, out_head=s) == INVALID
    else:
        assert _append(batch=batch, heads_q=2, qo_token=s, qo_head=s) == INVALID
