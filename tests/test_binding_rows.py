"""What the binding says of rows that a call does not write.  No GPU."""
import pytest

import paper_2606_21023_amd as heal


@pytest.mark.parametrize("call", ["heal_kv_append", "heal_kv_read", "heal_kv_select", "heal_kv_attention", "heal_lora_add"])
def test_rows_of_no_sequence_are_named(call):
    """Each of these takes cu and may return a new tensor: whoever pads a batch behind cu[-1] has to
    know that those rows are not written."""
    said = " ".join(getattr(heal, call).__doc__.split()).lower()
    assert "no sequence" in said and "not written" in said
