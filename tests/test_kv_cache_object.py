"""heal.KVCache keeps the addresses that it was made with.  No GPU."""
import pytest

import paper_2606_21023_amd as heal
from test_kv_host import _arrays

NAMES = ("k_codes", "v_codes", "scales", "k_mean", "k_recent", "v_recent")


def test_its_arrays_cannot_be_exchanged():
    """The calls would go on with the old memory, which may be another tensor's by then."""
    arrays = _arrays()
    c = heal.KVCache(*arrays)
    for name, old, new in zip(NAMES, arrays, _arrays()):
        with pytest.raises(heal.HealError):
            setattr(c, name, new)
        with pytest.raises(heal.HealError):
            delattr(c, name)
        assert getattr(c, name) is old
    for name in ("blocks", "slots", "heads", "dim", "block", "device", "anything"):
        with pytest.raises(heal.HealError):
            setattr(c, name, 1)
    assert (c.blocks, c.slots, c.heads, c.dim, c.block) == (3, 2, 2, 64, 16)
