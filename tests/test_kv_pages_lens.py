"""Lengths that are not there are refused by every call that reads them.  No GPU."""
import pytest

from test_kv_host import _batch
from test_kv_pages_host import FAKE, INVALID, OK, _compact, _fork, _release, _reserve

NO_COLUMNS = dict(table=None, table_cols=0)


@pytest.mark.parametrize("table", [dict(), NO_COLUMNS, dict(table=FAKE, table_cols=0)], ids=str)
def test_calls_without_lens_are_refused(table):
    """A table without columns included: reserving still looks each sequence up."""
    assert _release(lens=None, **table) == INVALID
    assert _fork(lens=None, **table) == INVALID
    assert _reserve(batch=_batch(lens=None), **table) == INVALID
    assert _reserve(batch=_batch(lens=None, cu=None, tokens=3, seqs=3), **table) == INVALID


def test_calls_that_do_not_read_lens_need_none():
    assert _release(rows=0, lens=None, **NO_COLUMNS) == OK
    assert _fork(rows=0, lens=None, **NO_COLUMNS) == OK
    # (compacting reads none: it is asked for its lists alone)
    assert _compact(count=None, **NO_COLUMNS) == INVALID
