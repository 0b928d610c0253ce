"""Calls of rope, cache_read and verify_drafts that ask for nothing, or for more than a launch takes (no GPU needed)."""
import pytest

from paper_2605_19660_amd import binding as ob
from test_new_tokens_refusals import cache_struct, read


def test_reading_neither_keys_nor_values_is_the_abi_s_error():
    with pytest.raises(ob.OscarError) as e:
        ob.cache_read(None)
    assert e.value.status == ob.ERR_INVALID_ARG
    assert read(cache_struct(), k=None, v=None) == ob.ERR_INVALID_ARG


def test_a_read_past_what_a_launch_takes_is_refused():
    c = cache_struct(max_pages=1 << 24, num_pages=1 << 24, batch=1)
    assert read(c, T=(1 << 31) - 1) == ob.ERR_INVALID_ARG
