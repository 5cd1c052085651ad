"""Key rows that are found by the queries' row0 are as many as the query rows: other calls would read outside k and v, and are refused before any
launch (no GPU needed)."""
import ctypes as C

import pytest

from paper_2411_00853_amd import binding as sv

PLACE = 4096      # never dereferenced


def call(q_rows, k_rows, k=PLACE, k_row0=None):
    a = sv.spec_prompt_attn_args(PLACE, k, k, 512, 128, 128, 512, PLACE, k_row0, 8, 2, 64, 3, q_rows, k_rows, 0, 0, 0.125, PLACE)
    rc = sv.lib().spec_prompt_attention(C.byref(a), None, 0, None)
    return rc, sv.lib().spec_last_error()


@pytest.mark.parametrize("q_rows,k_rows", [(10, 9), (10, 11), (1, 2), (10, 0), (10, 2 ** 31 - 1)])
def test_other_numbers_of_rows_are_refused(q_rows, k_rows):
    rc, message = call(q_rows, k_rows)
    assert rc == -1 and b"k_row0" in message, (rc, message)


def test_no_key_rows_and_no_keys():
    rc, message = call(10, 0, k=None)
    assert rc == -1 and b"k_row0" in message, (rc, message)


def test_calls_without_rows_do_nothing():
    assert call(0, 9)[0] == 0       # nothing is read
