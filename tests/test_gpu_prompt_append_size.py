"""Numbers of rows that no launch takes."""
import pytest

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk", [(1, 1), (2, 1), (4, 2), (32, 8)])
@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16])
def test_too_many_rows_are_refused(hq, hk, rows):
    """Their number is beyond what a launch's grid holds; refused before anything runs."""
    h, _, _ = ref.handle(1, hq, hk, 64, 3, 96)
    x, row0, slot = ref.normal(1, 4, (hq + 2 * hk) * 64, dtype=ref.BF16), ref.ints([0, 4]), ref.ints([0])
    ld = x.shape[1]
    rc = sv.lib().spec_prompt_append(h.ptr, 0, sv._ptr(x), ld, sv._ptr(x), ld, sv._ptr(row0), sv._ptr(slot), None, 1, rows, None)
    assert rc == -2 and b"too many" in sv.lib().spec_last_error()
