"""Host-side checks of the decode entry points and of their binding that need no GPU, beside test_decode_abi.py."""
import pytest

from paper_2607_25291_amd import binding as B


def refused(status, call, *a, **kw):
    with pytest.raises(B.CosaError) as e:
        call(*a, **kw)
    assert e.value.status == status, str(e.value)


def test_outputs_of_an_empty_page_map_must_not_overlap():
    def call(cu=None, slots=None, rows=0, taken=None):
        B.cosa_page_map(0, 16, 8, None, None, None, 0, None, None, None, cu, slots, rows, taken, stream=0)
    call()
    call(rows=9)  # nothing to write to
    for kw in (dict(cu=4096, taken=4096), dict(cu=4096, slots=4088, rows=2), dict(taken=4096 + 8 * 9 - 4, slots=4096, rows=9)):
        refused(B.COSA_ERR_INVALID_ARG, call, **kw)
        assert "overlap" in B.cosa_last_error()
