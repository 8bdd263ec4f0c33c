"""CPU checks of dbw_adamw_step's small arguments: what the kernel reads as 4-byte words has to lie on 4 bytes."""
import pytest

from paper_2004_14696_gb300 import dbw
from test_block_refusals import P, STEP, call, lib  # noqa: F401


@pytest.mark.parametrize("change", [dict(t=P + 2), dict(grad_scale=P + 1), dict(status=P + 2)])
def test_pointers_off_their_elements_are_refused(lib, change):  # noqa: F811
    got, text = call(lib, "dbw_adamw_step", STEP, **change)
    assert got == dbw.DBW_EALIGN and text.startswith("dbw_adamw_step:"), (got, text)
