"""Numbers of sequences and forks of which 32 bits would keep what looks right are refused (CPU: stand-ins for tensors)."""
import pytest

import paper_2510_15312_amd as vf
from test_more_devices import CALLS, I32, F32, WIDE, _tensors, current, reached  # noqa: F401

MANY = WIDE + 3
ROWS = dict(lens=(I32, MANY), block_table=(I32, MANY, 4), kv_len=(I32, MANY))


@pytest.mark.parametrize("which,specs", [
    (1, ROWS), (1, dict(src=(I32, WIDE + 2), dst=(I32, WIDE + 2), tokens=(I32, WIDE + 2), copies=(I32, WIDE + 2, 2))),
    (2, dict(ROWS, keep=(I32, MANY), copies=(I32, MANY, 2))), (3, dict(ROWS, table_out=(I32, MANY, 4))),
    (5, dict(row_off=(I32, MANY + 1), penalties=(F32, MANY, 3), history=(I32, MANY, 7), history_len=(I32, MANY), prompt_len=(I32, MANY)))])
def test_numbers_past_32_bits(reached, current, which, specs):  # noqa: F811
    call, tensors, more = CALLS[which]
    with pytest.raises(vf.VfError):
        call(**_tensors({name: spec for name, spec in dict(tensors, **specs).items() if name in tensors}, 1), **more)
    assert not reached
