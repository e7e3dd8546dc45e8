"""Sizes at which a kernel's 32-bit positions would wrap are refused on the host, before any launch (CPU)."""
import pytest

from paper_2609_32869_gb300 import binding as B
from test_beam_refusals import _attend, _plan, _status


@pytest.mark.parametrize("max_len", [2 ** 31 - 1, 2 ** 31 - 1023])
def test_attention_positions(max_len):
    """A warp steps up to 255 positions past the last one it sees, and a step is 64 wide.  One table row (stride 0)
    bounds nothing here."""
    assert _status(_attend, max_len=max_len, table_stride=0) == B.WF_ERR_UNSUPPORTED
    assert B.wf_kv4_attention_scratch_bytes(1, 1, 4, 2, 64, max_len) == 0


def test_attention_longest_has_a_size():
    assert B.wf_kv4_attention_scratch_bytes(1, 1, 4, 2, 64, 2 ** 31 - 1024) > 0


@pytest.mark.parametrize("cap", [2 ** 31 - 1, 2 ** 31 - 2 ** 20])
def test_plan_slots(cap):
    """The slots after the last token are filled by the whole grid, 256 a CTA and up to 1024 CTAs at a time."""
    assert _status(_plan, cap=cap) == B.WF_ERR_UNSUPPORTED
