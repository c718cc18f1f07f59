"""More of what the paged operators refuse (tests/test_paged_refusals.py): no GPU needed, the addresses are never followed."""
import pytest

from paper_2603_09215_b200 import binding as B
from tests import test_paged_refusals as base


@pytest.mark.parametrize("bad", [dict(status=base.A + 2), dict(inject_short_copy=-1)])
def test_attention_refuses_status(bad):
    assert base.attend(base.attn_args(status=base.A)) == B.OK  # (no rows)
    assert base.attend(base.attn_args(**bad)) == B.EINVAL


@pytest.mark.parametrize("rows,ids", [((1 << 28), 40000), ((1 << 29) + 1, 262144), ((1 << 31) - 1, 8193)])
def test_sample_refuses_more_rows_than_a_launch_numbers(rows, ids):
    """(Their count times the CTAs of a row would come round to a few.)"""
    assert base.call("sparsk_sample", base.sample_args(n_rows=rows, n_ids=ids, row_stride=0)) == B.ECAPACITY
