"""More of what the paged operators refuse (tests/test_paged_refusals.py): no GPU needed, the addresses are never followed."""
import pytest

from paper_2603_09215_b200 import binding as B
from tests import test_paged_refusals as base


@pytest.mark.parametrize("bad", [dict(status=base.A + 2), dict(inject_short_copy=-1)])
def test_attention_refuses_status(bad):
    assert base.attend(base.attn_args(status=base.A)) == B.OK  # (no rows)
    assert base.attend(base.attn_args(**bad)) == B.EINVAL
