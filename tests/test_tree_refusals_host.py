"""Arguments of calls on trees that used to pass the checks and gave wrong numbers (no GPU: no pointer is followed)."""
import pytest

from test_tree_abi_host import EINVAL, EWORKSPACE, attention, ctx, lib


@pytest.mark.parametrize("sign", [1, -1])
def test_scales_that_overflow_with_the_base(lib, ctx, sign):
    """Scores are taken to base 2: scale times log2(e) has to be finite."""
    assert attention(lib, ctx, scale=sign * 2.3e38) == EWORKSPACE
    assert attention(lib, ctx, scale=sign * 2.4e38) == EINVAL
