"""rope_kv_append on both sides of the number of tokens at which a workgroup takes a whole token."""
import pytest

import test_kv_append_gpu as append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["f16", "int4"])
@pytest.mark.parametrize("M", [767, 768, 2049])
@pytest.mark.parametrize("heads,hk,D,page,axes,sections,R,interleaved", [
    (9, 3, 128, 16, 3, (16, 24, 24), 128, False), (4, 2, 64, 32, 1, None, 32, True),
    (5, 1, 256, 64, 2, (100, 28), 256, False)])
def test_tokens(M, heads, hk, D, page, axes, sections, R, interleaved, fmt):
    append.test_append(M, heads, hk, D, page, axes, sections, R, interleaved, fmt)
