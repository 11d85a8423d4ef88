"""How a caller says that nothing is shared: the call is then cut as mdss_cache_attention's (no GPU needed)."""
import pytest

import paper_2410_18234_amd as mdss
from test_abi_cache import desc


@pytest.mark.parametrize("max_own", [0, 500])
@pytest.mark.parametrize("S,n,hq", [(1, 1, 2), (4096, 1, 8), (60000, 2, 2), (300, 40, 64)])
def test_nothing_is_shared(S, n, hq, max_own):
    lib, T, width = mdss.load_library(), S * n, 100
    for most in (1, 63):
        want = lib.mdss_workspace_bytes_attention(desc(), T, S, width, hq, 1, n, most + max_own if max_own else 0)
        assert lib.mdss_workspace_bytes_attention_shared(desc(), T, S, S // 4, width, hq, 1, n, 4 * n, most, max_own) == want
    # unknown: two and more parts of every row
    assert lib.mdss_workspace_bytes_attention_shared(desc(), T, S, S // 4, width, hq, 1, n, 4 * n, 0, max_own) >= 2 * T * hq * 66 * 4
