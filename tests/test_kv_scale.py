"""The scale of the attention: what its product with log2(e) holds in 32 bits, on the host."""
import math

import pytest

from paper_2609_36601_amd import binding as b
from tests.test_kv_abi import heads, lib, pool, table, tokens  # noqa: F401


@pytest.mark.parametrize("scale,taken", [(2.0**127, True), (-2.0**127, True), (2.0**127 * (1 + 2.0**-23), False), (-2.5e38, False),
                                         (3.4e38, False), (math.inf, False), (-math.inf, False), (math.nan, False),
                                         (0.0, True), (2.0**-149, True)])
def test_scales(lib, scale, taken):  # noqa: F811
    h = heads()
    # without a workspace: what is taken so far is refused for that, before a device is touched
    st = lib.saki_kv_attention(table(), pool(), 0, tokens(), 2, h, h, None, scale, 0, 0, None, 0, None)
    assert st == (6 if taken else 3) and b.STATUS[st] == ("SAKI_E_WORKSPACE" if taken else "SAKI_E_VALUE")
