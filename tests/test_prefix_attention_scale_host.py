"""CPU check of prefix_attention's scale: one whose product with log2(e) overflows fp32 is refused."""
import pytest

from test_prefix_attention_host import _call, _desc, ll  # noqa: F401  (ll: a fixture)


@pytest.mark.parametrize("scale", [2.0 ** 127, 2.5e38, 3.4e38])
def test_scales_past_the_range_are_refused(ll, scale):  # noqa: F811
    assert _call(ll, _desc(ll, scale=scale), ws_bytes=16) == 1
    assert _call(ll, _desc(ll, scale=2.0 ** 127 * (1 - 2.0 ** -24)), ws_bytes=16) == 7      # the next refusal
