"""More of attention's refusals at the C entry; no GPU is used."""
import pytest

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests.test_attention_ops import BAD, FAKE, NULL, call  # noqa: E402


@pytest.mark.parametrize("back", [False, True])
def test_key_heads_without_a_query_head(back):
    """Nothing would write their gradients."""
    assert call(back, h=0, kv=2) == BAD and call(back, h=0, kv=1, batch=1, seq=1) == BAD
    assert call(back, h=0, kv=0) == pamm.OK
