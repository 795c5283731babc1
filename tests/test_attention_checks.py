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


@pytest.mark.parametrize("back", [False, True])
def test_written_rows_that_begin_where_a_tensor_does(back):
    """The log-sums of the forward call and the workspace of the backward call are written while the tensors are read."""
    names = ("dO", "Q", "K", "V", "O", "dQ", "dK", "dV") if back else ("Q", "K", "V", "O")
    apart = {n: dict(data=FAKE * (i + 4)) for i, n in enumerate(names)}
    for n in names:
        where = apart[n]["data"]
        assert call(back, **apart, **(dict(ws=where, lse=FAKE * 2) if back else dict(lse=where))) == BAD, n
    if back:
        assert call(back, **apart, ws=FAKE * 2, lse=FAKE * 2) == BAD
