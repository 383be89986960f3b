"""gift_kv_tables where space is short: what still gets its verdict, and where the blocks are that left the free list."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from test_kv_tables import make, run  # noqa: E402
from paper_2608_25431_amd import gift  # noqa: E402


@pytest.mark.parametrize("n,hi,nhi", [(40, 70, 40), (12, 400, 3000), (6, 50, 60000)])
def test_requests_that_add_nothing_need_no_slots(n, hi, nhi):
    r = np.random.default_rng(n)
    c = make(r, n, 16, 1, hi, nhi // 2, nhi, 3)
    c["new"][1::2] = 0
    c["n_slots"] = int(c["new"][:n // 2].sum()) - 1  # the rows of the last one that adds something there pass the array
    last = (n // 2 - 1) // 2 * 2
    got = run(c)
    want = [gift.SEG_OK if b < last or c["new"][b] == 0 else gift.SEG_NO_SPACE for b in range(n)]
    assert got["verdicts"].tolist() == want
    assert (got["lens_out"] == c["lens"] + np.where(np.array(want) == gift.SEG_OK, c["new"], 0)).all()
