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


@pytest.mark.parametrize("n,nhi", [(24, 60), (7, 3000)])
def test_no_block_is_lost(n, nhi):
    # steps with wrong ids in the list and tables that name foreign blocks: what a caller finds by the rules of release is
    # every block of the cache, once
    r = np.random.default_rng(n)
    c = make(r, n, 16, 1, 200, 1, nhi, 4, extra_width=600, spare=0)
    n_blocks = len(c["labels"])
    outside = 0x7FFFFFFF
    cached = c["tab"][c["tab"] < n_blocks]
    c["free"] = np.concatenate([c["free"], np.setdiff1d(np.arange(n_blocks), np.concatenate([c["free"], cached]))])
    seen = set()
    for step in range(12):
        mixed = r.permutation(n)[:2]
        kept = {}
        for b in mixed:  # the caller's own record of what the entry held
            if c["lens"][b]:
                kept[b] = c["tab"][b, 0]
                c["tab"][b, 0] = c["tab"][(b + 1) % n, 0] if c["users"][b] != c["users"][(b + 1) % n] else n_blocks
        wrong = r.integers(0, max(1, len(c["free"])))
        c["free"] = np.insert(c["free"], wrong, n_blocks + step)
        c["new"] = r.integers(0, nhi + 1, n) * (r.random(n) < 0.5)
        c["n_slots"] = int(c["new"].sum())
        got = run(c)
        c["tab"], c["labels"] = got["tables"].view(np.uint32).astype(np.int64), got["labels"].view(np.uint32).astype(np.int64)
        c["lens"], taken = got["lens_out"].astype(np.int64), int(got["taken"][0])
        seen |= set(got["verdicts"].tolist())
        for b, block in kept.items():
            c["tab"][b, 0] = block
        left = c["free"][:taken]
        left = left[left < n_blocks]
        c["free"] = np.concatenate([c["free"][taken:], left[c["labels"][left] == gift.LABEL_UNOWNED]])
        c["free"] = c["free"][c["free"] < n_blocks]
        for b in range(n):
            if got["verdicts"][b] == gift.SEG_OWNER_MIXED or r.random() < 0.2:  # released; another request comes in its place
                held = c["tab"][b][c["tab"][b] < n_blocks]
                assert (c["labels"][held] == c["users"][b]).all()
                c["labels"][held] = gift.LABEL_UNOWNED
                c["free"] = np.concatenate([c["free"], held])
                c["tab"][b], c["lens"][b] = outside, 0
        held = c["tab"][c["tab"] < n_blocks]
        everywhere = np.sort(np.concatenate([c["free"], held]))
        assert (everywhere == np.arange(n_blocks)).all(), f"step {step}: blocks lost or held twice"
        assert (c["labels"][c["free"]] == gift.LABEL_UNOWNED).all()
    assert seen == {gift.SEG_OK, gift.SEG_OWNER_MIXED, gift.SEG_NO_SPACE}
