"""gift_kv_tables and who owns what it takes: free lists that name blocks which somebody owns or the same block for two
users; tables that name free blocks.  No block comes to two users or changes its owner."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from kv_helpers import expect_tables  # noqa: E402
from test_kv_tables import make, run  # noqa: E402
from paper_2608_25431_amd import gift  # noqa: E402


def users_of_their_own(c):
    """Every request its own user."""
    n = len(c["lens"])
    c["users"] = np.arange(n)
    c["labels"][:] = gift.LABEL_UNOWNED
    for b in range(n):
        c["labels"][c["tab"][b, :-(-c["lens"][b] // c["block"])]] = b
    return c


def need(c):
    return -(-(c["lens"] + c["new"]) // c["block"]) - -(-c["lens"] // c["block"])


def same(got, want):
    for k in want:
        w = want[k] if k == "slots" else want[k].astype(np.uint32).view(np.int32)
        assert (got[k] == w).all(), f"{k}: {(got[k] != w).sum()} differ, first at {np.argwhere(got[k] != w)[:1].tolist()}"


def conserved(c, got):
    """Every block that left the list is in the table of a request of its owner, or nobody's; a block that had an owner has
    the same one."""
    labels, tables = got["labels"].view(np.uint32), got["tables"].view(np.uint32)
    had = c["labels"] != gift.LABEL_UNOWNED
    assert (labels[had] == c["labels"][had]).all()
    have, want = -(-c["lens"] // c["block"]), -(-(c["lens"] + c["new"]) // c["block"])
    entered = tables != c["tab"].astype(np.uint32)
    col = np.arange(tables.shape[1])
    assert not entered[(col < have[:, None]) | (col >= want[:, None])].any()
    ids, req = tables[entered], np.nonzero(entered)[0]
    assert (labels[ids] == c["users"][req]).all()
    new = np.nonzero(~had & (labels != gift.LABEL_UNOWNED))[0]
    assert set(new.tolist()) <= set(ids.tolist())
    assert set(ids.tolist()) <= set(c["free"][:got["taken"][0]].tolist())
    refused = ~entered.any(1) & (want > have)
    assert (got["verdicts"][refused] != gift.SEG_OK).all()


@pytest.mark.parametrize("n,hi,nhi", [(30, 60, 40), (12, 400, 3000), (4, 100, 60000)])  # each number of threads a request
def test_blocks_of_other_owners_are_not_taken(n, hi, nhi):
    r = np.random.default_rng(n)
    c = users_of_their_own(make(r, n, 16, 1, hi, nhi // 2, nhi, 4))
    at = np.cumsum(need(c))  # where the requests' shares of the list end
    assert at[-1] == len(c["free"])
    c["free"][at[0] - 1] = c["tab"][1, 0]             # somebody's block, as the last one of a claim
    c["free"][at[1]] = c["tab"][n - 1, 0]
    c["labels"][c["free"][at[2]]] = gift.LABEL_PARAM  # model parameters
    owned = np.isin(np.arange(len(c["free"])), [at[0] - 1, at[1], at[2]])
    # to the request, such a block is what an id outside the cache is
    want = expect_tables(c["users"], c["lens"], c["new"], 16, np.where(owned, len(c["labels"]), c["free"]), c["tab"],
                         c["labels"], c["n_slots"])
    assert (want["verdicts"][[0, 2, 3]] == gift.SEG_NO_SPACE).all() and (want["verdicts"] == gift.SEG_OK).sum() == n - 3
    got = run(c)
    same(got, want)
    conserved(c, got)


@pytest.mark.parametrize("n,nhi", [(9, 400), (9, 9000), (3, 200000)])
def test_a_refused_request_gives_back_what_was_nobodys(n, nhi):
    r = np.random.default_rng(n)
    c = users_of_their_own(make(r, n, 16, 30, 300, nhi // 2, nhi, 1))
    at = np.concatenate([[0], np.cumsum(need(c))])
    for b in range(0, n, 2):
        mine, theirs = at[b] + (at[b + 1] - at[b]) // 3, at[b + 1] - 1
        c["labels"][c["free"][mine]] = b                       # the user's own, in use elsewhere: it stays so
        c["labels"][c["free"][theirs]] = n + 5                 # another's: the request is refused
    got = run(c)
    conserved(c, got)
    assert (got["verdicts"][::2] == gift.SEG_NO_SPACE).all() and (got["verdicts"][1::2] == gift.SEG_OK).all()
    for b in range(0, n, 2):
        share = c["free"][at[b]:at[b + 1]]
        assert (got["labels"][share].view(np.uint32) == c["labels"][share]).all()


@pytest.mark.parametrize("n,hi,nhi", [(300, 60, 40), (12, 400, 3000), (4, 100, 60000)])
def test_a_step_that_is_run_again(n, hi, nhi):
    r = np.random.default_rng(n)
    c = make(r, n, 16, 1, hi, 0, nhi, 4)
    want = expect_tables(c["users"], c["lens"], c["new"], 16, c["free"], c["tab"], c["labels"], c["n_slots"])
    same(run(c), want)
    c["tab"], c["labels"] = want["tables"], want["labels"]
    same(run(c), want)


@pytest.mark.parametrize("n,nhi", [(40, 40), (9, 9000), (3, 50000)])
def test_ids_that_the_list_gives_to_two_users(n, nhi):
    r = np.random.default_rng(n)
    for _ in range(6):
        c = users_of_their_own(make(r, n, 16, 0, 0, nhi // 2, nhi, 1))
        at = np.concatenate([[0], np.cumsum(need(c))])
        twice = r.permutation(n)[:n // 3 * 2].reshape(2, -1)
        for a, b in twice.T:
            c["free"][r.integers(at[a], at[a + 1])] = c["free"][r.integers(at[b], at[b + 1])]
        got = run(c)
        conserved(c, got)
        ok = got["verdicts"] == gift.SEG_OK
        assert not (ok[twice[0]] & ok[twice[1]]).any() and np.delete(ok, twice).all()


@pytest.mark.parametrize("n,hi", [(64, 200), (12, 20000)])
def test_tables_that_name_free_blocks(n, hi):
    r = np.random.default_rng(n)
    for seed in range(10):
        c = users_of_their_own(make(r, n, 16, 100, hi, 17, 40, 1))
        have = -(-c["lens"] // 16)
        for b in range(0, n, 3):   # names a block that another user's request takes in this step
            c["tab"][b, r.integers(0, have[b])] = c["free"][-1 - (b % 2)] if b < n // 2 else c["free"][b % 2]
        got = run(c)
        conserved(c, got)
        # the first and the last requests may have taken such a block themselves; the others named somebody else's
        assert (got["verdicts"][3:n - 3:3] == gift.SEG_OWNER_MIXED).all()
        assert (np.delete(got["verdicts"], np.arange(0, n, 3)) == gift.SEG_OK).all()


@pytest.mark.parametrize("n,nhi", [(20, 60), (5, 9000)])
def test_labels_that_no_user_has(n, nhi):
    # blocks of the model's parameters, or nobody's, are not a request's because it says so
    r = np.random.default_rng(n)
    c = users_of_their_own(make(r, n, 16, 30, 300, nhi // 2, nhi, 1))
    for b, label in ((1, gift.LABEL_UNOWNED), (3, gift.LABEL_PARAM)):
        c["users"][b] = label
        c["labels"][c["tab"][b, :-(-c["lens"][b] // 16)]] = label
    got = run(c)
    conserved(c, got)
    assert got["verdicts"].tolist() == [gift.SEG_OWNER_MIXED if b in (1, 3) else gift.SEG_OK for b in range(n)]
    rows = got["row_begin"]
    for b in (1, 3):
        assert (got["tables"][b] == c["tab"][b].astype(np.uint32).view(np.int32)).all()
        assert (got["slots"][rows[b]:rows[b + 1]] == -1).all() and got["lens_out"][b] == c["lens"][b]
