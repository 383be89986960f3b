"""Arrays of the paged-cache calls that overlap or are not aligned to their elements, without a GPU: device addresses are made
up, since the C entry points refuse such arguments before they touch a device."""
import pytest

from paper_2608_25431_amd import gift
from test_kv_refusals import A, append, attention, lib, tables  # noqa: F401

# rows 6, heads 32, head_dim 128: out is 49152 bytes, lse 768; the cache is 4 * 10 * 65536 bytes from A on
CACHE = 4 * 10 * 65536
APART = dict(row_begin=20 * A, lens=21 * A, tables=22 * A, mask=23 * A, verdicts=24 * A)


@pytest.mark.parametrize("bad", [
    dict(lse=5 * A), dict(lse=5 * A + 49148), dict(lse=5 * A - 764), dict(lse=2 * A + 8), dict(lse=3 * A), dict(lse=4 * A + 4),
    dict(lse=A + CACHE - 4), dict(lse=20 * A + 8), dict(lse=21 * A + 4), dict(lse=22 * A + 28), dict(lse=23 * A + 20),
    dict(lse=24 * A - 760), dict(row_begin=5 * A), dict(lens=5 * A + 16), dict(tables=5 * A - 28), dict(mask=5 * A + 49148),
    dict(verdicts=5 * A + 400)])
def test_attention_outputs_that_overlap(lib, bad):  # noqa: F811
    assert attention(lib, **{**APART, **bad}) == gift.E_INVALID
    assert "overlap" in gift.last_error()


@pytest.mark.parametrize("bad", [dict(lse=6 * A + 2), dict(row_begin=20 * A + 1), dict(lens=21 * A + 2), dict(tables=22 * A + 3),
                                 dict(mask=23 * A + 2), dict(verdicts=24 * A + 1)])
def test_attention_arrays_that_are_not_aligned(lib, bad):  # noqa: F811
    assert attention(lib, **{**APART, **bad}) == gift.E_INVALID
    assert "aligned" in gift.last_error()


@pytest.mark.parametrize("bad", [dict(slots=6 * A + 4), dict(index=7 * A + 2), dict(slots=A), dict(slots=A - 8),
                                 dict(index=A + CACHE - 4)])
def test_append(lib, bad):  # noqa: F811
    assert append(lib, **bad) == gift.E_INVALID
    assert "aligned" in gift.last_error() or "overlap" in gift.last_error()


@pytest.mark.parametrize("bad", ["users", "lens", "new_lens", "free_blocks", "tables", "block_labels", "row_begin", "lens_out",
                                 "taken", "verdicts"])
def test_tables(lib, bad):  # noqa: F811
    assert tables(lib, **{bad: 40 * A + 2}) == gift.E_INVALID
    assert "aligned" in gift.last_error()
    assert tables(lib, slots=40 * A + 4) == gift.E_INVALID
