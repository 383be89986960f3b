"""Scores so far apart that a row's output is the V of its best key: finite queries and keys give it at any size."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from kv_helpers import Batch  # noqa: E402
from paper_2608_25431_amd import gift  # noqa: E402


@pytest.fixture(scope="module")
def work():
    return gift.AttentionWork()


def best(b, scale):
    """Per row and head: V of the best key, its score, and whether 32-bit scores (over head_dim products) tell it from the
    others and leave them nothing (40 and more below it: e^-40 of 1500 keys is under 2^-45)."""
    q, k, v = (x.double().numpy() for x in b.parts())
    h, g, dim = b.cache.heads, b.group, b.cache.dim
    out, top, clear = np.zeros((q.shape[0], h * g, dim)), np.zeros((q.shape[0], h * g)), np.zeros((q.shape[0], h * g), bool)
    first = np.concatenate([[0], np.cumsum(b.lens)])
    for r, length in enumerate(b.lens):
        lo, hi = b.row_begin[r], b.row_begin[r + 1]
        for j in range(h * g):
            kk, vv = (np.concatenate([c[first[r]:first[r + 1], j // g].double().numpy(), d[lo:hi, j // g]])
                      for c, d in ((b.ck, k), (b.cv, v)))
            s = q[lo:hi, j] @ kk.T * scale
            s[:, length:][np.triu(np.ones((hi - lo, hi - lo), bool), 1)] = -np.inf
            e = (dim + 8) * 2.0 ** -24 * (np.abs(q[lo:hi, j]) @ np.abs(kk).T).max(1) * scale
            order = np.sort(s, 1)
            out[lo:hi, j], top[lo:hi, j] = vv[s.argmax(1)], order[:, -1]
            clear[lo:hi, j] = order[:, -1] - order[:, -2] > 2 * e + 40
    return out, top, clear


@pytest.mark.parametrize("dtype,q_scale,scale", [("bf16", 1e6, 0.1), ("bf16", 1e11, 0.1), ("bf16", 1e17, 1.0),
                                                 ("f16", 1e4, 1e4), ("f16", 1e4, 1e8)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("drafts", [[3, 2, 1], [14, 10, 9], [30, 20, 15], [70, 31, 49]])
def test_the_best_key_takes_all(work, dtype, q_scale, scale, dim, drafts):
    b = Batch([1500, 70, 5], drafts, dtype, heads=2, group=4, dim=dim, mask=None, seed=dim, q_scale=q_scale)
    want, top, clear = best(b, scale)
    assert clear.mean() > 0.8
    out, lse = (x.double().numpy() for x in b.run(work, scale=scale))
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    # the weight of the best key is 1 up to its own rounding, and so is the sum that divides by it
    u = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -11  # half the distance from 1 to the next number
    off = np.abs(out - want) - 2 * u * np.abs(want)
    assert (off[clear] <= 0).all(), f"{(off[clear] > 0).any(-1).mean():.2f} of the rows are wrong"
    assert (np.abs(lse - top) <= (dim + 16) * 2.0 ** -22 * np.abs(top))[clear].all()
