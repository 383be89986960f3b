"""Infinities and NaN in cached rows of V: every row of the request sees them, so they reach the elements that they are in,
whatever tile, round and number of waves they fall into, and nothing else."""
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


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("length", [33, 70, 150, 161, 250])  # the last cached tile shares its round with drafted ones
@pytest.mark.parametrize("drafts", [5, 12, 25, 50])          # 20, 48, 100 and 200 rows at a KV head
def test_cached_values_that_are_not_finite(work, dtype, dim, length, drafts):
    heads, group, element = 2, 4, 37
    b = Batch([length, 40], [drafts, drafts], dtype, heads=heads, group=group, dim=dim, mask="holes", seed=length)
    want, _, tol, _ = b.expect()
    hit = np.zeros(want.shape, bool)
    hit[:drafts, group:, element] = True  # rows of the first request at the second KV head
    for bad, place in ((float("nan"), length - 1), (float("inf"), length // 32 * 32 % length), (-float("inf"), 3)):
        row = b.cache.v[b.layer, int(b.tab[0, place // 16]), place % 16]
        was = float(row[1, element])
        row[1, element] = bad
        out, lse = (x.double().numpy() for x in b.run(work))
        row[1, element] = was
        assert not np.isfinite(out[hit]).any(), f"{bad} at {place}: {np.isfinite(out[hit]).sum()} outputs are finite"
        assert (np.abs(out - want) <= tol)[~hit].all() and np.isfinite(lse).all()
