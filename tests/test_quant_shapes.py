"""gift_quant_attention in the kernels that a call takes by the rows of a request, the number of its columns and the size of a
head: each with causal and masked rows, requests of many lengths in one call, lengths that end inside tiles and blocks."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

gpu = pytest.mark.gpu
needs = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
pytestmark = [gpu, needs]


@pytest.fixture(scope="module")
def work():
    from paper_2608_25431_amd import gift
    w = gift.AttentionWork()
    yield w
    w.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
# at 2 query heads a KV head 24 rows on average, and 143
@pytest.mark.parametrize("rows", [[20, 1, 25, 2], [140, 3]])
@pytest.mark.parametrize("mask", [None, "tree"])
def test_keys_shared_by_one_wave_and_by_eight(work, dtype, dim, rows, mask):
    from quant_helpers import Requests
    r = Requests(np.array([1, 231, 100, 77])[:len(rows)] + rows, rows, dtype, 1, 2, dim, 16, mask=mask)
    r.check(r.run(work))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("longest", [300, 1500])  # columns that stay whole, and that are divided
def test_more_single_tokens_than_workgroups_of_eight_waves(work, dtype, dim, longest):
    from quant_helpers import Requests
    r = np.random.default_rng(dim)
    lens = r.integers(1, 300, 130)
    lens[40] = longest
    q = Requests(lens, np.ones(130, np.int64), dtype, 2, 2, dim, 16, order="token")
    q.check(q.run(work))
