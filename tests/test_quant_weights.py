"""The weights of gift_quant_attention have the bits of gift_tree_attention's, 16 in bfloat16 and 11 in float16 down to 2^-29
of the largest, in every kernel that a call may take.  Queries are whole numbers, keys too and exact in 8 bits, so that scores
are exact; V is what its 8 bits stand for.  What is left of the bound is the weights' own rounding and the output's."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_tree_attention_weights import expected, inputs, nearest, truncated

gpu = pytest.mark.gpu
needs = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")


def cached(dtype, x):
    """The bytes of rows (n, dim) in the cache, of their factors, and the values they stand for."""
    from quant_helpers import quantised, rounded, values
    b, f = quantised(rounded(x, dtype), dtype)
    return b, f, values(b, f, dtype)


@pytest.mark.parametrize("dtype,mistake", [("bf16", nearest(torch.bfloat16)), ("bf16", truncated(8)), ("f16", truncated(9)),
                                           ("f16", nearest(torch.bfloat16))])
def test_the_bounds_see_weights_of_fewer_bits(dtype, mistake):
    q, k, v = inputs(100, 200, 64, 1)
    v = cached(dtype, v)[2]
    want, _, tol, _ = expected(dtype, q, k, v, 0.125)
    wrong = expected(dtype, q, k, v, 0.125, mistake)[0]
    assert (np.abs(wrong - want) > tol).any()


def check(dtype, q, k, v, work, rows, requests=1, block=16):
    """The last `rows` tokens of one request, which all of them see.  More requests are the same again, over the same blocks."""
    from kv_helpers import DEV, DT, i32
    from paper_2608_25431_amd import gift
    from quant_helpers import NAN, QuantCache
    (keys, dim), t = k.shape, DT[dtype]
    n = -(-keys // block)
    cache = QuantCache(1, dim, block, n + 1)
    ids = np.random.default_rng(3).permutation(n + 1)[:n]
    exact = []
    for x, elements, factors in ((k, cache.k, cache.kf), (v, cache.v, cache.vf)):
        b, f, value = cached(dtype, x)
        exact.append(value)
        for to, what, fill in ((elements, b, NAN), (factors, np.pad(f, ((0, 0), (0, cache.space - f.shape[1]))), 255)):
            pad = np.full((n * block, what.shape[1]), fill, np.uint8)
            pad[:keys] = what
            to[0, torch.from_numpy(ids).to(DEV), :, 0] = torch.from_numpy(pad).view(n, block, -1).to(DEV)
    assert (exact[0] == k).all()
    group = len(q) // rows
    dq = torch.from_numpy(q).to(t).view(rows, group, dim).to(DEV).repeat(requests, 1, 1)
    out, lse = torch.empty_like(dq), torch.empty(rows * requests, group, device=DEV)
    mask = torch.full((rows * requests, -(-rows // 32)), -1, dtype=torch.int32, device=DEV)
    gift.quant_attention(work, *cache.args(), 0, dq, i32(np.arange(requests + 1) * rows), i32([keys] * requests),
                         i32(np.tile(ids, (requests, 1))), out, mask=mask, lse=lse, scale=0.125)
    want, ends, tol, etol = expected(dtype, q, k, exact[1], 0.125, chain=256 if requests == 1 else keys)
    off = np.abs(out.cpu().double().numpy().reshape(requests, *want.shape) - want)
    assert (off <= tol).all(), f"{(off > tol).mean():.3g} outside, worst {np.max(off / tol):.3g} of the bound"
    assert (np.abs(lse.cpu().double().numpy().reshape(requests, -1) - ends) <= etol).all()


@pytest.fixture(scope="module")
def work():
    from paper_2608_25431_amd import gift
    w = gift.AttentionWork()
    yield w
    w.destroy()


@gpu
@needs
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
# times 4 query heads: tiles of 16 columns, eight waves a workgroup and four, then each number of waves that share keys
@pytest.mark.parametrize("rows,requests", [(1, 1), (1, 300), (5, 1), (12, 1), (25, 1), (60, 1)])
@pytest.mark.parametrize("keys", [100, 200])
def test_bits_of_weights(work, dtype, dim, rows, requests, keys):
    q, k, v = inputs(4 * rows, keys, dim, dim + rows)
    check(dtype, q, k, v, work, rows, requests)


@gpu
@needs
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("octaves", [12, 20, 26, 28])
@pytest.mark.parametrize("rows,keys,dim", [(1, 40000, 64), (30, 8192, 128)])
def test_many_keys_far_below_one(work, dtype, octaves, rows, keys, dim):
    # attention sinks: one key holds most of the weight and has no part in the output
    q, k, v = inputs(4 * rows, keys, dim, 5, sink=round(octaves * np.log(2) / dim / 0.125 * 2) / 2)
    check(dtype, q, k, v, work, rows)
