"""The weights of gift_tree_attention have the bits that it states: 16 in bfloat16, 11 in float16 down to 2^-29 of the
largest.  Queries and keys are small whole numbers, so that scores are exact, and what is left of the bound is the weights'
own rounding and the output's."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
needs = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")

# of an output: half the distance from 1 to the next number
U = {"bf16": torch.finfo(torch.bfloat16).eps / 2, "f16": torch.finfo(torch.float16).eps / 2}
WEIGHT = {"bf16": 2.0 ** -16, "f16": 2.0 ** -11}  # of a weight: what the header states


def inputs(rows, keys, dim, seed, sink=None):
    """q, k, v of one head.  sink: key 0 has this score above 0, all others about 0, and its V is 0."""
    r = np.random.default_rng(seed)
    q, k, v = r.integers(-1, 2, (rows, dim)), r.integers(-2, 3, (keys, dim)), r.standard_normal((keys, dim))
    if sink is not None:
        q[:] = r.integers(0, 2, dim) * 2 - 1  # the same for all rows, so that one key can be far above for all
        k = r.integers(-1, 2, (keys, dim))
        k[0] = q[0] * sink
        v += 0.5
        v[0] = 0
    return q.astype(np.float64), k.astype(np.float64), v


def expected(dtype, q, k, v, scale, rounding=None, chain=256):
    """(out, lse, bound on out, bound on lse) in 64 bits.  rounding: a mistake to plant, applied to weights with the largest
    at 1.

    Scores are whole numbers below 2^24, exact in 32 bits.  An exponent c (s - m) has the rounding of c (2^-24 of it), of
    c m and of the sum (2^-24 of each); the exponential itself 2^-21.  So e = 3 ln 2 2^-24 c (|s| + |m|) + 2^-21, once for
    the weights that are multiplied by V and once for their sum.  Sums are in 32 bits: with one column of rows a workgroup
    has at most two rounds, in which a wave adds 128 keys; four waves and two times up to 64 parts are joined: fewer than 256
    roundings of 2^-24 one after the other, and no more than there are keys (chain).  float16 weights below 2^-29 of the largest are
    off by up to 2^-40 of it."""
    s = q @ k.T * scale
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    total = p.sum(1, keepdims=True)
    w = p if rounding is None else rounding(p)
    out = w @ v / total
    part = p @ np.abs(v) / total
    sums = min(len(k), chain) * 2.0 ** -24
    e = 3 * 2.0 ** -24 * (np.abs(s).max(1, keepdims=True) + np.abs(m)) + 2.0 ** -21
    tol = U[dtype] * np.abs(out) + (WEIGHT[dtype] + 2 * e + sums) * part
    if dtype == "f16":
        tol += 2.0 ** -40 * np.abs(v).sum(0) / total
    return out, (m + np.log(total))[:, 0], tol, (2 * e + sums + 2.0 ** -22 * np.abs(m))[:, 0]


def truncated(bits):
    def cut(p):
        a = p.astype(np.float32).view(np.uint32)
        return (a & np.uint32(0xFFFFFFFF << (24 - bits) & 0xFFFFFFFF)).view(np.float32).astype(np.float64)
    return cut


def nearest(kind):
    return lambda p: torch.from_numpy(p).to(kind).double().numpy()


@pytest.mark.parametrize("dtype,mistake", [("bf16", nearest(torch.bfloat16)), ("bf16", truncated(8)), ("f16", truncated(9)),
                                           ("f16", nearest(torch.bfloat16))])
def test_the_bounds_see_weights_of_fewer_bits(dtype, mistake):
    q, k, v = inputs(100, 200, 64, 1)
    want, _, tol, _ = expected(dtype, q, k, v, 0.125)
    wrong = expected(dtype, q, k, v, 0.125, mistake)[0]
    assert (np.abs(wrong - want) > tol).any()


@pytest.mark.parametrize("octaves", [25, 26])
def test_the_bounds_see_lost_tails(octaves):
    q, k, v = inputs(2, 131072, 64, 2, sink=round(octaves * np.log(2) / 64 / 0.125 * 2) / 2)
    want, _, tol, _ = expected("f16", q, k, v, 0.125)
    wrong = expected("f16", q, k, v, 0.125, nearest(torch.float16))[0]
    assert (np.abs(wrong - want) > tol).any()


def check(dtype, q, k, v, scale, work, drafted, requests=1, block=16):
    """The rows of one request; the last `drafted` keys are its drafted rows' own, which all its rows see.  More
    requests are the same again, over the same blocks."""
    from kv_helpers import DEV, DT, Cache, i32
    from paper_2608_25431_amd import gift
    dim, t = q.shape[1], DT[dtype]
    cached = len(k) - drafted
    n = -(-cached // block)
    c = Cache(dtype, 1, dim, block, n + 1)
    ids = np.random.default_rng(3).permutation(n + 1)[:n]
    for view, x in ((c.k, k), (c.v, v)):
        pad = torch.full((n * block, dim), float("nan"), dtype=t)
        pad[:cached] = torch.from_numpy(x[:cached]).to(t)
        view[0, torch.from_numpy(ids).to(DEV), :, 0] = pad.view(n, block, dim).to(DEV)
    group = len(q) // drafted
    dq = torch.from_numpy(q).to(t).view(drafted, group, dim).to(DEV)
    dk, dv = (torch.from_numpy(x[cached:]).to(t).view(drafted, 1, dim).to(DEV) for x in (k, v))
    dq, dk, dv = (x.repeat(requests, 1, 1) for x in (dq, dk, dv))
    rows = drafted * requests
    out, lse = torch.empty_like(dq), torch.empty(rows, group, device=DEV)
    mask = torch.full((rows, -(-drafted // 32)), -1, dtype=torch.int32, device=DEV)
    kv, fmt = c.args()
    gift.tree_attention(work, kv, fmt, 0, dq, dk, dv, i32(np.arange(requests + 1) * drafted),
                        i32([cached] * requests), i32(np.tile(ids, (requests, 1))), out, mask=mask, lse=lse, scale=scale)
    v = torch.from_numpy(v).to(t).double().numpy()
    want, ends, tol, etol = expected(dtype, q, k, v, scale, chain=256 if requests == 1 else len(k))
    off = np.abs(out.cpu().double().numpy().reshape(requests, *want.shape) - want)
    assert (off <= tol).all(), f"{(off > tol).mean():.3g} outside, worst {np.max(off / tol):.3g} of the bound"
    assert (np.abs(lse.cpu().double().numpy().reshape(requests, -1) - ends) <= etol).all()


@pytest.fixture(scope="module")
def work():
    from paper_2608_25431_amd import gift
    return gift.AttentionWork()


@gpu
@needs
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("drafted", [5, 12, 25, 60])  # times 4: each number of waves that share keys
@pytest.mark.parametrize("keys", [100, 200])
def test_bits_of_weights(work, dtype, dim, drafted, keys):
    q, k, v = inputs(4 * drafted, keys, dim, dim + drafted)
    check(dtype, q, k, v, 0.125, work, drafted)


@gpu
@needs
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("octaves", [12, 17, 20, 25, 26, 28])
@pytest.mark.parametrize("drafted,keys,dim", [(2, 131072, 64), (30, 16384, 128), (1, 40000, 256)])
def test_many_keys_far_below_one(work, dtype, octaves, drafted, keys, dim):
    # attention sinks: one key holds most of the weight and has no part in the output
    q, k, v = inputs(4 * drafted, keys, dim, 5, sink=round(octaves * np.log(2) / dim / 0.125 * 2) / 2)
    check(dtype, q, k, v, 0.125, work, drafted)


@gpu
@needs
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("octaves", [17, 25, 29])
@pytest.mark.parametrize("requests,drafted,keys,dim", [(512, 2, 16384, 64), (512, 13, 4096, 128), (512, 25, 4096, 96),
                                                       (512, 20, 2048, 256), (512, 45, 8192, 128)])
def test_columns_of_one_workgroup(work, dtype, octaves, requests, drafted, keys, dim):
    # as many columns as workgroups: a wave's reference is the sink's score for all keys that follow it
    q, k, v = inputs(4 * drafted, keys, dim, 6, sink=round(octaves * np.log(2) / dim / 0.125 * 8) / 8)
    check(dtype, q, k, v, 0.125, work, drafted, requests)
