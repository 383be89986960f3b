"""Calls around the quantised cache of more rows than a launch has workgroups for.  A launch of 2^32 threads or more along
a dimension runs nothing, without an error, and a call has up to 2^31 - 1 rows."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_launch_plan import symbol

from paper_2608_25431_amd import gift

gpu = pytest.mark.gpu
needs = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
THREADS = 256


class RowsPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in ("rows", "parts", "launch")]


def launches(p):
    return 1 <= p.rows <= p.launch and -(-p.launch // p.rows) * THREADS < 1 << 32 and 1 <= p.parts < 1 << 16


COUNTS = [1, 7, 1023, 1024, 17203, 1 << 24, 1 << 27, (1 << 27) + 1, 1 << 30, (1 << 31) - 1]


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_every_count_of_norm_and_rotation_launches(dim):
    plan = symbol("_ZN4gift17qk_norm_rope_plan")
    plan.restype = RowsPlan
    for n in COUNTS:
        for q_heads, k_heads in ((1, 0), (0, 1), (10, 10), (32, 8), (64, 8), (1 << 20, 1)):
            if n * (q_heads + k_heads) < 1 << 32:  # more is refused
                p = plan(ctypes.byref(gift._QkRows(n_rows=n, q_heads=q_heads, k_heads=k_heads, head_dim=dim)))
                assert launches(p) and p.rows <= 8, (n, q_heads, k_heads)


def test_every_count_of_rows_read_launches():
    plan = symbol("_ZN4gift18kv_read_quant_plan")
    plan.restype = RowsPlan
    for n in COUNTS:
        for layers in (1, 16, 100000):
            assert launches(plan(ctypes.byref(gift._KvRead(n_rows=n, n_layers=layers)))), (n, layers)


@gpu
@needs
def test_norm_and_rotation_of_more_rows_than_a_launch_s():
    """The same bits as in parts of few rows."""
    from kv_helpers import DEV
    n = (1 << 21) + 100003
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(n, 1, 64, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.rand(64, generator=g, device=DEV).to(torch.bfloat16) + 0.5
    places = torch.randint(0, 1 << 20, (n,), generator=g, device=DEV, dtype=torch.int32)
    freq = 10000.0 ** -(torch.arange(32, device=DEV) / 32)
    want = torch.empty_like(x)
    for at in range(0, n, 100003):
        part = slice(at, at + 100003)
        gift.qk_norm_rope(x[part], None, want[part], None, places[part], freq, q_weight=w)
    gift.qk_norm_rope(x, None, x, None, places, freq, q_weight=w)
    assert torch.equal(x, want)


@gpu
@needs
def test_more_rows_read_than_a_launch_s():
    """Requests that end before, in and behind the second launch's rows; rows before the first and behind the last stay."""
    from kv_helpers import DEV, i32
    from quant_helpers import QuantCache, quantised, values
    per, block, blocks = 65536 * 4 * 16, 128, 5
    n = per + 70003
    cache = QuantCache(1, 64, block, blocks)
    x = torch.randn(2, blocks * block, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).double().numpy()
    want = []
    for y, elements, factors in ((x[0], cache.k, cache.kf), (x[1], cache.v, cache.vf)):
        b, f = quantised(y, "bf16")
        elements.copy_(torch.from_numpy(b).view(1, blocks, block, 1, 64))
        factors.copy_(torch.from_numpy(np.pad(f, ((0, 0), (0, 2)))).view(1, blocks, block, 1, 4))
        want.append(torch.from_numpy(values(b, f, "bf16")).to(DEV, torch.bfloat16))
    begin = np.array([5, 1000, per + 3, n - 4])
    lens = np.array([900, per + 50000, 60000])
    first = np.array([0, 17, 64])
    width = -(-int(lens.max()) // block)
    tab = np.random.default_rng(2).integers(0, blocks, (3, width))  # a block may come up again where it is only read
    k, v = torch.full((2, 1, n, 1, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    gift.kv_read_quant(*cache.args(), i32(tab), i32(lens), i32(begin), k, v, first=i32(first))
    for got, w in zip((k, v), want):
        got = got[0, :, 0]
        assert (got[:5] == 7).all() and (got[-4:] == 7).all()
        for b in range(3):
            token = torch.arange(int(first[b]), int(first[b] + begin[b + 1] - begin[b]), device=DEV)
            there = token < int(lens[b])
            token = token.clamp(max=int(lens[b]) - 1)
            rows = w[torch.from_numpy(tab[b]).to(DEV)[token // block] * block + token % block]
            assert torch.equal(got[begin[b]:begin[b + 1]], torch.where(there[:, None], rows, 0.0)), b
