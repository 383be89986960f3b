"""gift_kv_append on the GPU: every byte of the cache against a copy in numpy."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from kv_helpers import DEV, DT, Cache, i32  # noqa: E402
from paper_2608_25431_amd import gift  # noqa: E402


def bits(x):
    return x.cpu().contiguous().view(torch.int16).numpy()


@pytest.mark.parametrize("dtype,heads,dim,block,order,parts,layers,n_src,n_slots", [
    ("bf16", 8, 128, 16, "head", 1, 3, 40, 17), ("bf16", 8, 128, 16, "token", 1, 32, 1, 1),
    ("f16", 1, 64, 1, "head", 2, 1, 5, 5), ("f16", 5, 96, 32, "token", 2, 2, 300, 299),
    ("bf16", 3, 256, 64, "head", 2, 2, 33, 31), ("bf16", 10, 64, 8, "token", 1, 4, 1000, 777),
    ("f16", 16, 128, 128, "head", 1, 2, 2100, 2048)])
@pytest.mark.parametrize("indexed", [False, True])
def test_rows_reach_their_slots(dtype, heads, dim, block, order, parts, layers, n_src, n_slots, indexed):
    r = np.random.default_rng(n_src)
    blocks = n_slots // block + 3
    c = Cache(dtype, heads, dim, block, blocks, layers, order, parts, fill=None)
    c.data.view(torch.int16).random_(-32768, 32767)  # any bits: rows are copied as they are, NaNs included
    slots = r.permutation(blocks * block)[:n_slots].astype(np.int64)
    slots[r.random(n_slots) < 0.1] = -1
    index = r.permutation(n_src)[:n_slots] if indexed else np.arange(n_slots)
    if n_slots > 20:  # outside the cache, far outside, outside the sources
        slots[3], slots[4], slots[5] = blocks * block, 1 << 40, -(1 << 40)
        if indexed:
            index[6], index[7] = n_src, 0xFFFFFFFF
    src = torch.empty(layers, n_src, 2 * heads, dim, dtype=DT[dtype], device=DEV)
    src.view(torch.int16).random_(-32768, 32767)
    k, v = src[:, :, :heads], src[:, :, heads:]
    want = torch.from_numpy(bits(c.data).copy())
    shape = (layers, blocks, block, heads, dim)
    strides = (c.layer_stride, c.block_stride, c.token, c.head, 1)
    kw, vw = torch.as_strided(want, shape, strides, 0), torch.as_strided(want, shape, strides, c.v_off)
    kh, vh = torch.from_numpy(bits(k)), torch.from_numpy(bits(v))
    for s, i in zip(slots, index):
        if 0 <= s < blocks * block and i < n_src:
            kw[:, s // block, s % block], vw[:, s // block, s % block] = kh[:, i], vh[:, i]
    kv, fmt = c.args()
    gift.kv_append(kv, fmt, torch.from_numpy(slots).to(DEV), k, v, index=i32(index) if indexed else None)
    got = bits(c.data)
    assert (got == want.numpy()).all(), f"{(got != want.numpy()).sum()} elements differ"


def test_sources_of_other_strides():
    c = Cache("bf16", 4, 64, 16, 4, 3, "token", 1, fill=0.0)
    k = torch.randn(4, 20, 3, 64, device=DEV).to(torch.bfloat16).permute(2, 1, 0, 3)  # [layer][row][head], head outermost
    v = torch.randn(20, 3, 4, 128, device=DEV).to(torch.bfloat16).permute(1, 0, 2, 3)[..., 64:]
    kv, fmt = c.args()
    gift.kv_append(kv, fmt, torch.arange(30, 50, device=DEV), k, v)
    assert torch.equal(c.k.reshape(3, 64, 4, 64)[:, 30:50], k) and torch.equal(c.v.reshape(3, 64, 4, 64)[:, 30:50], v)
    assert (c.k.reshape(3, 64, 4, 64)[:, :30] == 0).all() and (c.k.reshape(3, 64, 4, 64)[:, 50:] == 0).all()


def test_offsets_past_32_bits():
    # a cache of 6.5 GB: the last layer's last block lies past 2^32 bytes, and so does the last source row
    c = Cache("bf16", 8, 128, 16, 3200, 31, "head", 1, fill=None)
    assert 2 * c.layer_stride * 30 > 1 << 32
    c.k[30, 3199, 15].fill_(0)
    src = torch.empty(31, 36000, 16, 128, dtype=torch.bfloat16, device=DEV)
    assert 2 * src[:30].numel() > 1 << 32
    src[:, 35999] = torch.randn(31, 16, 128, device=DEV)
    kv, fmt = c.args()
    gift.kv_append(kv, fmt, torch.tensor([3200 * 16 - 1], device=DEV), src[:, :, :8], src[:, :, 8:], index=i32([35999]))
    assert torch.equal(c.k[:, 3199, 15], src[:, 35999, :8]) and torch.equal(c.v[:, 3199, 15], src[:, 35999, 8:])


def test_no_rows():
    c = Cache("bf16", 2, 64, 16, 2, fill=1.0)
    kv, fmt = c.args()
    rows = torch.zeros(1, 0, 2, 64, dtype=torch.bfloat16, device=DEV)
    gift.kv_append(kv, fmt, torch.zeros(0, dtype=torch.int64, device=DEV), rows, rows)
    some = torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16, device=DEV)
    gift.kv_append(kv, fmt, torch.zeros(0, dtype=torch.int64, device=DEV), some, some)
    assert (c.data == 1).all()
