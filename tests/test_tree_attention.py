"""gift_tree_attention on the GPU against its definition in 64 bits.  Everything in a cache that no request owns is NaN,
so nothing that a row does not see may have a part in it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from kv_helpers import DEV, Batch, Cache, i32  # noqa: E402
from paper_2608_25431_amd import gift  # noqa: E402


@pytest.fixture(scope="module")
def work():
    return gift.AttentionWork()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("drafts", [[3, 9, 1], [14, 10, 3], [33, 20, 15], [70, 31, 49]])
def test_rows_that_share_keys(work, dim, dtype, drafts):
    # 17, 36, 90 and 200 rows at a KV head on average: each number of waves that share a tile, with part-filled ones
    b = Batch([201, 0, 1030], drafts, dtype, heads=2, group=4, dim=dim, mask="holes", seed=dim + drafts[0])
    b.check(b.run(work))


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 257, 400]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("mask", ["tree", "holes", None])
def test_lengths_and_types(work, dtype, dim, mask):
    r = np.random.default_rng(dim)
    b = Batch(LENS, r.integers(0, 9, len(LENS)), dtype, dim=dim, mask=mask, seed=dim, heads=2, group=2)
    b.check(b.run(work))


@pytest.mark.parametrize("heads,group,drafts", [
    (1, 1, [1]), (8, 4, [1, 1, 1]), (3, 7, [5, 0, 13]), (2, 8, [4, 3, 5]), (2, 8, [8, 9, 7]), (1, 8, [33, 17, 1]),
    (2, 4, [64, 2, 31]), (1, 16, [32, 33, 0]), (1, 1, [65, 129, 32]), (2, 3, [100, 1, 97])])
@pytest.mark.parametrize("block,order,parts", [(16, "head", 1), (1, "token", 2), (128, "token", 1)])
def test_heads_and_layouts(work, heads, group, drafts, block, order, parts):
    lens = [150, 0, 77][:len(drafts)]
    b = Batch(lens, drafts, heads=heads, group=group, dim=64 if block == 1 else 128, block=block, order=order,
              parts=parts, seed=heads + group)
    b.check(b.run(work))


@pytest.mark.parametrize("lens,drafts,heads,group,dim", [
    ([5000], [3], 2, 4, 128), ([9001, 1], [1, 1], 1, 1, 64), ([3000, 0, 1700], [20, 6, 1], 1, 8, 96),
    ([4100], [40], 1, 4, 256), ([2500, 2499], [50, 60], 1, 2, 128),
    ([20001, 5], [3, 1], 1, 2, 64), ([40000], [2], 1, 1, 96)])  # parts joined in runs of 16 and of 64
def test_long_axes_are_split_and_joined(work, lens, drafts, heads, group, dim):
    b = Batch(lens, drafts, "f16" if dim == 64 else "bf16", heads=heads, group=group, dim=dim, seed=7, q_scale=2.0)
    got = b.run(work)
    b.check(got)
    again = b.run(work)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])  # the same bits, whoever came last


def test_many_requests(work):
    r = np.random.default_rng(3)
    n = 700  # more requests than threads of a workgroup
    b = Batch(r.integers(0, 40, n), r.integers(0, 3, n), heads=1, group=2, dim=64, seed=3)
    b.check(b.run(work))


@pytest.mark.parametrize("mask", ["random", None])
def test_any_mask(work, mask):
    # bits of later rows and past the drafts; words beyond the drafts of a request
    b = Batch([40, 0, 9], [37, 64, 2], heads=2, group=4, dim=128, mask=mask, seed=11)
    b.check(b.run(work))


def test_masks_narrower_than_the_draft(work):
    b = Batch([20, 0], [70, 33], heads=1, group=2, dim=64, seed=12)
    b.bits = np.ascontiguousarray(b.bits[:, :32])
    b.check(b.run(work))


def test_only_cached_keys(work):
    b = Batch([40, 0, 33], [5, 2, 1], heads=2, group=4, dim=128, mask=None, seed=13)
    b.check(b.run(work, drafted=False), drafted=False)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_unseen_rows_have_no_part(work, bad):
    # three drafted rows hold non-finite K and V and no row but themselves sees them; two of them see nothing at all
    for drafts, dim in (([12], 128), ([40], 64), ([9], 96), ([35], 256)):
        b = Batch([50], drafts, heads=2, group=4, dim=dim, mask="random", seed=14)
        h, g = 2, 4
        for row in (1, 5, 8):
            b.bits[:, row] = 0
        b.bits[1] = 0
        b.qkv[5, h * g + h:] = bad
        b.qkv[1, h * g:] = bad
        b.qkv[8, h * g:h * g + h] = bad
        got = b.run(work)
        clean = b.qkv.clone()
        clean[[1, 5, 8], h * g:] = 0.0
        b.qkv = clean
        b.check(got)
        # a row that sees such a V takes it, the others do not
        b.qkv[5, h * g + h:, 3] = bad
        b.bits[2, 5] = 1
        out = b.run(work)[0]
        hit = torch.zeros(out.shape, dtype=torch.bool)
        hit[2, :, 3] = True
        assert not torch.isfinite(out[hit]).any() and torch.isfinite(out[~hit]).all()
        b.qkv[5, h * g + h:, 3] = 0.0
        want = b.expect()
        off = (out.double().numpy() - want[0])[~hit.numpy()]
        assert (np.abs(off) <= want[2][~hit.numpy()]).all()


def test_verdicts_and_uncovered_rows(work):
    b = Batch([300, 20, 0, 45], [6, 7, 2, 3], heads=2, group=2, dim=64, seed=15)
    b.verdicts = np.array([0, gift.SEG_OWNER_MIXED, 0, gift.SEG_NO_SPACE])
    got = b.run(work)
    b.check(got)
    assert (got[0][6:13] == 0).all() and (got[1][6:13] == -np.inf).all()
    # rows before the first request's and after the last one's belong to nobody
    b.verdicts = None
    pad = Batch([300, 20, 0, 45], [6, 7, 2, 3], heads=2, group=2, dim=64, seed=15)
    first, last = torch.randn(4, 8, 64).to(torch.bfloat16), torch.randn(9, 8, 64).to(torch.bfloat16)
    pad.qkv = torch.cat([first, b.qkv, last])
    pad.bits = np.concatenate([np.ones((4, 32), np.uint8), b.bits, np.ones((9, 32), np.uint8)])
    out, lse = pad.run(work, row_begin=i32(b.row_begin + 4))
    b.check((out[4:-9], lse[4:-9]))
    for x in (out[:4], out[-9:]):
        assert (x == 0).all()
    assert (lse[:4] == -np.inf).all() and (lse[-9:] == -np.inf).all()


def test_no_requests_and_no_rows(work):
    b = Batch([10], [3], heads=1, group=1, dim=64)
    out, lse = b.run(work, row_begin=i32([0]), lens=i32([]), tables=i32([]).reshape(0, 1))
    assert (out == 0).all() and (lse == -np.inf).all()
    none = Batch([10], [0], heads=1, group=1, dim=64)
    assert none.run(work)[0].numel() == 0


def test_row_ranges_that_do_not_rise(work):
    # what the device arrays hold is cut to the buffers: no access outside them, rows of a sound request right
    b = Batch([30, 40], [4, 5], heads=1, group=2, dim=64, seed=16)
    out, _ = b.run(work, row_begin=i32([0, 4, 4000000000]))
    b.check((out, None))
    out, _ = b.run(work, row_begin=i32([0, 4, 1]))
    assert (out[4:] == 0).all()


def test_table_entries_outside_the_cache(work):
    b = Batch([200, 64], [3, 2], heads=2, group=2, dim=64, seed=17)
    b.tab[0, 2], b.tab[0, 9], b.tab[1, 0] = b.cache.n_blocks, 0xFFFFFFFF, 0x80000000
    gone = {0: (2, 9), 1: (0,)}
    b.check(b.run(work), unseen=lambda req, pos: np.isin(pos // 16, gone[req]))


def test_lengths_past_the_table(work):
    b = Batch([64, 30], [3, 2], heads=1, group=2, dim=64, seed=18)
    b.tab = b.tab[:, :4]
    b.check(b.run(work, lens=i32([0xFFFFFFFF, 30])))  # cut to the 4 blocks of the row


def test_strided_operands(work):
    b = Batch([70, 5], [9, 4], heads=2, group=2, dim=64, seed=19)
    store = torch.full((13, 3, 4, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    wide = torch.full((2, 20), -3, dtype=torch.int32, device=DEV)
    tables = wide[:, 4:4 + b.width]
    tables.copy_(i32(b.tab))
    got = b.run(work, out=store[:, 1], tables=tables, lse=False)
    b.check(got)
    assert (store[:, 0] == 5).all() and (store[:, 2] == 5).all()
    heads_first = torch.empty(4, 13, 64, dtype=torch.bfloat16, device=DEV)
    b.run(work, out=heads_first.permute(1, 0, 2))
    assert torch.equal(heads_first.permute(1, 0, 2).cpu(), got[0])


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(work, scale):
    b = Batch([300, 3], [6, 2], "f16", heads=1, group=4, dim=64, seed=20)
    b.check(b.run(work, scale=scale), scale=scale)


def test_offsets_past_32_bits(work):
    # the request's blocks are the last of a layer that starts past 2^32 bytes
    b = Batch([100, 37], [5, 3], heads=8, group=2, dim=128, n_layers=1, layer=0, seed=21)
    big = Cache("bf16", 8, 128, 16, 3200, 24, "head", 1, fill=None)
    used = b.cache.n_blocks
    big.k[23, 3200 - used:] = b.cache.k[0]
    big.v[23, 3200 - used:] = b.cache.v[0]
    assert 2 * big.layer_stride * 23 > 1 << 32
    b.tab[b.tab < used] += 3200 - used
    b.cache, b.layer = big, 23
    b.check(b.run(work))


def test_other_streams(work):
    b = Batch([900, 10], [5, 8], heads=2, group=4, dim=128, seed=22)
    want = b.run(work)
    s = torch.cuda.Stream()
    mine = gift.AttentionWork(stream=s)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = b.run(mine)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_captured_step_replays(work):
    # tables, append and attention of one step in a graph; lengths change between the replays
    block, heads, group, dim, n = 16, 2, 4, 128, 5
    kw = dict(heads=heads, group=group, dim=dim, n_layers=1, layer=0, seed=23)
    b = Batch([40, 700, 16, 1, 0], [3, 1, 4, 8, 2], **kw)
    kv, fmt = b.cache.args()
    dev = b.qkv.to(DEV)
    q, k, v = dev[:, :8], dev[:, 8:10], dev[:, 10:]
    rows = dev.shape[0]
    out = torch.empty(rows, heads * group, dim, dtype=dev.dtype, device=DEV)
    lse = torch.empty(rows, heads * group, device=DEV)
    users, labels = i32(np.arange(n)), i32(np.full(b.cache.n_blocks, gift.LABEL_UNOWNED))
    for i in range(n):
        labels[torch.from_numpy(b.tab[i][b.tab[i] < b.cache.n_blocks]).to(DEV)] = i
    lens, new, tables = i32(b.lens), i32(np.zeros(n)), i32(b.tab)
    slots, begin = torch.full((4,), -1, dtype=torch.int64, device=DEV), i32(np.zeros(n + 1))
    lens_out, taken, verdicts = i32(np.zeros(n)), i32([0]), i32(np.zeros(n))
    row_begin, mask, free = i32(b.row_begin), b.mask_words(), i32([])
    index = i32([0, 1, 2, 3])
    own = gift.AttentionWork()

    def step():
        gift.kv_tables(users, lens, new, block, free, tables, labels, slots, begin, lens_out, taken, verdicts)
        gift.kv_append(kv, fmt, slots, k.unsqueeze(0), v.unsqueeze(0), index=index)
        gift.tree_attention(own, kv, fmt, 0, q, k, v, row_begin, lens_out, tables, out, mask=mask, verdicts=verdicts,
                            lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keep = b.cache.data.clone()
    for add in ([0, 0, 0, 0, 0], [2, 0, 0, 1, 0], [1, 1, 0, 2, 0], [0, 3, 0, 0, 0]):
        lens.copy_(i32(b.lens))
        new.copy_(i32(add))
        b.cache.data.copy_(keep)
        step()
        torch.cuda.synchronize()
        want = out.clone(), lse.clone(), b.cache.data.clone()
        assert verdicts.tolist() == [0] * n and lens_out.tolist() == (b.lens + add).tolist()
        out.zero_()
        lse.zero_()
        b.cache.data.copy_(keep)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert torch.equal(b.cache.data.view(torch.int16), want[2].view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("q_scale", [0.3, 3.0, 12.0])
@pytest.mark.parametrize("drafts", [[4, 3], [40, 45]])
def test_scores_that_stay_and_that_jump(work, dtype, q_scale, drafts):
    # maxima that later keys pass by less than the weights' reference follows, and by far more
    b = Batch([1500, 333], drafts, dtype, heads=1, group=4, dim=128, seed=24, q_scale=q_scale)
    b.check(b.run(work))


@pytest.mark.parametrize("drafts", [7, 25, 60])
def test_rows_do_not_depend_on_the_rows_beside_them(work, drafts):
    # other queries in the same call, some far larger: a row that does not see their keys has the same bits
    b = Batch([900], [drafts], heads=1, group=4, dim=128, seed=25)
    b.bits = np.eye(drafts, b.bits.shape[1], dtype=np.uint8)
    one = b.run(work)
    b.qkv[1:, :4] *= 9.0
    two = b.run(work)
    assert torch.equal(one[0][0], two[0][0]) and torch.equal(one[1][0], two[1][0])
    assert not torch.equal(one[0][1:], two[0][1:])
