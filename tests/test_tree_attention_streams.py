"""Calls on several streams at once, with one AttentionWork: columns that several workgroups share are joined in a workspace
of the stream's own."""
import gc

import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from kv_helpers import DEV, Batch, i32  # noqa: E402
from paper_2608_25431_amd import gift  # noqa: E402


class Call:
    """One batch's call with everything on the device."""

    def __init__(self, b):
        self.b, (self.kv, self.fmt) = b, b.cache.args()
        dev, h, g = b.qkv.to(DEV), b.cache.heads, b.group
        self.q, self.k, self.v = dev[:, :h * g], dev[:, h * g:h * g + h], dev[:, h * g + h:]
        self.ints = i32(b.row_begin), i32(b.lens), i32(b.tab)
        self.mask = b.mask_words()

    def __call__(self, work):
        out = torch.empty(self.q.shape, dtype=self.q.dtype, device=DEV)
        lse = torch.empty(self.q.shape[:2], device=DEV)
        gift.tree_attention(work, self.kv, self.fmt, self.b.layer, self.q, self.k, self.v, *self.ints, out, mask=self.mask,
                            lse=lse)
        return out, lse


def test_one_workspace_object_on_three_streams():
    calls = [Call(Batch(lens, drafts, heads=4, group=4, dim=dim, seed=dim))
             for lens, drafts, dim in (([30000, 9], [3, 2], 128), ([15000], [25], 64), ([20000, 700], [50, 3], 128))]
    work = gift.AttentionWork()
    want = [c(work) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[] for _ in calls]
    for _ in range(20):
        for i, (s, c) in enumerate(zip(streams, calls)):
            with torch.cuda.stream(s):
                got[i].append(c(work))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for out, lse in g:
            assert torch.equal(out, w[0]) and torch.equal(lse, w[1])
    work.destroy()


def test_a_workspace_dropped_during_a_capture():
    call = Call(Batch([9000, 3], [3, 2], heads=2, group=4, dim=128, seed=3))
    work, other = gift.AttentionWork(), [gift.AttentionWork()]
    want = call(work)
    call(other[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(work)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.clear()
        gc.collect()
        got = call(work)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        again = call(work)
        assert torch.equal(again[0], want[0])
        got[0].zero_()
        got[1].zero_()
    work.destroy()


def test_no_workspace_is_made_during_a_capture():
    call = Call(Batch([9000, 3], [3, 2], heads=2, group=4, dim=128, seed=4))
    work = gift.AttentionWork()
    want = call(work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(gift.GiftError, match="being captured"):
            gift.AttentionWork()
        got = call(work)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got[0].zero_()
    work.destroy()
