"""What the binding of the paged-cache calls checks before it calls the library, without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_25431_amd import gift  # noqa: E402
from test_kv_refusals import Fake, cache, form  # noqa: E402

I = torch.int32


class Recorder:
    """Stands in for the library: takes every call and remembers its arguments; workspaces are numbers from 100 on."""

    def __init__(self):
        self.calls, self.made = [], 100

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return gift.OK
        return call

    def gift_attention_work_create(self, stream, out):
        self.calls.append(("gift_attention_work_create", (stream,)))
        out._obj.value = self.made
        self.made += 1
        return gift.OK

    def gift_last_error(self):
        return b"no memory"

    def of(self, name, at=0):
        return [args[at] for n, args in self.calls if n == name]


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(gift, "lib", lambda: r)
    return r


def attend(work=None, stream=0, **over):
    a = dict(q=Fake((6, 32, 128)), k=Fake((6, 8, 128)), v=Fake((6, 8, 128)), row_begin=Fake((3,), I), lens=Fake((2,), I),
             tables=Fake((2, 4), I), out=Fake((6, 32, 128)), mask=Fake((6, 1), I), verdicts=Fake((2,), I),
             lse=Fake((6, 32), torch.float32))
    a.update(over)
    work = work or type("W", (), {"handle": None})
    gift.tree_attention(work, cache(), form(), 0, a["q"], a["k"], a["v"], a["row_begin"], a["lens"], a["tables"], a["out"],
                        mask=a["mask"], verdicts=a["verdicts"], lse=a["lse"], stream=stream)


class Empty(Fake):
    def data_ptr(self):
        return 0 if self.numel() == 0 else Fake.data_ptr(self)


def test_a_mask_of_no_words_is_not_no_mask(recorder):
    attend()
    with pytest.raises(ValueError, match="mask: needs at least one word"):
        attend(mask=Empty((6, 0), I))
    none = dict(q=Empty((0, 32, 128)), out=Empty((0, 32, 128)), k=Empty((0, 8, 128)), v=Empty((0, 8, 128)))
    attend(mask=Empty((0, 0), I), lse=None, **none)
    assert [name for name, _ in recorder.calls] == ["gift_tree_attention"] * 2


def test_calls_on_several_streams_have_a_workspace_each(recorder, monkeypatch):
    capturing = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    work = gift.AttentionWork(stream=7)
    for stream in (7, 9, 0, 9, 7, 0):
        attend(work, stream)
    capturing[0] = True  # nothing may be made now: captured calls use the first one
    attend(work, 9)
    attend(work, 5)
    used = recorder.of("gift_tree_attention")
    assert used == [100, 101, 102, 101, 100, 102, 100, 100]
    assert recorder.of("gift_attention_work_create") == [7, 9, 0]
    assert recorder.of("gift_tree_attention", 4) == [7, 9, 0, 9, 7, 0, 9, 5]
    work.destroy()
    work.destroy()
    assert sorted(recorder.of("gift_attention_work_destroy")) == [100, 101, 102]


def test_a_dropped_workspace_is_freed_later(recorder):
    work = gift.AttentionWork(stream=7)
    del work  # anywhere, as by the garbage collector during a capture: no call may synchronise now
    assert not recorder.of("gift_attention_work_destroy")
    other = gift.AttentionWork(stream=7)
    assert recorder.of("gift_attention_work_destroy") == [100] and other.handle == 101
    third = gift.AttentionWork(stream=7)
    del third
    other.destroy()
    assert sorted(recorder.of("gift_attention_work_destroy")) == [100, 101, 102]


def test_a_workspace_that_was_never_made(recorder, monkeypatch):
    monkeypatch.setattr(Recorder, "gift_attention_work_create", lambda self, stream, out: gift.E_NOMEM)
    with pytest.raises(gift.GiftError):
        gift.AttentionWork(stream=7)
    assert not recorder.of("gift_attention_work_destroy")


def test_missing_arrays_are_refused_by_the_library():
    with pytest.raises(gift.GiftError, match="null"):
        attend(row_begin=None, verdicts=None)
    one = Fake((3,), I)
    with pytest.raises(gift.GiftError, match="null row_begin or taken"):
        gift.kv_tables(one, one, one, 16, one, Fake((3, 5), I), one, Fake((9,), torch.int64), None, one, one, one, stream=0)
