"""What the paged-cache calls refuse, without a GPU: the C entry points check their arguments before they touch a device,
so device addresses are made up here; the binding checks tensors before it calls the library."""
import ctypes
import os

import pytest

from paper_2608_25431_amd import gift

torch = pytest.importorskip("torch")

A = 1 << 40  # a made-up device address, 16-byte aligned


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gift.LIB_PATH):
        from paper_2608_25431_amd import build
        build.build()
    yield gift.lib()
    gift.lib().gift_attention_work_destroy(None)  # leaves no message behind for other tests


def cache(**over):
    a = dict(base=A, cache_bytes=4 * 10 * 65536, layer_stride=10 * 65536, block_stride=65536, part_stride=65536,
             chunk_bytes=65536, n_layers=4, n_parts=1, n_blocks=10)
    a.update(over)
    return gift._PagedKV(*(a[n] for n, _ in gift._PagedKV._fields_))


def form(**over):
    a = dict(dtype=gift.BF16, n_heads=8, head_dim=128, block_tokens=16, k_offset=0, v_offset=32768, token_stride=256,
             head_stride=4096)
    a.update(over)
    return gift._KvFormat(*(a[n] for n, _ in gift._KvFormat._fields_))


def attention(lib, work=A, kv=None, fmt=None, **over):
    a = dict(n_rows=6, n_reqs=2, n_heads=32, layer=0, scale=0.1, q=2 * A, k=3 * A, v=4 * A, out=5 * A, lse=6 * A,
             q_row_stride=8192, q_head_stride=256, k_row_stride=2048, k_head_stride=256, v_row_stride=2048,
             v_head_stride=256, out_row_stride=8192, out_head_stride=256, row_begin=A, lens=A, tables=A, table_width=4,
             table_stride=4, mask=A, mask_words=1, verdicts=None)
    a.update(over)
    args = gift._TreeAttention(*(a[n] for n, _ in gift._TreeAttention._fields_))
    return lib.gift_tree_attention(work, ctypes.byref(kv or cache()), ctypes.byref(fmt or form()), ctypes.byref(args),
                                   None)


BAD_CACHES = [dict(base=None), dict(base=A + 8), dict(chunk_bytes=65520), dict(n_layers=0), dict(block_stride=32768)]
BAD_FORMATS = [
    dict(dtype=0), dict(dtype=3), dict(n_heads=0), dict(head_dim=0), dict(head_dim=80), dict(head_dim=512),
    dict(block_tokens=0), dict(block_tokens=24), dict(k_offset=8), dict(v_offset=32776), dict(token_stride=264),
    dict(head_stride=4104), dict(token_stride=128), dict(head_stride=2048), dict(v_offset=128), dict(v_offset=0),
    dict(v_offset=32784), dict(n_heads=17), dict(block_tokens=32), dict(head_stride=1 << 63), dict(v_offset=1 << 63),
    dict(token_stride=(1 << 64) - 16)]


@pytest.mark.parametrize("kv", BAD_CACHES)
def test_caches(lib, kv):
    assert attention(lib, kv=cache(**kv)) == gift.E_INVALID
    assert append(lib, kv=cache(**kv)) == gift.E_INVALID


@pytest.mark.parametrize("fmt", BAD_FORMATS)
def test_formats(lib, fmt):
    assert attention(lib, fmt=form(**fmt)) == gift.E_INVALID
    assert append(lib, fmt=form(**fmt)) == gift.E_INVALID
    assert gift.last_error()


def test_caches_shorter_than_their_chunks(lib):
    short = cache(cache_bytes=4 * 10 * 65536 - 1)
    assert attention(lib, kv=short) == gift.E_RANGE and append(lib, kv=short) == gift.E_RANGE


@pytest.mark.parametrize("bad,status", [
    (dict(n_heads=0), -1), (dict(n_heads=12), -1), (dict(layer=4), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(q=2 * A + 2), -1),
    (dict(k=3 * A + 8), -1), (dict(out=5 * A + 4), -1), (dict(k=None), -1), (dict(v=None), -1),
    (dict(q_row_stride=8200), -1), (dict(q_head_stride=250), -1), (dict(k_row_stride=2056), -1),
    (dict(v_head_stride=2), -1), (dict(out_row_stride=8196), -1), (dict(out_head_stride=24), -1),
    (dict(row_begin=None), -1), (dict(lens=None), -1), (dict(tables=None), -1), (dict(table_stride=3), -1),
    (dict(mask_words=0), -1), (dict(out=2 * A), -1), (dict(out=2 * A + 40000), -1), (dict(out=3 * A + 1024), -1),
    (dict(out=4 * A - 16), -1), (dict(out=A + 65536), -1), (dict(out_row_stride=4096), -1), (dict(out_head_stride=0), -1),
    (dict(out_head_stride=128), -1), (dict(q_row_stride=1 << 63), -1), (dict(n_rows=1 << 31), -5),
    (dict(table_width=1 << 28, table_stride=1 << 28), -5), (dict(n_reqs=1 << 31), -5)])
def test_attention(lib, bad, status):
    assert attention(lib, **bad) == status
    assert gift.last_error()


def test_attention_without_workspace_or_arguments(lib):
    assert attention(lib, work=None) == gift.E_INVALID
    assert lib.gift_tree_attention(A, ctypes.byref(cache()), ctypes.byref(form()), None, None) == gift.E_INVALID
    assert lib.gift_tree_attention(A, None, ctypes.byref(form()), None, None) == gift.E_INVALID
    assert lib.gift_attention_work_create(None, None) == gift.E_INVALID
    assert lib.gift_attention_work_destroy(None) == gift.OK


def append(lib, kv=None, fmt=None, slots=6 * A, n_slots=5, index=None, **over):
    a = dict(k=2 * A, v=3 * A, n_rows=5, k_layer_stride=10240, k_row_stride=2048, k_head_stride=256,
             v_layer_stride=10240, v_row_stride=2048, v_head_stride=256)
    a.update(over)
    rows = gift._KvRows(*(a[n] for n, _ in gift._KvRows._fields_))
    return lib.gift_kv_append(ctypes.byref(kv or cache()), ctypes.byref(fmt or form()), slots, n_slots, index,
                              ctypes.byref(rows), None)


@pytest.mark.parametrize("bad,status", [
    (dict(slots=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(k=2 * A + 8), -1), (dict(v=3 * A + 2), -1),
    (dict(k_layer_stride=8), -1), (dict(k_row_stride=100), -1), (dict(v_head_stride=4), -1),
    (dict(k_layer_stride=1 << 63), -1), (dict(k=A + 4096), -1), (dict(v=A - 256), -1), (dict(n_slots=1 << 31), -5),
    (dict(n_rows=1 << 31), -5)])
def test_append(lib, bad, status):
    assert append(lib, **bad) == status
    assert gift.last_error()


def tables(lib, **over):
    a = dict(n_reqs=3, block_tokens=16, n_blocks=100, users=A, lens=2 * A, new_lens=3 * A, free_blocks=4 * A, n_free=7,
             table_width=9, table_stride=9, tables=5 * A, block_labels=6 * A, slots=7 * A, n_slots=8, row_begin=8 * A,
             lens_out=9 * A, taken=10 * A, verdicts=11 * A)
    a.update(over)
    step = gift._KvStep(*(a[n] for n, _ in gift._KvStep._fields_))
    return lib.gift_kv_tables(ctypes.byref(step), None)


@pytest.mark.parametrize("bad,status", [
    (dict(block_tokens=0), -1), (dict(block_tokens=12), -1), (dict(users=None), -1), (dict(lens=None), -1),
    (dict(new_lens=None), -1), (dict(free_blocks=None), -1), (dict(tables=None), -1), (dict(block_labels=None), -1),
    (dict(slots=None), -1), (dict(row_begin=None), -1), (dict(lens_out=None), -1), (dict(taken=None), -1),
    (dict(verdicts=None), -1), (dict(table_width=0), -1), (dict(n_blocks=0), -1), (dict(table_stride=8), -1),
    (dict(lens_out=2 * A), -1), (dict(lens_out=3 * A + 8), -1), (dict(verdicts=A), -1), (dict(tables=4 * A + 24), -1),
    (dict(row_begin=7 * A + 60), -1), (dict(taken=11 * A), -1), (dict(table_width=1 << 27, table_stride=1 << 27), -5),
    (dict(n_slots=1 << 31), -5), (dict(table_stride=1 << 63), -1)])
def test_tables(lib, bad, status):
    assert tables(lib, **bad) == status
    assert gift.last_error()


def test_null_structures(lib):
    assert lib.gift_kv_tables(None, None) == gift.E_INVALID
    assert lib.gift_kv_append(ctypes.byref(cache()), ctypes.byref(form()), A, 1, None, None, None) == gift.E_INVALID
    assert lib.gift_kv_append(ctypes.byref(cache()), None, A, 1, None, None, None) == gift.E_INVALID


class Fake:
    """Stands in for a CUDA tensor at a made-up address."""

    is_cuda = True

    def __init__(self, shape, dtype=torch.bfloat16, strides=None):
        t = torch.empty(0, dtype=dtype)
        self.shape, self.dtype, self.size = tuple(shape), dtype, t.element_size()
        self.strides = strides
        if strides is None:
            s, self.strides = 1, []
            for n in reversed(self.shape):
                self.strides.insert(0, s)
                s *= n

    def data_ptr(self):
        return A

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def element_size(self):
        return self.size

    def stride(self, d=None):
        return tuple(self.strides) if d is None else self.strides[d]

    def is_contiguous(self):
        return True


def test_binding_checks_attention_tensors():
    kv, fmt = cache(), form()
    I = torch.int32

    def call(**over):
        a = dict(q=Fake((6, 32, 128)), k=Fake((6, 8, 128)), v=Fake((6, 8, 128)), row_begin=Fake((3,), I), lens=Fake((2,), I),
                 tables=Fake((2, 4), I), out=Fake((6, 32, 128)), mask=Fake((6, 1), I), verdicts=Fake((2,), I),
                 lse=Fake((6, 32), torch.float32))
        a.update(over)
        work = type("W", (), {"handle": None})  # a null handle: the library refuses it, after the binding's checks
        gift.tree_attention(work, kv, fmt, 0, a["q"], a["k"], a["v"], a["row_begin"], a["lens"], a["tables"], a["out"],
                            mask=a["mask"], verdicts=a["verdicts"], lse=a["lse"], stream=0)

    with pytest.raises(gift.GiftError, match="null workspace"):
        call()
    for bad, message in [
            (dict(q=torch.zeros(6, 32, 128, dtype=torch.bfloat16)), "q: tensor must be on the GPU"),
            (dict(q=Fake((6, 32, 64))), "q: shape"), (dict(q=Fake((6, 32, 128), torch.float16)), "q: torch.float16"),
            (dict(k=Fake((5, 8, 128))), "k: shape"), (dict(v=Fake((6, 32, 128))), "v: shape"),
            (dict(q=Fake((6, 32, 128), strides=(8192, 256, 2))), "last dimension"), (dict(out=Fake((6, 8, 128))), "out: shape"),
            (dict(row_begin=Fake((2,), I)), "row_begin: 8 bytes"), (dict(lens=Fake((2,), torch.int64)), "lens: elements of 8"),
            (dict(tables=Fake((1, 4), I)), "tables: needs 2 rows"), (dict(mask=Fake((5, 1), I)), "mask: needs 6 rows"),
            (dict(mask=Fake((6, 1), torch.int64)), "mask: elements of 8"), (dict(verdicts=Fake((1,), I)), "verdicts: 4 bytes"),
            (dict(lse=Fake((6, 31), torch.float32)), "lse: 744 bytes"),
            (dict(tables=Fake((2, 4), I, strides=(8, 2))), "tables: needs")]:
        with pytest.raises(ValueError, match=message):
            call(**bad)


def test_binding_checks_append_and_table_tensors():
    kv, fmt = cache(), form()
    I, L = torch.int32, torch.int64
    k = Fake((4, 6, 8, 128))
    for args, kw, message in [
            ((Fake((5,), I), k, k), {}, "slots: elements of 4"), ((Fake((7,), L), k, k), {}, "k: 6 rows, the call needs 7"),
            ((Fake((5,), L), Fake((3, 6, 8, 128)), k), {}, "k: shape"), ((Fake((5,), L), k, Fake((4, 5, 8, 128))), {}, "v: shape"),
            ((Fake((5,), L), k, k), dict(index=Fake((4,), I)), "index: 16 bytes")]:
        with pytest.raises(ValueError, match=message):
            gift.kv_append(kv, fmt, *args, stream=0, **kw)
    with pytest.raises(ValueError, match="dtype"):
        gift.kv_format(torch.float32, 8, 128, 16, 256, 4096, 32768)
    with pytest.raises(TypeError):
        gift.kv_append(None, fmt, Fake((5,), L), k, k, stream=0)
    one = Fake((3,), I)

    def call(**over):
        a = dict(users=one, lens=one, new=one, free=one, tables=Fake((3, 5), I), labels=one, slots=Fake((9,), L),
                 begin=Fake((4,), I), lens_out=one, taken=one, verdicts=one)
        a.update(over)
        gift.kv_tables(a["users"], a["lens"], a["new"], 16, a["free"], a["tables"], a["labels"], a["slots"], a["begin"],
                       a["lens_out"], a["taken"], a["verdicts"], stream=0)

    for bad, message in [(dict(lens=Fake((2,), I)), "lens: 8 bytes"), (dict(slots=Fake((9,), I)), "slots: elements of 4"),
                         (dict(begin=one), "row_begin: 12 bytes"), (dict(tables=Fake((2, 5), I)), "tables: needs 3 rows"),
                         (dict(free=Fake((3,), L)), "free_blocks: elements of 8"), (dict(verdicts=Fake((2,), I)), "verdicts: 8 bytes")]:
        with pytest.raises(ValueError, match=message):
            call(**bad)
