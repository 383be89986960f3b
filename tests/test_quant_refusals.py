"""What the calls of the quantised cache refuse, without a GPU: the C entry points check their arguments before they touch a
device, so device addresses are made up here; the binding checks tensors before it calls the library."""
import ctypes
import os

import pytest

from paper_2608_25431_amd import gift

torch = pytest.importorskip("torch")

A = 1 << 40  # a made-up device address, 16-byte aligned
B = 1 << 33  # distance of made-up arrays


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gift.LIB_PATH):
        from paper_2608_25431_amd import build
        build.build()
    yield gift.lib()
    gift.lib().gift_attention_work_destroy(None)  # leaves no message behind for other tests


def made(cls, **values):
    return cls(*(values[n] for n, _ in cls._fields_))


def cache(**over):
    return made(gift._PagedKV, **{**dict(base=A, cache_bytes=4 * 10 * 32768, layer_stride=10 * 32768, block_stride=32768,
                                         part_stride=32768, chunk_bytes=32768, n_layers=4, n_parts=1, n_blocks=10), **over})


def form(**over):
    return made(gift._KvFormat, **{**dict(dtype=gift.E4M3, n_heads=8, head_dim=128, block_tokens=16, k_offset=0,
                                          v_offset=16384, token_stride=128, head_stride=2048), **over})


def factors(cache=None, **over):
    paged = made(gift._PagedKV, **{**dict(base=A + B, cache_bytes=4 * 10 * 1024, layer_stride=10240, block_stride=1024,
                                          part_stride=1024, chunk_bytes=1024, n_layers=4, n_parts=1, n_blocks=10),
                                   **(cache or {})})
    return made(gift._KvScales, **{**dict(cache=paged, k_offset=0, v_offset=512, token_stride=4, head_stride=64), **over})


def caches(a):
    return [ctypes.byref(x) if x is not None else None for x in
            (a.pop("kv", None) or cache(), a.pop("fmt", None) or form(), a.pop("scales", None) or factors())]


def append(lib, **over):
    a = dict(layer=0, n_layers=4, slots=A + 2 * B, n_slots=6, index=None, dtype=gift.BF16, k=A + 3 * B, v=A + 4 * B, n_rows=6,
             k_layer_stride=1 << 16, k_row_stride=2048, k_head_stride=256, v_layer_stride=1 << 16, v_row_stride=2048,
             v_head_stride=256)
    a.update(over)
    c = caches(a)
    rows = made(gift._KvRows, **{n: a[n] for n, _ in gift._KvRows._fields_})
    return lib.gift_kv_append_quant(*c, a["layer"], a["n_layers"], a["slots"], a["n_slots"], a["index"],
                                    ctypes.byref(rows) if a.get("rows", 1) else None, a["dtype"], None)


def read(lib, **over):
    a = dict(k=A + 3 * B, v=A + 4 * B, n_rows=6, k_layer_stride=1 << 16, k_row_stride=2048, k_head_stride=256,
             v_layer_stride=1 << 16, v_row_stride=2048, v_head_stride=256, dtype=gift.BF16, layer=0, n_layers=4, n_reqs=2,
             row_begin=A + 5 * B, first=None, lens=A + 6 * B, tables=A + 7 * B, table_width=4, table_stride=4, verdicts=None)
    a.update(over)
    c = caches(a)
    return lib.gift_kv_read_quant(*c, ctypes.byref(made(gift._KvRead, **a)), None)


def attention(lib, work=A, **over):
    a = dict(n_rows=6, n_reqs=2, n_heads=32, layer=0, dtype=gift.BF16, scale=0.1, q=A + 2 * B, out=A + 3 * B, lse=A + 4 * B,
             q_row_stride=8192, q_head_stride=256, out_row_stride=8192, out_head_stride=256, row_begin=A + 5 * B,
             lens=A + 6 * B, tables=A + 7 * B, table_width=4, table_stride=4, mask=A + 8 * B, mask_words=1, verdicts=None)
    a.update(over)
    c = caches(a)
    return lib.gift_quant_attention(work, *c, ctypes.byref(made(gift._QuantAttention, **a)), None)


def qk(lib, **over):
    a = dict(n_rows=6, q_heads=32, k_heads=8, head_dim=128, dtype=gift.BF16, q=A, k=A + B, q_out=A + 2 * B, k_out=A + 3 * B,
             q_row_stride=8192, q_head_stride=256, k_row_stride=2048, k_head_stride=256, q_out_row_stride=8192,
             q_out_head_stride=256, k_out_row_stride=2048, k_out_head_stride=256, q_weight=A + 4 * B, k_weight=A + 5 * B,
             eps=1e-6, rotary_dim=128, interleaved=0, n_axes=2, sections=(40, 24, 0, 0), inv_freq=A + 6 * B,
             positions=A + 7 * B, position_stride=6)
    a.update(over)
    a["sections"] = (ctypes.c_uint32 * 4)(*a["sections"])
    return lib.gift_qk_norm_rope(ctypes.byref(made(gift._QkRows, **a)), None)


BAD_CACHES = [
    dict(kv=cache(base=None)), dict(kv=cache(chunk_bytes=32752)), dict(kv=cache(n_layers=0)),
    dict(fmt=form(dtype=gift.BF16)), dict(fmt=form(dtype=4)), dict(fmt=form(head_dim=80)), dict(fmt=form(n_heads=0)),
    dict(fmt=form(block_tokens=24)), dict(fmt=form(token_stride=136)), dict(fmt=form(token_stride=112)),
    dict(fmt=form(head_stride=1024)), dict(fmt=form(n_heads=17)), dict(fmt=form(v_offset=16)),
    dict(scales=factors(dict(base=None))), dict(scales=factors(dict(n_layers=3))), dict(scales=factors(dict(n_blocks=9))),
    dict(scales=factors(dict(chunk_bytes=1000))), dict(scales=factors(dict(chunk_bytes=512))),
    dict(scales=factors(dict(base=A + 16))), dict(scales=factors(k_offset=2)), dict(scales=factors(token_stride=3)),
    dict(scales=factors(head_stride=62)), dict(scales=factors(token_stride=0)), dict(scales=factors(head_stride=32)),
    dict(scales=factors(v_offset=4)), dict(scales=factors(v_offset=1 << 63)), dict(scales=factors(v_offset=516)),
    # 8 bytes a row
    dict(fmt=form(head_dim=256, n_heads=4, token_stride=256, head_stride=4096), scales=factors(token_stride=12)),
    dict(fmt=form(head_dim=256, n_heads=4, token_stride=256, head_stride=4096), scales=factors(v_offset=516)),
]


@pytest.mark.parametrize("how", BAD_CACHES)
def test_caches(lib, how):
    for call in (append, read, attention):
        assert call(lib, **how) == gift.E_INVALID


def test_null_arguments(lib):
    kv, fmt, x = (ctypes.byref(y) for y in (cache(), form(), factors()))
    for bad in ((None, fmt, x), (kv, None, x), (kv, fmt, None)):
        assert lib.gift_kv_append_quant(*bad, 0, 4, A, 1, None, None, gift.BF16, None) == gift.E_INVALID
        assert lib.gift_kv_read_quant(*bad, ctypes.byref(gift._KvRead()), None) == gift.E_INVALID
        assert lib.gift_quant_attention(A, *bad, ctypes.byref(gift._QuantAttention()), None) == gift.E_INVALID
    assert append(lib, rows=None) == gift.E_INVALID
    assert lib.gift_kv_read_quant(kv, fmt, x, None, None) == gift.E_INVALID
    assert lib.gift_quant_attention(A, kv, fmt, x, None, None) == gift.E_INVALID
    assert lib.gift_quant_attention(None, kv, fmt, x, ctypes.byref(gift._QuantAttention()), None) == gift.E_INVALID
    assert lib.gift_qk_norm_rope(None, None) == gift.E_INVALID


def test_chunks_past_the_cache(lib):
    for how in (dict(kv=cache(cache_bytes=4 * 10 * 32768 - 1)), dict(scales=factors(dict(cache_bytes=40 * 1024 - 1)))):
        for call in (append, read, attention):
            assert call(lib, **how) == gift.E_RANGE


@pytest.mark.parametrize("how", [
    dict(dtype=0), dict(dtype=gift.E4M3), dict(layer=1), dict(layer=5, n_layers=0), dict(n_layers=5),
    dict(layer=0xFFFFFFFF, n_layers=2), dict(slots=None), dict(slots=A + 2 * B + 4), dict(index=A + 2), dict(k=None), dict(v=None),
    dict(k=A + 8), dict(k_row_stride=2056), dict(v_layer_stride=8), dict(k_layer_stride=1 << 63), dict(k=A + 32768),
    dict(v=A + B + 512), dict(slots=A + B + 8), dict(index=A + 4)])
def test_append(lib, how):
    assert append(lib, **how) == gift.E_INVALID


def test_sizes_past_the_range(lib):
    assert append(lib, n_slots=1 << 31) == gift.E_TOO_LARGE
    assert append(lib, n_rows=1 << 31) == gift.E_TOO_LARGE
    assert read(lib, n_rows=1 << 31) == gift.E_TOO_LARGE
    assert read(lib, table_width=1 << 27, table_stride=1 << 27) == gift.E_TOO_LARGE
    assert attention(lib, n_rows=1 << 31) == gift.E_TOO_LARGE
    assert attention(lib, n_rows=1 << 28) == gift.E_TOO_LARGE  # times 32 heads
    assert attention(lib, table_width=1 << 27, table_stride=1 << 27) == gift.E_TOO_LARGE
    assert qk(lib, n_rows=1 << 31) == gift.E_TOO_LARGE
    assert qk(lib, n_rows=1 << 30, position_stride=1 << 30) == gift.E_TOO_LARGE  # times 40 heads


def test_nothing_to_do(lib):
    """Calls without rows, layers or heads do nothing, and ask for none of their arrays."""
    assert append(lib, n_slots=0, slots=None, k=None, v=None) == gift.OK
    assert append(lib, n_layers=0, k=None, v=None) == gift.OK
    assert append(lib, n_rows=0, k=None, v=None) == gift.OK
    assert read(lib, n_rows=0, k=None, v=None) == gift.OK
    assert read(lib, n_layers=0, k=None, v=None) == gift.OK
    assert read(lib, n_reqs=0, row_begin=None, lens=None, tables=None) == gift.OK
    assert qk(lib, n_rows=0, q=None, k=None, positions=None) == gift.OK
    assert qk(lib, q_heads=0, k_heads=0) == gift.OK


@pytest.mark.parametrize("how", [
    dict(dtype=0), dict(layer=1), dict(layer=5, n_layers=0), dict(row_begin=None), dict(lens=None), dict(tables=None),
    dict(table_stride=3), dict(lens=A + 2), dict(first=A + 1), dict(k=None), dict(v=A + 8), dict(k_row_stride=2056),
    dict(k=A), dict(v=A + B), dict(k=A + 5 * B), dict(v=A + 6 * B), dict(first=A + 3 * B), dict(verdicts=A + 4 * B),
    dict(tables=A + 3 * B + 64),
    # rows that overlap: by stride, and K's with V's
    dict(k_row_stride=1024), dict(k_head_stride=128), dict(v_layer_stride=0), dict(k_layer_stride=1 << 63),
    dict(v=A + 3 * B), dict(v=A + 3 * B + 1024), dict(v=A + 3 * B + 2048)])
def test_read(lib, how):
    assert read(lib, **how) == gift.E_INVALID


def test_keys_and_values_in_one_buffer(lib):
    """K and V heads beside each other in a row: refused for the device that is not there, not for the arrays."""
    wide = dict(v=A + 3 * B + 2048, k_row_stride=4096, v_row_stride=4096)
    assert read(lib, **wide) != gift.E_INVALID
    assert read(lib, **{**wide, "v_row_stride": 8192}) == gift.E_INVALID
    # queries and keys in place, in the buffer of a projection
    wide = dict(q=A, q_out=A, k=A + 8192, k_out=A + 8192, **{f"{x}_row_stride": 12288 for x in ("q", "k", "q_out", "k_out")})
    assert qk(lib, **wide) != gift.E_INVALID
    assert qk(lib, **{**wide, "k": A + 8192 - 256, "k_out": A + 8192 - 256}) == gift.E_INVALID
    assert qk(lib, **{**wide, "k_out": A + 8192 + 256}) == gift.E_INVALID
    assert qk(lib, **{**wide, "k_row_stride": 10240, "k_out_row_stride": 10240}) == gift.E_INVALID


@pytest.mark.parametrize("how", [
    dict(work=None), dict(dtype=0), dict(dtype=gift.E4M3), dict(n_heads=0), dict(n_heads=12), dict(layer=4),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(row_begin=None), dict(lens=None), dict(tables=None),
    dict(table_stride=3), dict(mask_words=0), dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 3 * B + 8),
    dict(q_row_stride=8200), dict(out_head_stride=264), dict(out_head_stride=128), dict(out_row_stride=4096),
    dict(lse=A + 4 * B + 2), dict(mask=A + 1), dict(out=A + 32768), dict(out=A + B), dict(lse=A + B), dict(lse=A + 4),
    dict(out=A + 2 * B), dict(lse=A + 3 * B), dict(out=A + 5 * B), dict(lse=A + 6 * B), dict(mask=A + 3 * B),
    dict(verdicts=A + 4 * B), dict(out_row_stride=1 << 63)])
def test_attention(lib, how):
    assert attention(lib, **how) == gift.E_INVALID


@pytest.mark.parametrize("how", [
    dict(dtype=0), dict(dtype=gift.E4M3), dict(head_dim=32), dict(head_dim=112), dict(eps=-1e-6), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(rotary_dim=144), dict(rotary_dim=120), dict(rotary_dim=64), dict(interleaved=2), dict(n_axes=0),
    dict(n_axes=5), dict(n_axes=1), dict(sections=(40, 25, 0, 0)), dict(sections=(0xFFFFFFFF, 65, 0, 0)), dict(position_stride=5),
    dict(inv_freq=None), dict(positions=None), dict(inv_freq=A + 2), dict(positions=A + 2), dict(q=None), dict(k_out=None),
    dict(q=A + 8), dict(k_weight=A + 8), dict(q_row_stride=8200), dict(k_out_head_stride=8), dict(q_row_stride=1 << 63),
    # outputs that overlap: themselves, their inputs, the other side, and what the call reads
    dict(q_out_head_stride=128), dict(q_out_row_stride=4096), dict(k_out_row_stride=0), dict(q_out=A + 256),
    dict(q_out=A, q_out_row_stride=16384), dict(q_out=A + B), dict(k_out=A + 2 * B), dict(k_out=A), dict(q_weight=A + 2 * B + 512),
    dict(k_weight=A + 2 * B), dict(inv_freq=A + 3 * B + 16), dict(positions=A + 2 * B + 8)])
def test_qk(lib, how):
    assert qk(lib, **how) == gift.E_INVALID


def test_binding():
    t = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        gift.qk_norm_rope(t, None, t, None)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        gift.qk_norm_rope(t.float(), None, t, None)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        gift.kv_append_quant(cache(), form(), factors(), torch.zeros(1, dtype=torch.int64), t.view(torch.float8_e4m3fn), t)
    with pytest.raises(TypeError):
        gift.kv_append_quant(cache(), form(), None, torch.zeros(1, dtype=torch.int64), t, t)
    with pytest.raises(TypeError):
        gift.kv_scales(None, 512, 4, 64)
    with pytest.raises(ValueError, match="on the GPU"):
        gift.kv_read_quant(cache(), form(), factors(), None, torch.zeros(1, dtype=torch.int32), None, t, t)
    with pytest.raises(ValueError, match="on the GPU"):
        gift.quant_attention(None, cache(), form(), factors(), 0, t, None, torch.zeros(1, dtype=torch.int32), None, t)
    assert gift.kv_format(torch.float8_e4m3fn, 8, 128, 16, 128, 2048, 16384).dtype == gift.E4M3
