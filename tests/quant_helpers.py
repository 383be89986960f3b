"""Helpers of the quantised cache's tests: references in 64 bits written from the definitions in include/gift_kv.h, and a
quantised cache with its requests."""
import numpy as np
import torch

from kv_helpers import DEV, DT, NO_BLOCK, i32
from paper_2608_25431_amd import gift

GROUP = 32
NAN = 0x7F


def _element(b):
    e, m = b >> 3 & 15, b & 7
    v = np.nan if (b & 127) == NAN else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -v if b & 128 else v


ELEMENTS = np.array([_element(b) for b in range(256)])  # what each byte stands for, apart from its factor
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # of a rounding to the type, relative
LEAST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}  # and below its normal range, absolute
LARGEST = {"bf16": 255 * 2.0 ** 120, "f16": 65504.0}


def quantised(x, dtype):
    """Bytes of the elements of rows (..., dim) of 64-bit values that are of `dtype`, and of their factors."""
    y = x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    fine = np.isfinite(y)
    top = np.abs(np.where(fine, y, 0)).max(-1)
    power = np.full(top.shape, 27 - 127)  # the smallest with top <= 448 * 2^power
    while (top > 448 * 2.0 ** power).any():
        power = np.where(top > 448 * 2.0 ** power, power + 1, power)
    z = np.where(fine, y, 0) / 2.0 ** power[..., None]
    step = 2.0 ** np.maximum(np.frexp(z)[1] - 4, -9)
    z = np.round(z / step) * step  # ties to even
    z = np.where(np.abs(z) * 2.0 ** power[..., None] > LARGEST[dtype], np.sign(z) * 240, z)
    b = np.searchsorted(ELEMENTS[:NAN], np.abs(z)).astype(np.uint8)
    b = np.where(fine, b, NAN).astype(np.uint8) | (np.signbit(y) * 128).astype(np.uint8)
    return b.reshape(x.shape), (power + 127).astype(np.uint8)


def rounded(x, dtype):
    """64-bit values of 64-bit values rounded to the type."""
    with np.errstate(over="ignore"):
        if dtype == "f16":
            return x.astype(np.float16).astype(np.float64)
        return torch.from_numpy(x).to(torch.float32).to(DT[dtype]).double().numpy()  # elements have few bits: one rounding


def values(elements, factors, dtype):
    y = ELEMENTS[elements].reshape(elements.shape[:-1] + (elements.shape[-1] // GROUP, GROUP))
    y = y * 2.0 ** (factors[..., :y.shape[-2]].astype(np.float64) - 127)[..., None]
    return rounded(y.reshape(elements.shape), dtype)


class QuantCache:
    """A quantised paged cache.  Every element is NaN and every factor 2^128 at first: what no request owns must not count."""

    def __init__(self, heads, dim, block, n_blocks, n_layers=1, order="head", parts=1, device=DEV):
        self.heads, self.dim, self.block, self.n_blocks, self.n_layers, self.parts = heads, dim, block, n_blocks, n_layers, parts
        self.space = 8 if dim == 256 else 4
        self.data, self.k, self.v, self.geo = self._make(dim, order, NAN, device)
        self.factors, self.kf, self.vf, self.fgeo = self._make(self.space, order, 255, device)

    def _make(self, row, order, fill, device):
        plane = self.heads * self.block * row
        token, head = (row, self.block * row) if order == "head" else (self.heads * row, row)
        chunk = max(16, 1 << (plane * (1 if self.parts == 2 else 2) - 1).bit_length())
        v_off = chunk if self.parts == 2 else plane
        block = chunk * self.parts
        layer = block * self.n_blocks
        data = torch.full((layer * self.n_layers,), fill, dtype=torch.uint8, device=device)
        shape, strides = (self.n_layers, self.n_blocks, self.block, self.heads, row), (layer, block, token, head, 1)
        return (data, torch.as_strided(data, shape, strides, 0), torch.as_strided(data, shape, strides, v_off),
                (layer, block, token, head, chunk, v_off))

    def args(self):
        paged = [gift.paged_kv(data, data.numel(), g[0], g[1], g[4], g[4], self.n_layers, self.parts, self.n_blocks)
                 for data, g in ((self.data, self.geo), (self.factors, self.fgeo))]
        _, _, token, head, _, v_off = self.geo
        fmt = gift.kv_format(torch.float8_e4m3fn, self.heads, self.dim, self.block, token, head, v_off)
        _, _, token, head, _, v_off = self.fgeo
        return paged[0], fmt, gift.kv_scales(paged[1], v_off, token, head)


class Requests:
    """Requests with all their tokens, those of their rows last, in scattered blocks of a quantised cache."""

    def __init__(self, lens, rows, dtype="bf16", heads=2, group=2, dim=64, block=16, order="head", parts=1, n_layers=2,
                 layer=1, mask=None, seed=0, spare=2, q_scale=1.0, kv_scale=(1.0, 1.0)):
        r = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.lens, self.rows, self.dtype, self.layer, self.group = np.asarray(lens), np.asarray(rows), dtype, layer, group
        n, have = len(lens), -(-self.lens // block)
        self.cache = QuantCache(heads, dim, block, int(have.sum()) + spare, n_layers, order, parts)
        self.width = max(1, int(have.max()) if n else 1) + 1
        self.tab = np.full((n, self.width), NO_BLOCK, np.int64)
        self.tab[np.arange(self.width)[None, :] < have[:, None]] = r.permutation(self.cache.n_blocks)[:have.sum()]
        total, count = int(self.lens.sum()), int(self.rows.sum())
        x = torch.randn(2, total, heads, dim, generator=g) * torch.tensor(kv_scale).view(2, 1, 1, 1)
        b, f = quantised(x.to(DT[dtype]).double().numpy(), dtype)
        self.pos = np.concatenate([np.arange(x) for x in self.lens]) if total else np.zeros(0, np.int64)
        self.req = np.repeat(np.arange(n), self.lens)
        at = (torch.from_numpy(self.tab[self.req, self.pos // block]).to(DEV), torch.from_numpy(self.pos % block).to(DEV))
        c = self.cache
        for i, (elements, factors) in enumerate(((c.k, c.kf), (c.v, c.vf))):
            elements[layer][at] = torch.from_numpy(b[i]).to(DEV)
            pad = np.zeros((total, heads, c.space), np.uint8)
            pad[..., :f.shape[-1]] = f[i]
            factors[layer][at] = torch.from_numpy(pad).to(DEV)
        self.k, self.v = values(b, f, dtype)
        self.q = (torch.randn(count, heads * group, dim, generator=g) * q_scale).to(DT[dtype])
        self.begin = np.concatenate([[0], np.cumsum(self.rows)])
        self.bits = None
        if mask is not None:
            words = max(1, -(-int(self.rows.max()) // 32)) if n else 1
            self.bits = np.zeros((count, 32 * words), np.uint8)
            for b in range(n):
                for i in range(self.rows[b]):
                    row = self.begin[b] + i
                    if i:
                        self.bits[row] = self.bits[self.begin[b] + r.integers(max(0, i - 6), i)]
                    self.bits[row, i] = 1
            if mask == "holes":
                self.bits[r.random(count) < 0.4] = 0
            elif mask == "random":
                self.bits = (r.random(self.bits.shape) < 0.5).astype(np.uint8)  # bits past the rows are set too
        self.verdicts = None

    def mask_words(self):
        if self.bits is None:
            return None
        return torch.from_numpy(np.packbits(self.bits, axis=1, bitorder="little").view(np.int32).copy()).to(DEV)

    def run(self, work, out=None, lse=True, **over):
        """The call on the GPU; returns (out, lse) on the host."""
        q = self.q.to(DEV)
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV) if out is None else out
        ls = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV) if lse else None
        a = dict(row_begin=i32(self.begin), lens=i32(self.lens), tables=i32(self.tab), mask=self.mask_words(),
                 verdicts=None if self.verdicts is None else i32(self.verdicts), scale=None, stream=None)
        a.update(over)
        gift.quant_attention(work, *self.cache.args(), self.layer, q, a["row_begin"], a["lens"], a["tables"], out,
                             mask=a["mask"], verdicts=a["verdicts"], lse=ls, scale=a["scale"], stream=a["stream"])
        torch.cuda.synchronize()
        return out.cpu(), None if ls is None else ls.cpu()

    def seen(self, b):
        """Which of request b's tokens its rows see."""
        d, length = int(self.rows[b]), int(self.lens[b])
        j = np.arange(length)[None, :] - (length - d)  # tokens' numbers among the rows' own
        i = np.arange(d)[:, None]
        if self.bits is None:
            return j <= i
        bits = self.bits[self.begin[b]:self.begin[b + 1]].astype(bool)
        at = np.clip(j, 0, bits.shape[1] - 1)
        return (j < 0) | (np.take_along_axis(bits, np.broadcast_to(at, (d, length)), 1) & (j < bits.shape[1]))

    def expect(self, scale=None, unseen=None):
        """(out, lse, bound on out, bound on lse) in 64 bits.

        K and V are exact.  Scores are sums of dim products in 32 bits, off by e <= (dim + 8) 2^-24 sum |q k| scale, and
        their exponentials by 2^-20 and 2^-22 of the score more.  A weight is rounded to the type once (the sum of the weights
        is of unrounded ones), and so is the output.  With u half a step of the type,
            |out - exact| <= u |out| + (u + 2 e) sum p |v|
        and f16 weights below 2^-29 of the largest are off by 2^-39 of it, which is less than LEAST for each key."""
        q = self.q.double().numpy()
        h, g, dim = self.cache.heads, self.group, self.cache.dim
        u = HALF_STEP[self.dtype]
        scale = dim ** -0.5 if scale is None else scale
        out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
        tol, ltol = np.zeros(q.shape), np.zeros(q.shape[:2])
        first = np.concatenate([[0], np.cumsum(self.lens)])
        for b in range(len(self.lens)):
            lo, hi = self.begin[b], self.begin[b + 1]
            if lo == hi or (self.verdicts is not None and self.verdicts[b]):
                continue
            see = self.seen(b)
            if unseen is not None:
                see[:, unseen(b, np.arange(int(self.lens[b])))] = False
            for j in range(h * g):
                kk, vv = (x[first[b]:first[b + 1], j // g] for x in (self.k, self.v))
                for i in range(hi - lo):
                    some = np.nonzero(see[i])[0]
                    if not len(some):
                        continue
                    s = kk[some] @ q[lo + i, j] * scale
                    m = s.max()
                    p = np.exp(s - m)
                    total = p.sum()
                    with np.errstate(invalid="ignore"):
                        o = (p[:, None] * vv[some]).sum(0) / total
                        size = (p[:, None] * np.abs(vv[some])).sum(0) / total
                    out[lo + i, j], lse[lo + i, j] = o, m + np.log(total)
                    e = (dim + 8) * 2.0 ** -24 * (np.abs(kk[some]) @ np.abs(q[lo + i, j])).max() * abs(scale)
                    e += 2.0 ** -22 * np.abs(s).max() + 2.0 ** -20
                    tol[lo + i, j] = u * np.abs(o) + (u + 2 * e) * size + LEAST[self.dtype] * (len(some) + 1)
                    ltol[lo + i, j] = e + 2.0 ** -22 * abs(lse[lo + i, j])
        return out, lse, tol, ltol

    def check(self, got, **how):
        out, lse, tol, ltol = self.expect(**how)
        o = got[0].double().numpy()
        number = np.isfinite(out)
        assert (np.isfinite(o) == number).all(), f"{(np.isfinite(o) != number).sum()} outputs are finite or not, wrongly"
        over = np.where(number, np.abs(np.where(number, o - out, 0)) - tol, -1)
        assert (over <= 0).all(), f"out: {(over > 0).sum()} of {over.size} outside, worst {over.max():.3g} over " \
            f"{tol.flat[over.argmax()]:.3g} at {np.unravel_index(over.argmax(), over.shape)}"
        if got[1] is not None:
            l = got[1].double().numpy()
            none = np.isinf(lse)
            assert (l[none] == -np.inf).all(), "rows that see nothing"
            off = np.abs(l[~none] - lse[~none])
            assert (off <= ltol[~none]).all(), f"lse: worst {off.max():.3g}"
