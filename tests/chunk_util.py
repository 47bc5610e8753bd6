"""Caches, chunks and their oracle for the tests of fasa_cache_write, fasa_cache_read and fasa_chunk_attend."""
from __future__ import annotations

import numpy as np
import torch

from oracle import chunk_oracle as CO
from paper_2602_03152_amd import binding as fb

D = 128
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def host(t):
    """Values of a tensor in float64; stored bytes as they are."""
    return t.cpu().numpy() if t.dtype == torch.uint8 else t.detach().double().cpu().numpy()


class Cache:
    """A cache of `batch` sequences of up to `cap` tokens, paged (page > 0) or not, of any format, filled with rubbish that no result
    may depend on: NaN bits in plain rows and scales."""

    def __init__(self, batch, hkv, cap, fmt, dtype, page=16, heads_first=True, seed=0, gap=0, spare=3):
        self.batch, self.hkv, self.cap, self.fmt, self.dtype, self.page = batch, hkv, cap, fmt, dtype, page
        rng = np.random.default_rng(seed)
        size = page or (cap + 15) // 16 * 16
        self.size, nb = size, (cap + size - 1) // size
        blocks = batch * nb + (spare if page else 0)
        self.heads_first = heads_first or not page
        shape = (blocks, hkv, size + gap, D) if self.heads_first else (blocks, size + gap, hkv, D)
        store = torch.uint8 if fmt != "plain" else DT[dtype]
        fill = 0x7f if fmt != "plain" else float("nan")
        self.K = torch.full(shape, fill, dtype=store, device="cuda")
        self.V = torch.full(shape, fill, dtype=store, device="cuda")
        self.ks = self.vs = None
        if fmt != "plain":
            self.ks = torch.full((blocks, hkv, (size + 3) // 4 * 4), float("nan"), device="cuda")
            self.vs = torch.full_like(self.ks, float("nan"))
        table = rng.permutation(blocks)[:batch * nb].reshape(batch, nb).astype(np.int32) if page else np.arange(batch, dtype=np.int32)[:, None]
        self.table = torch.from_numpy(np.ascontiguousarray(table)).cuda()
        self.paging = fb.make_paging(self.table, page, blocks) if page else None
        self.cache = fb.make_cache(self.K, self.V, fmt, self.ks, self.vs)
        st = self.K.stride()
        self.strides = dict(kv_stride_b=st[0], kv_stride_h=st[1] if self.heads_first else st[2], kv_stride_n=st[2] if self.heads_first else st[1])

    def shape(self, hq, n_ctx, budget=1):
        return fb.make_shape(self.batch, hq, self.hkv, D, 16, n_ctx, (max(n_ctx, self.cap) + 63) // 64 * 64, budget, self.dtype, **self.strides)

    def at(self, b, n):
        """(block, offset) of tokens n of sequence b"""
        n = np.asarray(n)
        return self.table.cpu().numpy()[b, n // self.size], n % self.size

    def stored(self, which, b, h, n):
        """Stored rows and scales of tokens n."""
        pool, scale = (self.K, self.ks) if which == "K" else (self.V, self.vs)
        blk, off = (torch.from_numpy(np.ascontiguousarray(x)).cuda().long() for x in self.at(b, n))
        rows = pool[blk, h, off] if self.heads_first else pool[blk, off, h]
        return rows, None if scale is None else scale[blk, h, off]

    def put(self, b, h, k, v):
        """Tokens 0 .. of sequence b, head h, from float64 rows, through the oracle's format."""
        n = np.arange(len(k))
        blk, off = (torch.from_numpy(np.ascontiguousarray(x)).cuda().long() for x in self.at(b, n))
        for x, pool, scale in ((k, self.K, self.ks), (v, self.V, self.vs)):
            if self.fmt == "plain":
                rows = torch.from_numpy(x).cuda().to(pool.dtype)
            else:
                codes, s = CO.quantise(x, self.fmt)
                rows = torch.from_numpy(codes).cuda()
                scale[blk, h, off] = torch.from_numpy(s).cuda()
            if self.heads_first:
                pool[blk, h, off] = rows
            else:
                pool[blk, off, h] = rows

    def rows(self, which, b, h, n):
        """What tokens n stand for, float64."""
        r, s = self.stored(which, b, h, n)
        return host(r) if s is None else CO.dequantise(host(r), s.cpu().numpy(), self.fmt)


def draw_rows(rng, shape, dtype, gain=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * gain).to(DT[dtype])


class Chunk:
    """The new tokens of sequences of lens tokens, news of them new; packed: rows one after another in the order `order`, with pad rows
    behind each sequence, at the start and at the end; stride_gap: elements between rows beyond dense ones."""

    def __init__(self, lens, news, packed=False, n_new=None, n_ctx=None, by_seq=True, stride_gap=0, seed=0):
        self.lens, self.news = list(lens), list(news)
        self.n_new = n_new or max(max(news), 1)
        self.n_ctx = n_ctx or max(max(lens), 1)
        self.gap, self.batch = stride_gap, len(lens)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
        self.n_new_seq, self.n_ctx_seq = (i32(news), i32(lens)) if by_seq else (None, None)
        self.start = [b * self.n_new for b in range(self.batch)]
        self.n_rows, self.row_start = self.batch * self.n_new, None
        if packed:
            at, self.start = 2, [0] * self.batch
            for b in np.random.default_rng(seed).permutation(self.batch):
                self.start[b] = at
                at += self.news[b] + int(b % 2)
            self.n_rows = at + 1
            self.row_start = i32(self.start)

    def make(self, shape, heads):
        return fb.make_chunk(shape, self.n_new, self.n_new_seq, self.n_ctx_seq, self.row_start, self.n_rows if self.row_start is not None else 0,
                             q_stride=heads[0] * D + self.gap, kv_stride=heads[1] * D + self.gap, o_stride=heads[0] * D + self.gap)

    def buffer(self, heads, dtype, fill=float("nan")):
        """[n_rows][heads][D] with the chunk's stride, filled; the second result is the memory it lies in."""
        base = torch.full((self.n_rows, heads * D + self.gap), fill, dtype=DT[dtype], device="cuda")
        return base[:, :heads * D].view(self.n_rows, heads, D) if not self.gap else base[:, :heads * D].unflatten(1, (heads, D)), base


def tolerance(O, A, L, dtype, wide):
    """How far O may be from the oracle's, element by element.
    Logits: a float32 sum of d products, scaled (and, of 8-bit rows, scaled once more): off by at most (d + 4) 2^-24 L, L = sum |q_i k_i| / sqrt(d).
    A weight is off by as much of itself, once in the numerator and once in the sum of weights: 2 (d + 4) 2^-24 L A, A = the weighted mean of |V|; exp2
    (an ulp or two), the sums over tokens and the merges: 2^-18 A.
    bf16: O is rounded once, 2^-8 |O|, and the weights go into the product with V as bf16 numbers (wide: 2^-8 A) or as two (2^-15 A)."""
    e = (2 * (D + 4) * 2.0 ** -24 * L[..., None] + 2.0 ** -18) * A
    if dtype == "bf16":
        e = e + 2.0 ** -8 * np.abs(O) + (2.0 ** -8 if wide else 2.0 ** -15) * A
    return e + 1e-30
