"""fasa_cache_write and fasa_cache_read: formats against the float64 oracle, bit for bit; what is not written stays."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as CO
from paper_2602_03152_amd import binding as fb
from tests.chunk_util import D, DT, Cache, Chunk, draw_rows, host

pytestmark = pytest.mark.gpu
FORMATS = ["plain", "int8", "e4m3"]


def awkward(rng, shape, dtype):
    """Rows of every kind: ordinary, multiples of half a step (ties), tiny, huge, zero, one value, subnormal."""
    x = rng.standard_normal(shape)
    flat = x.reshape(-1, D)
    for i in range(len(flat)):
        kind = i % 9
        if kind == 1:      # a scale that is a power of two, values on ties of int8 and e4m3
            flat[i] = rng.integers(-254, 255, D) / 2.0
            flat[i, 0] = 127.0
        elif kind == 2:
            flat[i] = rng.integers(-40, 41, D) * 2.0 ** rng.integers(-12, 3, D) / 16
            flat[i, 5] = 448.0
        elif kind == 3:
            flat[i] *= 1e-30
        elif kind == 4:
            flat[i] *= 1e37
        elif kind == 5:
            flat[i] = 0
        elif kind == 6:
            flat[i] = 0
            flat[i, 77] = -3.7
        elif kind == 7:
            flat[i] *= 2.0 ** -131
        elif kind == 8:
            flat[i] *= 2.0 ** rng.integers(-20, 20, D)
    return torch.from_numpy(x).to(DT[dtype])


def write(lens, news, hkv, fmt, dtype, page=16, heads_first=True, seed=0, make=awkward, gap=0, **kw):
    rng = np.random.default_rng(seed)
    c = Chunk(lens, news, seed=seed, **kw)
    cache = Cache(len(lens), hkv, c.n_ctx, fmt, dtype, page, heads_first, seed, gap)
    shape = cache.shape(hkv, c.n_ctx)
    new = []
    for _ in range(2):
        x, _base = c.buffer(hkv, dtype)
        for b in range(len(lens)):
            if news[b]:
                x[c.start[b]:c.start[b] + news[b]] = make(rng, (news[b], hkv, D), dtype).cuda()
        new.append(x)
    before = [None if t is None else t.clone() for t in (cache.K, cache.V, cache.ks, cache.vs)]
    fb.fasa_cache_write(shape, cache.paging, cache.cache, c.make(shape, (hkv, hkv)), new[0], new[1])
    torch.cuda.synchronize()
    return c, cache, shape, new, before


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def check_written(c, cache, new, before, hkv):
    touched = [torch.zeros(x.shape[:-1] if i < 2 else x.shape, dtype=torch.bool) for i, x in enumerate(before) if x is not None]
    for b, (N, n) in enumerate(zip(c.lens, c.news)):
        if n == 0:
            continue
        tok = np.arange(N - n, N)
        blk, off = cache.at(b, tok)
        for h in range(hkv):
            for i, which in enumerate("KV"):
                x = new[i][c.start[b]:c.start[b] + n, h]
                rows, scale = cache.stored(which, b, h, tok)
                if cache.fmt == "plain":
                    assert np.array_equal(bits(rows), bits(x))
                else:
                    codes, s = CO.quantise(host(x), cache.fmt)
                    got_s = scale.cpu().numpy()
                    assert np.array_equal(got_s.view(np.uint32), s.view(np.uint32)), "scales"
                    # (-0 and +0 are the same number of either format's)
                    same = CO.values(host(rows), cache.fmt) == CO.values(codes, cache.fmt)
                    assert same.all(), "codes: %s" % [(host(x)[r, j], s[r], host(rows)[r, j], codes[r, j]) for r, j in np.argwhere(~same)[:3]]
                if cache.heads_first:
                    touched[i][blk, h, off] = True
                else:
                    touched[i][blk, off, h] = True
                if scale is not None:
                    touched[2 + i][blk, h, off] = True
    now = [t for t in (cache.K, cache.V, cache.ks, cache.vs) if t is not None]
    for i, (x, y) in enumerate(zip(now, [t for t in before if t is not None])):
        keep = ~touched[i]
        assert np.array_equal(bits(x.cpu()[keep]), bits(y.cpu()[keep])), "what is not of the chunk was written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("packed", [False, True])
def test_write_mixed_lengths(fmt, dtype, packed):
    lens, news = [0, 1, 100, 259, 65, 300], [0, 1, 0, 1, 65, 33]
    c, cache, _, new, before = write(lens, news, 3, fmt, dtype, seed=2, packed=packed, stride_gap=8)
    check_written(c, cache, new, before, 3)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [0, 1, 8, 32])
@pytest.mark.parametrize("heads_first", [True, False])
def test_write_page_sizes_and_layouts(fmt, page, heads_first):
    c, cache, _, new, before = write([70, 41], [50, 41], 5, fmt, "bf16", page, heads_first, seed=page, gap=2)
    check_written(c, cache, new, before, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_many_values_are_the_nearest_code(fmt, dtype):
    """100000 rows: a code that is off next to a tie shows in some of them."""
    rng = np.random.default_rng(11)
    n, hkv = 2048, 8
    make = lambda r, s, d: draw_rows(r, s, d, 1.0) * torch.from_numpy(2.0 ** r.integers(-8, 8, (s[0], s[1], 1))).to(DT[d])   # noqa: E731
    c, cache, _, new, before = write([n], [n], hkv, fmt, dtype, 64, seed=int(rng.integers(1000)), make=make, by_seq=False)
    check_written(c, cache, new, before, hkv)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_rows_with_infinities_and_nans(fmt):
    def make(rng, shape, dtype):
        x = draw_rows(rng, shape, dtype)
        x[1, 0, 3], x[2, 1, 127], x[3, 0, 0] = float("inf"), float("nan"), float("-inf")
        return x
    c, cache, shape, new, before = write([5], [5], 2, fmt, "bf16", make=make)
    check_written(c, cache, new, before, 2)
    out = torch.zeros(1, 2, 5, D, dtype=torch.bfloat16, device="cuda")
    fb.fasa_cache_read(shape, cache.paging, cache.cache, None, None, 0, 5, out, None)
    bad = torch.isnan(out).any(-1).cpu().numpy()[0]
    assert np.array_equal(bad, [[False, True, False, True, False], [False, False, True, False, False]])
    assert torch.isnan(out[0, 0, 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [0, 4, 32])
def test_read_range(fmt, dtype, page):
    lens, hkv = [200, 0, 77, 131], 3
    c, cache, shape, new, _ = write(lens, lens, hkv, fmt, dtype, page, seed=4, make=draw_rows)
    for n0, n1 in ((0, 200), (13, 150), (199, 200), (5, 5)):
        out = [torch.full((4, hkv, n1 - n0, D), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
        fb.fasa_cache_read(shape, cache.paging, cache.cache, None, c.n_ctx_seq, n0, n1, out[0], out[1])
        torch.cuda.synchronize()
        for b, N in enumerate(lens):
            end = max(n0, min(n1, N))
            for h in range(hkv):
                for o, which in zip(out, "KV"):
                    if end > n0:
                        want = torch.from_numpy(cache.rows(which, b, h, np.arange(n0, end))).to(DT[dtype])
                        assert torch.equal(o[b, h, :end - n0].cpu(), want)
                    assert (o[b, h, end - n0:] == 7.0).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_read_list(fmt):
    """Entries in any order, twice, out of range; only K, only V; a part of the list."""
    lens, hkv, B = [200, 90], 2, 150
    c, cache, shape, new, _ = write(lens, lens, hkv, fmt, "bf16", 16, seed=4, make=draw_rows)
    shape.budget = B
    rng = np.random.default_rng(1)
    T = rng.integers(0, 200, (2, hkv, B)).astype(np.int32)
    T[1] %= 90
    T[0, 0, 7], T[0, 1, 8], T[1, 0, 9] = -4, 1 << 30, 95
    Td = torch.from_numpy(T).cuda()
    for n0, n1, use in ((0, B, "KV"), (20, 61, "K"), (80, B, "V")):
        out = [torch.full((2, hkv, n1 - n0, D), 7.0, dtype=torch.bfloat16, device="cuda") if w in use else None for w in "KV"]
        fb.fasa_cache_read(shape, cache.paging, cache.cache, Td, c.n_ctx_seq, n0, n1, out[0], out[1])
        torch.cuda.synchronize()
        for b, N in enumerate(lens):
            end = min(n1, B, N)
            for h in range(hkv):
                for o, which in zip(out, "KV"):
                    if o is None:
                        continue
                    tok = np.clip(T[b, h, n0:end], 0, N - 1)
                    assert torch.equal(o[b, h, :end - n0].cpu(), torch.from_numpy(cache.rows(which, b, h, tok)).to(torch.bfloat16))
                    assert (o[b, h, end - n0:] == 7.0).all()
