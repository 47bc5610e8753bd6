"""fasa_chunk_attend against the float64 oracle: from single tokens to chunks, ragged, packed, paged and contiguous, every format."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as CO
from paper_2602_03152_amd import binding as fb
from tests.chunk_util import D, Cache, Chunk, draw_rows, host, tolerance

pytestmark = pytest.mark.gpu


def build(lens, news, hq, hkv, fmt="plain", dtype="bf16", page=16, heads_first=True, seed=0, gain=1.0, gap=0, **kw):
    """A filled cache, a chunk, q and O of it, a prepared workspace."""
    rng = np.random.default_rng(seed)
    c = Chunk(lens, news, seed=seed, **kw)
    cache = Cache(len(lens), hkv, c.n_ctx, fmt, dtype, page, heads_first, seed, gap)
    for b, n in enumerate(lens):
        for h in range(hkv):
            if n:
                cache.put(b, h, host(draw_rows(rng, (n, D), dtype, gain)), host(draw_rows(rng, (n, D), dtype)))
    shape = cache.shape(hq, c.n_ctx)
    chunk = c.make(shape, (hq, hkv))
    q, _ = c.buffer(hq, dtype)
    for b in range(len(lens)):
        if news[b]:
            q[c.start[b]:c.start[b] + news[b]] = draw_rows(rng, (news[b], hq, D), dtype).cuda()
    O, base = c.buffer(hq, dtype, fill=77.0)
    nbytes = fb.fasa_chunk_workspace_bytes(shape, chunk)
    ws = torch.full((nbytes,), 0x5A, dtype=torch.uint8, device="cuda")
    fb.fasa_workspace_init(shape, ws, nbytes)
    return dict(c=c, cache=cache, shape=shape, chunk=chunk, q=q, O=O, base=base, ws=ws, nbytes=nbytes, hq=hq, hkv=hkv, dtype=dtype)


def call(t, stream=None):
    fb.fasa_chunk_attend(t["shape"], t["cache"].paging, t["cache"].cache, t["chunk"], t["q"], t["O"], t["ws"], t["nbytes"], stream)


def expected(t):
    """{(b, h): (O, A, L)} of the oracle"""
    c, G = t["c"], t["hq"] // t["hkv"]
    out = {}
    for b, (N, n) in enumerate(zip(c.lens, c.news)):
        n = min(n, N)
        if n == 0:
            continue
        tok = np.arange(N)
        for h in range(t["hkv"]):
            q = host(t["q"][c.start[b]:c.start[b] + n, h * G:(h + 1) * G])
            out[b, h] = CO.chunk_attend(q, t["cache"].rows("K", b, h, tok), t["cache"].rows("V", b, h, tok))
    return out


def check(t, want=None):
    c, G = t["c"], t["hq"] // t["hkv"]
    torch.cuda.synchronize()
    got = host(t["base"]).copy()
    assert np.isfinite(got).all()
    wide = t["dtype"] == "bf16" and c.n_new * G > 16
    untouched = np.ones(c.n_rows, bool)
    for (b, h), (O, A, L) in (want or expected(t)).items():
        n = O.shape[0]
        rows = slice(c.start[b], c.start[b] + n)
        untouched[rows] = False
        g = got[rows, :t["hq"] * D].reshape(n, t["hq"], D)[:, h * G:(h + 1) * G]
        over = np.abs(g - O) - tolerance(O, A, L, t["dtype"], wide)
        assert over.max() <= 0, "sequence %d head %d: %.3g over the bound at %s" % (b, h, over.max(), np.unravel_index(over.argmax(), over.shape))
    assert (got[untouched] == 77.0).all(), "rows of no sequence were written"
    if c.gap:
        assert (got[:, t["hq"] * D:] == 77.0).all(), "what lies between two rows was written"


FORMATS = ["plain", "int8", "e4m3"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 63, 65, 300, 1531])
def test_single_tokens(fmt, dtype, N):
    t = build([N, max(1, N - 3)], [1, 1], 8, 2, fmt, dtype, seed=N)
    call(t)
    check(t)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8])
@pytest.mark.parametrize("n", [1, 2, 4, 5, 17, 33])
def test_groups_and_chunk_lengths(G, n):
    t = build([n + 70], [n], 2 * G, 2, "plain", seed=10 * G + n)
    call(t)
    check(t)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [0, 1, 2, 4, 8, 16, 64, 256])
@pytest.mark.parametrize("heads_first", [True, False])
def test_page_sizes_and_layouts(fmt, page, heads_first):
    for n in (1, 9, 40):
        t = build([203, 77], [n, n], 8, 2, fmt, page=page, heads_first=heads_first, seed=page + n, gap=0 if n == 1 else 16)
        call(t)
        check(t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("packed", [False, True])
def test_mixed_lengths(fmt, dtype, packed):
    """Sequences without tokens, without new ones, all new, one new; padded and packed, rows with gaps."""
    lens, news = [0, 1, 100, 259, 65, 300, 17], [0, 1, 0, 1, 65, 33, 9]
    t = build(lens, news, 12, 3, fmt, dtype, seed=5, packed=packed, stride_gap=24 if packed else 0)
    call(t)
    check(t)


def test_lengths_are_clamped():
    """Negative and too large lengths on the device, first rows that are out of range: clamped, as documented."""
    t = build([300, 40, 0, 20], [5, 40, 0, 20], 8, 2, seed=3, n_new=40, n_ctx=300)
    t["c"].n_ctx_seq.copy_(torch.tensor([1000, 40, -7, 20], dtype=torch.int32))
    t["c"].n_new_seq.copy_(torch.tensor([5, 400, 3, 1 << 30], dtype=torch.int32))
    call(t)
    check(t)
    t = build([300, 40, 50], [5, 12, 4], 8, 2, seed=4, packed=True)
    t["c"].row_start.copy_(torch.tensor([-5, t["c"].n_rows - 3, 1 << 30], dtype=torch.int32))
    t["q"].normal_()
    call(t)
    t["c"].start, t["c"].news = [0, t["c"].n_rows - 3, 0], [5, 3, 0]
    check(t)


def test_table_entries_out_of_range_and_behind_the_end_do_no_harm():
    t = build([130, 37], [3, 37], 8, 2, "int8", seed=6, n_ctx=300)
    want = expected(t)
    table = t["cache"].table
    table[0, 9:] = 1 << 30
    table[1, 3:] = -1
    call(t)
    check(t, want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [1, 20, 130])
def test_large_logits(fmt, n):
    """Logits of some hundreds: nearly all weight on a token or two."""
    t = build([n + 333], [n], 8, 2, fmt, seed=n, gain=30.0)
    call(t)
    check(t)


NOT_FINITE = [("bf16", "plain", 2, 4, 70), ("bf16", "int8", 2, 4, 70), ("f32", "e4m3", 2, 20, 70), ("f32", "plain", 2, 20, 70), ("bf16", "plain", 2, 40, 333),
              ("bf16", "int8", 2, 40, 333), ("bf16", "e4m3", 40, 70, 1100), ("bf16", "plain", 40, 70, 1100)]


@pytest.mark.parametrize("dtype,fmt,hkv,n,N,which", [(*case, w) for case in NOT_FINITE for w in (["K"] if case[1] == "plain" else ["K", "V", "both"])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_token_that_is_not_finite_reaches_no_earlier_one(dtype, fmt, hkv, n, N, which, bad):
    """The chunk's last but two token has a row of NaN or infinities: tokens before it are as without, those from it on are NaN.  (Plain rows of V have to be finite.)"""
    t = build([N], [n], 4 * hkv, hkv, fmt, dtype, seed=n, page=16)
    k, v = (draw_rows(np.random.default_rng(n), (n, hkv, D), dtype).cuda() for _ in range(2))
    fb.fasa_cache_write(t["shape"], t["cache"].paging, t["cache"].cache, t["chunk"], k, v)
    call(t)
    good = t["O"].clone()
    if which != "V":
        k[n - 3] = bad
    if which != "K":
        v[n - 3] = bad
    fb.fasa_cache_write(t["shape"], t["cache"].paging, t["cache"].cache, t["chunk"], k, v)
    call(t)
    torch.cuda.synchronize()
    first = t["c"].start[0]
    assert torch.equal(t["O"][first:first + n - 3], good[first:first + n - 3])
    assert not torch.isfinite(t["O"][first + n - 3:first + n].float()).any()


def test_equal_keys_give_the_mean():
    t = build([129], [17], 4, 1, seed=1)
    t["cache"].K.fill_(0.5)
    call(t)
    check(t)


@pytest.mark.parametrize("n", [1, 3, 40])
def test_many_splits_and_again(n):
    """A long cache shared out to many workgroups; the workspace is prepared for the next call, of other sizes too."""
    t = build([9001], [n], 8, 2, "int8", seed=n)
    call(t)
    check(t)
    first = t["O"].clone()
    s = build([333, 500], [1, 1], 8, 2, seed=9)
    s["ws"], s["nbytes"] = t["ws"], t["nbytes"]
    assert s["nbytes"] >= fb.fasa_chunk_workspace_bytes(s["shape"], s["chunk"])
    fb.fasa_workspace_init(s["shape"], s["ws"], s["nbytes"])
    for _ in range(3):
        call(s)
        check(s)
    call(t)
    torch.cuda.synchronize()
    assert torch.equal(first, t["O"])         # no order of additions that changes


def test_rows_do_not_depend_on_their_neighbours_or_on_when():
    """Two streams with workspaces of their own, at once."""
    a, b = build([700, 800], [2, 2], 8, 2, seed=1), build([900], [40], 8, 2, "e4m3", seed=2)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        call(a, sa)
        call(b, sb)
    check(a)
    check(b)


@pytest.mark.parametrize("n", [1, 24])
def test_captured_and_replayed_as_lengths_grow(n):
    t = build([300, 200], [n, n], 8, 2, "int8", seed=8, n_ctx=300)
    lens, news = t["c"].n_ctx_seq, t["c"].n_new_seq
    call(t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(t)
    for step in range(4):
        t["c"].lens = [300 - 70 * step, 200 - 50 * step]
        t["c"].news = [n, max(1, n - 7 * step)]
        lens.copy_(torch.tensor(t["c"].lens, dtype=torch.int32))
        news.copy_(torch.tensor(t["c"].news, dtype=torch.int32))
        t["base"].fill_(77.0)
        g.replay()
        check(t)
