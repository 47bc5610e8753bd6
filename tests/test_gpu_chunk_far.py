"""Caches whose rows lie beyond 2^31 elements and 2^32 bytes, rows far apart, and lengths at the lines between the kernels' forms."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as CO
from paper_2602_03152_amd import binding as fb
from tests.chunk_util import D, DT, draw_rows, host, tolerance

pytestmark = pytest.mark.gpu


def _run(shape, paging, cache, n, hq, hkv, rows_of, seed, dtype="bf16"):
    """n new tokens written through the cache call, then attended: against the oracle on what rows_of(which, h) says the cache stands for."""
    rng = np.random.default_rng(seed)
    chunk = fb.make_chunk(shape, n)
    k, v = (draw_rows(rng, (n, hkv, D), dtype).cuda() for _ in range(2))
    fb.fasa_cache_write(shape, paging, cache, chunk, k, v)
    q = draw_rows(rng, (n, hq, D), dtype).cuda()
    out = torch.zeros(n, hq, D, dtype=DT[dtype], device="cuda")
    nbytes = fb.fasa_chunk_workspace_bytes(shape, chunk)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    fb.fasa_workspace_init(shape, ws, nbytes)
    fb.fasa_chunk_attend(shape, paging, cache, chunk, q, out, ws, nbytes)
    N = shape.n_ctx
    back = torch.zeros(1, hkv, N, D, dtype=DT[dtype], device="cuda")
    fb.fasa_cache_read(shape, paging, cache, None, None, 0, N, back, None)
    torch.cuda.synchronize()
    G = hq // hkv
    for h in range(hkv):
        K, V = rows_of(0, h, k, v), rows_of(1, h, k, v)
        want, A, L = CO.chunk_attend(host(q[:, h * G:(h + 1) * G]), K, V)
        got = host(out[:, h * G:(h + 1) * G])
        assert (np.abs(got - want) <= tolerance(want, A, L, dtype, dtype == "bf16" and n * G > 16)).all(), h
        assert torch.equal(back[0, h].cpu(), torch.from_numpy(K).to(DT[dtype]))


@pytest.mark.parametrize("fmt", ["plain", "int8", "e4m3"])
@pytest.mark.parametrize("n", [3, 40, 200])
def test_blocks_beyond_4_gib(fmt, n):
    hq, hkv, page, N = 4, 1, 16, 200
    row = D * (2 if fmt == "plain" else 1)
    blocks = (5 << 30) // (page * hkv * row)
    pool = [torch.empty(blocks, page, hkv, D, dtype=torch.bfloat16 if fmt == "plain" else torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(blocks, hkv, page, device="cuda") if fmt != "plain" else None for _ in range(2)]
    nb = (N + page - 1) // page
    table = torch.from_numpy((blocks - 1 - np.random.default_rng(0).permutation(4 * nb)[:nb]).astype(np.int32))[None].cuda()
    table[0, 1] = 3
    shape = fb.make_shape(1, hq, hkv, D, 16, N, 256, 1, "bf16", kv_stride_b=page * hkv * D, kv_stride_h=D, kv_stride_n=hkv * D)
    paging, cache = fb.make_paging(table, page, blocks), fb.make_cache(pool[0], pool[1], fmt, scale[0], scale[1])
    rng = np.random.default_rng(1)
    first = [draw_rows(rng, (N, hkv, D), "bf16") for _ in range(2)]
    whole = fb.make_chunk(shape, N)
    fb.fasa_cache_write(shape, paging, cache, whole, first[0].cuda(), first[1].cuda())

    def rows_of(i, h, k, v):
        x = np.concatenate([host(first[i])[:N - n, h], host((k, v)[i])[:, h]])
        return x if fmt == "plain" else CO.dequantise(*CO.quantise(x, fmt), fmt)
    _run(shape, paging, cache, n, hq, hkv, rows_of, 2)


@pytest.mark.parametrize("stride,N,n", [(1 << 24, 200, 3), (1 << 24, 200, 100), (1 << 27, 24, 2), (1 << 27, 24, 24)])
def test_rows_far_apart(stride, N, n):
    """A contiguous cache of rows 32 or 256 MiB apart (the latter beyond what the fastest form multiplies in 32 bits)."""
    hq, hkv = 8, 1
    base = [torch.empty((N - 1) * stride + D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shape = fb.make_shape(1, hq, hkv, D, 16, N, 256, 1, "bf16", kv_stride_b=0, kv_stride_h=0, kv_stride_n=stride)
    cache = fb.make_cache(base[0], base[1])
    rng = np.random.default_rng(3)
    first = [draw_rows(rng, (N, hkv, D), "bf16") for _ in range(2)]
    fb.fasa_cache_write(shape, None, cache, fb.make_chunk(shape, N), first[0].cuda(), first[1].cuda())
    rows_of = lambda i, h, k, v: np.concatenate([host(first[i])[:N - n, h], host((k, v)[i])[:, h]])   # noqa: E731
    _run(shape, None, cache, n, hq, hkv, rows_of, 4)


@pytest.mark.parametrize("fmt", ["plain", "int8"])
@pytest.mark.parametrize("G,n", [(1, 16), (1, 17), (4, 4), (4, 5), (8, 2), (8, 3), (1, 128), (1, 129), (4, 32), (4, 33), (7, 18), (7, 19), (8, 64), (8, 65), (1, 257)])
@pytest.mark.parametrize("N", [300, 1027])
def test_lines_between_the_forms(fmt, G, n, N):
    """Query rows of a KV head around 16, 128 and 256, tokens around whole tiles."""
    hkv, page = 2, 16
    blocks = (N + page - 1) // page
    pool = [torch.zeros(blocks, hkv, page, D, dtype=torch.bfloat16 if fmt == "plain" else torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(blocks, hkv, page, device="cuda") if fmt != "plain" else None for _ in range(2)]
    table = torch.arange(blocks, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    shape = fb.make_shape(1, hkv * G, hkv, D, 16, N, (N + 63) // 64 * 64, 1, "bf16", kv_stride_b=page * hkv * D, kv_stride_h=page * D, kv_stride_n=D)
    paging, cache = fb.make_paging(table, page, blocks), fb.make_cache(pool[0], pool[1], fmt, scale[0], scale[1])
    rng = np.random.default_rng(G * n)
    first = [draw_rows(rng, (N, hkv, D), "bf16") for _ in range(2)]
    fb.fasa_cache_write(shape, paging, cache, fb.make_chunk(shape, N), first[0].cuda(), first[1].cuda())

    def rows_of(i, h, k, v):
        x = np.concatenate([host(first[i])[:N - n, h], host((k, v)[i])[:, h]])
        return x if fmt == "plain" else CO.dequantise(*CO.quantise(x, fmt), fmt)
    _run(shape, paging, cache, n, hkv * G, hkv, rows_of, 5)


@pytest.mark.parametrize("batch", [2, 63, 64, 65])
def test_many_sequences(batch):
    """Up to 64 sequences of different lengths are shared out by length, more are not."""
    from tests.test_gpu_chunk_attend import build, call, check
    lens = [(37 * b) % 211 + 1 for b in range(batch)]
    t = build(lens, [1 + b % 2 for b in range(batch)], 4, 1, "e4m3", seed=batch)
    t["c"].news = [min(n, m) for n, m in zip(t["c"].news, lens)]
    call(t)
    check(t)
    t = build(lens, [min(n, 1 + b % 9) for b, n in enumerate(lens)], 4, 1, "plain", seed=batch, packed=True)
    call(t)
    check(t)


def test_rows_that_overlap_leave_the_workspace_prepared():
    """Two sequences on the same rows, more new tokens than there are rows: not allowed, but it ends, and the next call is right."""
    from tests.test_gpu_chunk_attend import build, call, check
    t = build([300, 280, 260], [2, 2, 2], 4, 1, seed=2, packed=True)
    good = t["c"].row_start.clone()
    t["c"].row_start.zero_()
    call(t)
    torch.cuda.synchronize()
    t["c"].row_start.copy_(good)
    t["base"].fill_(77.0)
    for _ in range(2):
        call(t)
        check(t)


def _many_heads(fmt, dtype, batch, hkv, G, N, lens, paged, n, page=16):
    hq = hkv * G
    byte = fmt != "plain"
    pool = [torch.zeros(batch, hkv, N, D, dtype=torch.uint8 if byte else DT[dtype], device="cuda") for _ in range(2)]
    pitch = (N + 3) // 4 * 4
    scale = [torch.zeros(batch, hkv, pitch, device="cuda") if byte else None for _ in range(2)]
    paging = None
    shape = fb.make_shape(batch, hq, hkv, D, 16, N, (N + 63) // 64 * 64, 1, dtype, kv_stride_b=hkv * N * D, kv_stride_h=N * D, kv_stride_n=D)
    if paged:                             # the same rows as blocks [block][page][head]
        blocks = batch * ((N + page - 1) // page)
        pool = [torch.zeros(blocks, page, hkv, D, dtype=torch.uint8 if byte else DT[dtype], device="cuda") for _ in range(2)]
        scale = [torch.zeros(blocks, hkv, page, device="cuda") if byte else None for _ in range(2)]
        table = torch.randperm(blocks, generator=torch.Generator().manual_seed(N), dtype=torch.int32).reshape(batch, -1).contiguous().cuda()
        paging = fb.make_paging(table, page, blocks)
        shape = fb.make_shape(batch, hq, hkv, D, 16, N, (N + 63) // 64 * 64, 1, dtype, kv_stride_b=page * hkv * D, kv_stride_h=D, kv_stride_n=hkv * D)
    cache = fb.make_cache(pool[0], pool[1], fmt, scale[0], scale[1])
    len_t = torch.tensor(lens, dtype=torch.int32, device="cuda") if len(set(lens)) > 1 else None
    gen = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn(batch * N, hkv, D, generator=gen, device="cuda", dtype=DT[dtype]) for _ in range(2))
    whole = fb.make_chunk(shape, N, n_new_seq=len_t, n_ctx_seq=len_t)
    fb.fasa_cache_write(shape, paging, cache, whole, k, v)
    q = torch.randn(batch * n, hq, D, generator=gen, device="cuda", dtype=DT[dtype]) * 2
    out = torch.zeros_like(q)
    chunk = fb.make_chunk(shape, n, n_ctx_seq=len_t)
    nbytes = fb.fasa_chunk_workspace_bytes(shape, chunk)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    fb.fasa_workspace_init(shape, ws, nbytes)
    fb.fasa_chunk_attend(shape, paging, cache, chunk, q, out, ws, nbytes)
    torch.cuda.synchronize()
    for b, m in enumerate(lens):
        for h in (0, hkv - 1):
            K, V = (host(x[b * N:b * N + m, h]) for x in (k, v))
            if byte:
                K, V = (CO.dequantise(*CO.quantise(x, fmt), fmt) for x in (K, V))
            rows = slice(b * n, b * n + n)
            want, A, L = CO.chunk_attend(host(q[rows, h * G:h * G + G]), K, V)
            assert (np.abs(host(out[rows, h * G:h * G + G]) - want) <= tolerance(want, A, L, dtype, dtype == "bf16" and n * G > 16)).all(), (b, h)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("fmt,dtype,batch,hkv,N", [("plain", "bf16", 1, 260, 4500), ("int8", "bf16", 1, 260, 8500), ("e4m3", "f32", 1, 260, 8700),
                                                   ("plain", "bf16", 2, 128, 9000), ("e4m3", "bf16", 2, 128, 17000)])
@pytest.mark.parametrize("n", [1, 4])
def test_parts_of_many_tiles(fmt, dtype, batch, hkv, N, paged, n):
    """So many KV heads that a workgroup has all of a sequence, or half: beyond the 64 tiles whose blocks a wave's lanes look up at once."""
    _many_heads(fmt, dtype, batch, hkv, 1, N, [N, N - 777][:batch], paged, n)


@pytest.mark.parametrize("fmt,paged", [("plain", True), ("int8", False)])
@pytest.mark.parametrize("hkv,G,n,N,batch", [(100, 8, 96, 3000, 1),      # two whole tiles a head, the third in two parts
                                             (64, 8, 160, 3100, 1),      # four, the fifth in four
                                             (32, 8, 160, 6000, 1),      # five, each in three parts, two rounds
                                             (64, 4, 200, 4001, 2),      # eight of two sequences
                                             (64, 7, 50, 5000, 3)])      # two a sequence, six in all
def test_full_rounds_and_parts(fmt, paged, hkv, G, n, N, batch):
    """More 256-row tiles than workgroups run at once, or almost as many: whole ones, then parts."""
    _many_heads(fmt, "bf16", batch, hkv, G, N, [N] * batch, paged, n)


@pytest.mark.parametrize("fmt,page", [("plain", 0), ("plain", 4), ("int8", 8), ("e4m3", 32), ("int8", 0)])
@pytest.mark.parametrize("G,n", [(1, 129), (1, 300), (3, 43), (7, 37), (7, 74), (8, 33), (4, 129)])
@pytest.mark.parametrize("lens", [[1025], [1087], [1531, 700], [1600, 300, 1100, 1025]])
def test_256_row_tiles_at_odd_sizes(fmt, page, G, n, lens):
    """The kernel of many query rows where tiles, tokens and blocks end anywhere; sequences of unequal lengths, one as long as its new tokens."""
    _many_heads(fmt, "bf16", len(lens), 66, G, max(lens), [max(m, n) for m in lens], page > 0, n, max(page, 1))


@pytest.mark.parametrize("n,page", [(40, 16), (40, 4), (20, 16), (20, 1)])
def test_many_rows_captured(n, page):
    """Parts and their merge in one graph, replayed as lengths change, with the program's own calls in between."""
    from tests.test_gpu_chunk_attend import build, call
    t = build([1100, 900], [n, n], 80, 20, "plain", page=page, seed=n, n_ctx=1200)
    lens = t["c"].n_ctx_seq
    call(t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(t)
    for a, b in ((1100, 900), (61, 333), (1090, 25), (700, 899), (1100, 900)):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        t["base"].fill_(77.0)
        call(t)
        eager = t["O"].clone()
        t["base"].fill_(77.0)
        g.replay()
        assert torch.equal(t["O"], eager), (a, b)


@pytest.mark.parametrize("fmt,paged", [("plain", True), ("int8", False), ("e4m3", True)])
@pytest.mark.parametrize("dtype,hkv,G,n,N,batch", [("f32", 64, 1, 70, 900, 1), ("f32", 64, 4, 33, 1200, 2), ("f32", 1, 1, 4800, 5000, 1), ("bf16", 64, 4, 4, 3000, 5),
                                                   ("bf16", 100, 8, 1, 2500, 3)])
def test_full_rounds_and_parts_of_16_row_tiles(dtype, hkv, G, n, N, batch, fmt, paged):
    _many_heads(fmt, dtype, batch, hkv, G, N, [N] * batch, paged, n)
