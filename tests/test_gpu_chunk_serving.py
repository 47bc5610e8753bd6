"""The cache and chunk calls together, as a serving program makes them, and beside the decode step: a prompt in chunks, single tokens, drafted ones, rows read
back for the packed copy and for a selected set."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as CO
from oracle import fasa_oracle as O
from paper_2602_03152_amd import binding as fb
from tests.chunk_util import D, DT, Cache, Chunk, draw_rows, host, tolerance

pytestmark = pytest.mark.gpu


class Server:
    """Sequences that grow chunk by chunk in one paged cache; keeps what was written to check against."""

    def __init__(self, batch, hq, hkv, fmt, dtype, cap, page, seed=0):
        self.hq, self.hkv, self.fmt, self.dtype, self.cap, self.batch = hq, hkv, fmt, dtype, cap, batch
        self.cache = Cache(batch, hkv, cap, fmt, dtype, page, heads_first=page != 32, seed=seed)
        self.shape = self.cache.shape(hq, cap)
        self.len = [0] * batch
        self.rng = np.random.default_rng(seed)
        self.rows = [[[], []] for _ in range(batch)]           # K and V rows as given, per sequence: [n][hkv][D]
        self.nbytes = fb.fasa_chunk_workspace_bytes(self.shape, fb.make_chunk(self.shape, cap))     # enough for all that comes
        self.ws = torch.full((self.nbytes,), 0x5A, dtype=torch.uint8, device="cuda")
        fb.fasa_workspace_init(self.shape, self.ws, self.nbytes)

    def step(self, news, packed):
        """news[b] new tokens of each sequence: their rows written, their queries attended.  Returns the largest error over its bound."""
        self.len = [n + k for n, k in zip(self.len, news)]
        c = Chunk(self.len, news, packed=packed, n_ctx=self.cap)
        chunk = c.make(self.shape, (self.hq, self.hkv))
        kv = [c.buffer(self.hkv, self.dtype)[0] for _ in range(2)]
        q = c.buffer(self.hq, self.dtype)[0]
        out, base = c.buffer(self.hq, self.dtype, fill=7.0)
        for b, n in enumerate(news):
            at = slice(c.start[b], c.start[b] + n)
            if n:
                for i in range(2):
                    x = draw_rows(self.rng, (n, self.hkv, D), self.dtype)
                    kv[i][at] = x.cuda()
                    self.rows[b][i].append(host(x))
                q[at] = draw_rows(self.rng, (n, self.hq, D), self.dtype).cuda()
        fb.fasa_cache_write(self.shape, self.cache.paging, self.cache.cache, chunk, kv[0], kv[1])
        fb.fasa_chunk_attend(self.shape, self.cache.paging, self.cache.cache, chunk, q, out, self.ws, self.nbytes)
        torch.cuda.synchronize()
        G = self.hq // self.hkv
        wide = self.dtype == "bf16" and c.n_new * G > 16
        for b, n in enumerate(news):
            if n == 0:
                continue
            for h in range(self.hkv):
                K, V = (self.stands_for(b, i)[:, h] for i in range(2))
                rows = slice(c.start[b], c.start[b] + n)
                want, A, L = CO.chunk_attend(host(q[rows, h * G:(h + 1) * G]), K, V)
                got = host(out[rows, h * G:(h + 1) * G])
                assert (np.abs(got - want) <= tolerance(want, A, L, self.dtype, wide)).all(), (b, h)

    def stands_for(self, b, i):
        """K (0) or V (1) rows of a sequence as its cache is to hold them, [N][hkv][D]"""
        x = np.concatenate(self.rows[b][i])
        return x if self.fmt == "plain" else CO.dequantise(*CO.quantise(x, self.fmt), self.fmt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["plain", "int8", "e4m3"])
@pytest.mark.parametrize("packed", [False, True])
def test_prompts_in_chunks_then_tokens(fmt, dtype, packed):
    s = Server(3, 8, 2, fmt, dtype, 200, 32 if packed else 16, seed=3)
    s.step([70, 1, 33], packed)           # prompts of different lengths, one of a single token
    s.step([40, 0, 90], packed)           # the rest of two of them, the other waits
    s.step([1, 1, 1], packed)             # a token each
    s.step([4, 2, 0], packed)             # drafted ones
    s.step([1, 130, 1], packed)           # a second prompt beside single tokens
    assert s.len == [116, 134, 125]


@pytest.mark.parametrize("fmt", ["plain", "int8", "e4m3"])
def test_decode_step_over_a_cache_that_is_read_back(fmt):
    """FASA over 8-bit blocks: the dominant dims packed from read keys, scores and selection as always, the selected rows read by list and attended."""
    batch, hq, hkv, F, N, B = 2, 8, 2, 16, 700, 90
    G = hq // hkv
    s = Server(batch, hq, hkv, fmt, "bf16", 704, 16, seed=5)
    s.step([N, N], False)
    shape = s.cache.shape(hq, N, B)
    K = torch.zeros(batch, hkv, N, D, dtype=torch.bfloat16, device="cuda")
    fb.fasa_cache_read(shape, s.cache.paging, s.cache.cache, None, None, 0, N, K, None)
    fc = torch.arange(0, 64, 4, dtype=torch.int32, device="cuda").repeat(hkv, 1).contiguous()
    dense = fb.make_shape(batch, hq, hkv, D, F, N, 704, B, "bf16", kv_stride_b=hkv * N * D, kv_stride_h=N * D)
    Kp = torch.zeros(batch, hkv, F, 704, 2, dtype=torch.bfloat16, device="cuda")
    fb.fasa_pack_kcache(dense, K, fc, Kp, 0, N)
    q = draw_rows(s.rng, (batch, hq, D), "bf16").cuda()
    S = torch.zeros(batch, hkv, 704, device="cuda")
    T = torch.zeros(batch, hkv, B, dtype=torch.int32, device="cuda")
    nbytes = max(fb.fasa_workspace_bytes(dense), s.nbytes)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    fb.fasa_workspace_init(dense, ws, nbytes)
    fb.fasa_score(dense, q, Kp, fc, S)
    fb.fasa_topk(dense, S, T, ws, nbytes)
    KT, VT = (torch.zeros(batch, hkv, B, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fb.fasa_cache_read(shape, s.cache.paging, s.cache.cache, T, None, 0, B, KT, VT)
    rows = fb.make_shape(batch, hq, hkv, D, F, B, 128, B, "bf16", kv_stride_b=hkv * B * D, kv_stride_h=B * D)
    out = torch.zeros(batch, hq, D, device="cuda")
    fb.fasa_dense_attend(rows, q, KT, VT, out, ws, nbytes)
    torch.cuda.synchronize()
    Kf, Tf = K.float().cpu().numpy(), np.sort(T.cpu().numpy(), axis=-1)
    assert np.array_equal(Tf, O.topk(S.cpu().numpy()[:, :, :N], B, N))
    V = np.stack([np.stack([s.stands_for(b, 1)[:N, h] for h in range(hkv)]) for b in range(batch)])
    V = torch.from_numpy(V).to(torch.bfloat16).float().numpy()
    want = O.sparse_attend(host(q).astype(np.float32), Kf, V, Tf)
    assert np.abs(host(out) - want).max() <= 2e-3
    # the same workspace goes on to serve single tokens over all of the cache
    s.ws, s.nbytes = ws, nbytes
    s.step([1, 1], False)


def test_graph_of_a_growing_batch():
    """Write and attention of one token each, captured once; replayed for every token with eager work in between."""
    batch, hq, hkv, cap = 3, 8, 2, 96
    cache = Cache(batch, hkv, cap, "int8", "bf16", 16, seed=4)
    shape = cache.shape(hq, cap)
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    chunk = fb.make_chunk(shape, 1, n_ctx_seq=lens)
    k, v = (torch.zeros(batch, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.zeros(batch, hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    nbytes = fb.fasa_chunk_workspace_bytes(shape, chunk)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    fb.fasa_workspace_init(shape, ws, nbytes)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fb.fasa_cache_write(shape, cache.paging, cache.cache, chunk, k, v)
        fb.fasa_chunk_attend(shape, cache.paging, cache.cache, chunk, q, out, ws, nbytes)
    rng = np.random.default_rng(0)
    for step in range(40):
        lens.copy_(torch.tensor([step + 1, step // 2 + 1, 2 * step + 1], dtype=torch.int32))
        for t in (k, v, q):
            t.copy_(draw_rows(rng, tuple(t.shape), "bf16"))
        out.fill_(9.0)
        g.replay()
        replayed = out.clone()
        fb.fasa_chunk_attend(shape, cache.paging, cache.cache, chunk, q, out, ws, nbytes)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), replayed.view(torch.int16))   # (bits: sequence 2 skips rows, which hold NaN)
        if step % 13 == 0:
            for b, n in enumerate(lens.tolist()):
                for h in range(hkv):
                    if step and b == 2:
                        continue
                    K, V = (cache.rows(w, b, h, np.arange(n)) for w in "KV")
                    want, A, L = CO.chunk_attend(host(q[b:b + 1, 4 * h:4 * h + 4]), K, V)
                    assert (np.abs(host(out[b:b + 1, 4 * h:4 * h + 4]) - want) <= tolerance(want, A, L, "bf16", False)).all()
