"""Cache and chunk entry points on a host without a GPU: what they refuse, before any HIP call; sizes; structures."""
import ctypes as C
import os
import subprocess

import pytest

from tests.test_abi_cpu import A, ROOT, _shape, fb

L = fb.lib
OK, EINVAL, EUNSUP, EWS = fb.FASA_OK, fb.FASA_EINVAL, fb.FASA_EUNSUPPORTED, fb.FASA_EWORKSPACE


def cache(fmt="plain", **kw):
    c = fb.make_cache(A, A, fmt)
    if fmt != "plain":
        c.k_scale = c.v_scale = A
        c.scale_stride_b, c.scale_stride_h = 8 * 1024, 1024
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def chunk(s=None, n_new=4, **kw):
    c = fb.make_chunk(s or _shape(), n_new)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def paging(**kw):
    p = fb.FasaPaging(A, 64, 16, 100, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def ref(x):
    return None if x is None else C.byref(x)


def write(s, pg, c, h, k=A, v=A):
    return L.fasa_cache_write(ref(s), ref(pg), ref(c), ref(h), k, v, None)


def read(s, pg, c, T=None, nc=None, n0=0, n1=10, K=A, V=A):
    return L.fasa_cache_read(ref(s), ref(pg), ref(c), T, nc, n0, n1, K, V, None)


def attend(s, pg, c, h, q=A, O=A, ws=A, size=0):
    """with no workspace: what is refused otherwise is refused before"""
    return L.fasa_chunk_attend(ref(s), ref(pg), ref(c), ref(h), q, O, ws, size, None)


def test_everything_is_fine_but_the_workspace():
    for fmt in ("plain", "int8", "e4m3"):
        for pg in (None, paging()):
            assert attend(_shape(), pg, cache(fmt), chunk()) == EWS
    assert attend(_shape(), None, cache(), chunk(row_start=A, n_rows=9, n_new_seq=A, n_ctx_seq=A)) == EWS


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), EINVAL), (dict(n_q_heads=30), EINVAL), (dict(head_dim=64), EUNSUP), (dict(n_q_heads=72), EUNSUP), (dict(n_ctx=0), EINVAL),
    (dict(n_ctx=1025), EINVAL), (dict(n_cap=1000), EINVAL), (dict(kv_stride_n=132), EINVAL), (dict(kv_stride_n=64), EINVAL)])
def test_bad_shapes(kw, code):
    s, ok = _shape(**kw), _shape()
    assert write(s, None, cache(), chunk(ok)) == code
    assert read(s, None, cache()) == code
    assert attend(s, None, cache(), chunk(ok)) == code
    assert write(None, None, cache(), chunk(ok)) == EINVAL
    assert fb.fasa_chunk_workspace_bytes(_shape(n_ctx=0), chunk(ok)) == 0


@pytest.mark.parametrize("fmt,kw", [
    ("plain", dict(K=None)), ("plain", dict(V=None)), ("plain", dict(K=A + 8)), ("plain", dict(format=3)), ("plain", dict(format=-1)),
    ("plain", dict(reserved=1)), ("plain", dict(k_scale=A)), ("plain", dict(v_scale=A)), ("int8", dict(k_scale=None)), ("e4m3", dict(v_scale=None)),
    ("int8", dict(k_scale=A + 4)), ("int8", dict(scale_stride_h=1022)), ("e4m3", dict(scale_stride_b=-4)), ("e4m3", dict(scale_stride_b=6))])
def test_bad_caches(fmt, kw):
    c = cache(fmt, **kw)
    assert write(_shape(), None, c, chunk()) == EINVAL
    assert read(_shape(), None, c) == EINVAL
    assert attend(_shape(), None, c, chunk()) == EINVAL
    assert attend(_shape(), None, None, chunk()) == EINVAL


def test_byte_rows_are_16_byte_aligned():
    s = _shape(kv_stride_n=136)
    assert attend(s, None, cache(), chunk()) == EWS
    assert attend(s, None, cache("int8"), chunk()) == EINVAL and read(s, None, cache("e4m3")) == EINVAL
    assert attend(_shape(kv_stride_h=1024 * 128 + 8), None, cache("int8"), chunk()) == EINVAL


@pytest.mark.parametrize("kw", [dict(n_new=0), dict(n_new=-3), dict(n_new=1001), dict(n_new_seq=A + 2), dict(n_ctx_seq=A + 1), dict(row_start=A + 3, n_rows=9),
                                dict(row_start=A), dict(n_rows=4), dict(row_start=A, n_rows=-1)])
def test_bad_chunks(kw):
    h = chunk(**kw)
    assert write(_shape(), None, cache(), h) == EINVAL
    assert attend(_shape(), None, cache(), h) == EINVAL
    assert fb.fasa_chunk_workspace_bytes(_shape(), h) == 0
    assert write(_shape(), None, cache(), None) == EINVAL


def test_row_strides():
    for kw in (dict(kv_stride=8 * 128 - 8), dict(kv_stride=8 * 128 + 4)):
        assert write(_shape(), None, cache(), chunk(**kw)) == EINVAL
        assert attend(_shape(), None, cache(), chunk(**kw)) == EWS             # (not a stride of this call)
    for kw in (dict(q_stride=32 * 128 - 8), dict(q_stride=32 * 128 + 4), dict(o_stride=31 * 128), dict(o_stride=32 * 128 + 2)):
        assert attend(_shape(), None, cache(), chunk(**kw)) == EINVAL


def test_sizes_beyond_31_bits():
    s = _shape(n_ctx=1 << 30, n_cap=1 << 30, kv_stride_h=0, kv_stride_b=0)
    assert attend(s, None, cache(), chunk(s, 1 << 28)) == EUNSUP
    assert write(s, None, cache(), chunk(s, 1 << 28)) == EUNSUP
    s = _shape(batch=64, n_ctx=1 << 26, n_cap=1 << 26, kv_stride_h=0, kv_stride_b=0)
    assert attend(s, None, cache(), chunk(s, 1 << 26)) == EUNSUP


def test_null_and_misaligned_tensors():
    s = _shape()
    for kw in (dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2)):
        assert write(s, None, cache(), chunk(), **kw) == EINVAL
    for kw in (dict(q=None), dict(O=None), dict(ws=None), dict(q=A + 8), dict(O=A + 4), dict(ws=A + 8)):
        assert attend(s, None, cache(), chunk(), size=1 << 40, **kw) == EINVAL
    for kw in (dict(K=None, V=None), dict(K=A + 8), dict(V=A + 2), dict(nc=A + 2), dict(T=A + 4), dict(n0=-1), dict(n0=11), dict(n1=1001), dict(T=A, n1=101)):
        assert read(s, None, cache(), **kw) == EINVAL
    assert read(_shape(budget=0), None, cache(), T=A) == EINVAL
    assert read(s, None, cache(), n0=7, n1=7) == OK                           # empty range: nothing to do
    assert read(_shape(budget=0), None, cache(), n0=7, n1=7, K=None, V=None) == OK


def test_paging():
    s = _shape()
    for kw, code in ((dict(block_table=None), EINVAL), (dict(block_table=A + 2), EINVAL), (dict(page_size=24), EINVAL), (dict(page_size=0), EINVAL),
                     (dict(max_blocks=62), EINVAL), (dict(n_pool_blocks=0), EINVAL), (dict(reserved=1), EINVAL),
                     (dict(page_size=1024, n_pool_blocks=1 << 22), EUNSUP)):
        pg = paging(**kw)
        assert write(s, pg, cache(), chunk()) == code
        assert attend(s, pg, cache(), chunk()) == code
        assert read(s, pg, cache(), T=A) == code
    assert read(s, paging(max_blocks=2), cache(), n0=5, n1=33) == EINVAL      # the table ends at 32
    assert read(s, paging(max_blocks=2), cache(), n0=5, n1=5) == OK


def test_workspace():
    s = _shape()
    for n_new in (1, 4, 100, 1000):
        h = chunk(n_new=n_new)
        need = fb.fasa_chunk_workspace_bytes(s, h)
        assert need % 256 == 0 and need >= fb.fasa_workspace_bytes(s) and need == fb.fasa_chunk_workspace_bytes(s, h)
    assert fb.fasa_chunk_workspace_bytes(_shape(budget=0), chunk()) == 0 and fb.fasa_chunk_workspace_bytes(s, chunk(q_stride=0)) > 0
    assert attend(_shape(budget=0), None, cache(), chunk()) == EWS             # the budget is not used


def test_lengths_that_31_bits_do_not_hold():
    s = _shape(n_ctx=0x7fff0001, n_cap=0x7fffffc0)
    assert attend(s, None, cache(), chunk()) == EUNSUP and write(s, None, cache(), chunk()) == EUNSUP
    assert fb.fasa_chunk_workspace_bytes(s, chunk()) == 0
    assert attend(_shape(n_ctx=0x7fff0000, n_cap=0x7fffffc0), None, cache(), chunk()) == EWS


def test_binding_raises_and_checks_structures():
    s = _shape()
    with pytest.raises(fb.FasaError) as e:
        fb.fasa_chunk_attend(s, None, cache(), chunk(), A, A, A, 0, stream=0)
    assert e.value.status == EWS
    with pytest.raises(fb.FasaError):
        fb.fasa_cache_write(s, None, cache(), chunk(), None, A, stream=0)
    with pytest.raises(fb.FasaError):
        fb.fasa_cache_read(s, None, cache(), None, None, 5, 4, A, A, stream=0)
    for args in ((s, s, cache(), chunk()), (s, None, chunk(), chunk()), (s, None, cache(), cache())):
        with pytest.raises(C.ArgumentError):
            fb.fasa_chunk_attend(*args, A, A, A, 0, 0)
    with pytest.raises(TypeError):
        fb.fasa_cache_write(s, None, None, chunk(), A, A, 0)


def test_structures_match_the_header(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    items = [(n, t) for n, t in (("fasa_cache", fb.FasaCache), ("fasa_chunk", fb.FasaChunk))]
    prints = ['printf("%%zu\\n", sizeof(%s));' % n for n, _ in items] + ['printf("%%zu\\n", offsetof(%s, %s));' % (n, f) for n, t in items for f, _ in t._fields_]
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fasa.h"\nint main(void) {\n%s\nreturn 0; }\n' % "\n".join(prints))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(t) for _, t in items] + [getattr(t, f).offset for _, t in items for f, _ in t._fields_]
