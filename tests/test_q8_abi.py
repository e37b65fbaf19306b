"""The 8-bit cache's entry points without a GPU: exported symbols, layout, workspace sizes, and the refusal of every bad argument
before anything is launched."""
import ctypes as C
import os

import numpy as np
import pytest

from paper_2505_18231_amd import api
from tests import q8_reference as R

FAKE = 0x10000   # an aligned address that no call may reach
FAR = 1 << 44


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(api.LIB_PATH):
        from paper_2505_18231_amd.build import build_library
        build_library(verbose=False)
    return api.lib()


def shape(**kw):
    s = api.make_q8_shape(128, 32, 8, 1024)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def cache(**kw):
    c = api.nsn_q8_cache(FAKE, FAKE, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(data=FAKE, b=0, h=128, t=1024):
    return api.nsn_rows(data, b, h, t)


@pytest.mark.parametrize("D", [64, 128])
def test_offsets_are_the_header_s_and_a_bijection(L, D):
    s = api.make_q8_shape(D, 8, 2, 256)
    for kind, fn in (("k", L.nsn_q8_k_code_offset), ("v", L.nsn_q8_v_code_offset)):
        got = np.array([[fn(C.byref(s), t, c) for c in range(D)] for t in range(128)])
        assert np.array_equal(got, R.offsets(kind, D, 128))
        assert sorted(got.ravel().tolist()) == list(range(128 * D))
        assert fn(C.byref(s), -1, 0) == -1 and fn(C.byref(s), 0, D) == -1 and fn(C.byref(s), 0, -1) == -1
    assert L.nsn_q8_v_code_offset(C.byref(s), (1 << 40) + 1, 0) == (1 << 40) * D + (D // 16)


BAD_SHAPES = [(dict(head_dim=96), -2), (dict(code_type=2), -2), (dict(io_type=2), -2), (dict(io_type=-1), -2), (dict(n_q_heads=12), -1),
              (dict(n_kv_heads=0), -1), (dict(n_q_heads=0), -1), (dict(n_q_heads=65536, n_kv_heads=1), -1), (dict(max_len=100), -1),
              (dict(max_len=0), -1), (dict(page_size=48), -1), (dict(page_size=-64), -1), (dict(page_size=192, n_pages=5), -1),
              (dict(page_size=64, n_pages=0), -1), (dict(n_q_heads=32768, n_kv_heads=32768), -1), (dict(max_len=(1 << 30) + 64), -1)]


def append(L, s, k=None, v=None, max_new=4, start=FAKE, n=FAKE, batch=1, kc=None, vc=None):
    return L.nsn_q8_append(C.byref(s), C.byref(k or rows()), C.byref(v or rows()), max_new, start, n, batch,
                           C.byref(kc or cache()), C.byref(vc or cache(codes=FAR, scales=FAR)), None)


def attend(L, s, q=None, n_q=1, q_lens=None, kc=None, vc=None, lens=FAKE, batch=1, max_seq=1024, scale=1.0, w_in=None, w_out=None,
           splits=0, out=FAR, lse=None, ws=FAKE, ws_bytes=1 << 40):
    return L.nsn_q8_attention(C.byref(s), C.byref(q or rows()), n_q, q_lens, C.byref(kc or cache()), C.byref(vc or cache()), lens, batch,
                              max_seq, scale, 0, w_in, w_out, splits, out, lse, ws, ws_bytes, None)


def evict(L, s, w=FAKE, lens=FAKE, batch=1, max_seq=1024, keep=64, first=0, recent=0, kc=None, vc=None, ko=None, vo=None, kept=FAKE,
          new=FAR, w_out=None, ws=FAKE, ws_bytes=1 << 40):
    return L.nsn_q8_evict(C.byref(s), w, lens, batch, max_seq, keep, first, recent, C.byref(kc or cache(codes=FAR, scales=FAR)),
                          C.byref(vc or cache(codes=2 * FAR, scales=2 * FAR)), C.byref(ko or cache(codes=3 * FAR, scales=3 * FAR)),
                          C.byref(vo or cache(codes=4 * FAR, scales=4 * FAR)), kept, new, w_out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,rc", BAD_SHAPES)
def test_bad_shapes_are_refused_everywhere(L, kw, rc):
    s = shape(**kw)
    assert append(L, s) == rc and attend(L, s) == rc and evict(L, s) == rc and L.nsn_last_error()
    for op in (api.NSN_OP_Q8_ATTENTION, api.NSN_OP_Q8_EVICT):
        assert api.nsn_q8_workspace_bytes(s, op, 1, 1, 64) == 0
    assert L.nsn_q8_k_code_offset(C.byref(s), 0, 0) == -1 and L.nsn_q8_v_code_offset(C.byref(s), 0, 0) == -1
    assert L.nsn_q8_append(None, C.byref(rows()), C.byref(rows()), 1, FAKE, FAKE, 1, C.byref(cache()), C.byref(cache()), None) == -1


@pytest.mark.parametrize("kw", [dict(codes=None), dict(scales=None), dict(codes=FAKE + 8), dict(scales=FAKE + 2)])
def test_bad_caches_are_refused(L, kw):
    s = shape()
    for name in ("kc", "vc"):
        for call in (append, attend, evict):
            assert call(L, s, **{name: cache(**kw)}) == -1
    for name in ("ko", "vo"):
        assert evict(L, s, **{name: cache(**kw)}) == -1
    paged = shape(page_size=64, n_pages=3)
    for call in (append, attend, evict):
        assert call(L, paged) == -1 and b"block_table" in L.nsn_last_error()


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=FAKE + 2), dict(b=4), dict(h=129), dict(t=1020)])
def test_rows_that_are_not_aligned_are_refused(L, bad):
    s = shape()
    assert append(L, s, k=rows(**bad)) == -1 and append(L, s, v=rows(**bad)) == -1 and attend(L, s, q=rows(**bad)) == -1
    assert b"rows" in L.nsn_last_error()


def test_other_arguments_are_refused(L):
    s = shape()
    for kw in (dict(start=None), dict(n=None), dict(batch=-1), dict(batch=65536), dict(max_new=-1)):
        assert append(L, s, **kw) == -1, kw
    assert append(L, s, batch=0) == 0 and append(L, s, max_new=0) == 0
    for kw in (dict(lens=None), dict(out=None), dict(out=FAR + 2), dict(batch=-1), dict(batch=65536), dict(n_q=-1), dict(splits=-1),
               dict(max_seq=-1), dict(max_seq=1025), dict(scale=float("nan")), dict(scale=float("inf")), dict(w_in=FAKE),
               dict(n_q=0, w_out=FAKE)):
        assert attend(L, s, **kw) == -1, kw
    assert attend(L, s, batch=0) == 0 and attend(L, s, n_q=0) == 0
    assert attend(L, s, n_q=1 << 23) == api.NSN_ERR_UNSUPPORTED
    need = api.nsn_q8_workspace_bytes(s, api.NSN_OP_Q8_ATTENTION, 1, 1, 1024)   # (that of a call with weights: the most)
    assert need > 0
    for kw in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=FAKE + 8)):
        assert attend(L, s, w_out=FAKE, **kw) == api.NSN_ERR_WORKSPACE, kw
    assert attend(L, s, ws_bytes=1 << 16) == api.NSN_ERR_WORKSPACE
    for kw in (dict(w=None), dict(w=FAKE + 4), dict(lens=None), dict(kept=None), dict(new=None), dict(batch=-1), dict(batch=65536), dict(max_seq=1025),
               dict(max_seq=-1), dict(keep=0), dict(keep=1025), dict(first=-1), dict(recent=-1), dict(first=40, recent=25), dict(w_out=FAKE)):
        assert evict(L, s, **kw) == -1, kw
    assert evict(L, s, batch=0) == 0
    assert api.nsn_q8_workspace_bytes(s, api.NSN_OP_ENCODE, 1, 1, 64) == 0


def test_an_eviction_into_the_cache_that_it_reads_is_refused(L):
    s, far = shape(), 1 << 44
    one = lambda i, d=0: cache(codes=i * far + d, scales=i * far + d)  # noqa: E731
    for a in ("kc", "vc"):
        for b in ("ko", "vo"):
            assert evict(L, s, **{a: one(9), b: one(9)}) == -1, (a, b)
            assert evict(L, s, **{a: one(9), b: one(9, 4096)}) == -1, (a, b)       # overlapping, not the same
            assert evict(L, s, **{a: one(9, 4096), b: one(9)}) == -1, (a, b)
    assert evict(L, s, ko=one(9), vo=one(9)) == -1
    paged = shape(page_size=64, n_pages=8)
    t = lambda i, table: cache(codes=i * far, scales=i * far, block_table=table)  # noqa: E731
    assert evict(L, paged, kc=t(1, FAKE), vc=t(2, FAKE), ko=t(1, FAKE), vo=t(2, 2 * FAKE)) == -1
    assert evict(L, paged, kc=t(1, FAKE), vc=t(2, FAKE), ko=t(1, 2 * FAKE), vo=t(2, FAKE)) == -1


def test_shape_of_the_python_form():
    with pytest.raises(AssertionError):
        api.make_q8_shape(128, 8, 8, 1024, dtype=__import__("torch").float32)


def test_an_append_to_one_cache_as_keys_and_values_is_refused(L):
    s, one = shape(), lambda a, b=0: cache(codes=a * FAR + b, scales=a * FAR + b)
    assert append(L, s, kc=one(1), vc=one(1)) == -1 and b"share" in L.nsn_last_error()
    assert append(L, s, kc=one(1), vc=one(1, 1024)) == -1 and append(L, s, kc=one(1, 1024), vc=one(1)) == -1
    paged = shape(page_size=64, n_pages=64)
    t = lambda table: api.nsn_q8_cache(FAR, 2 * FAR, table)
    assert append(L, paged, kc=t(FAKE), vc=t(FAKE)) == -1 and b"share" in L.nsn_last_error()


def test_outputs_in_the_inputs_are_refused(L):
    s = shape(n_q_heads=8, n_kv_heads=2)   # (rows: head stride 128, token stride 1024; a row is 2 * D bytes)
    end = FAR + (3 * 1024 + 7 * 128 + s.head_dim) * 2
    size = 4 * 8 * s.head_dim * 2
    q = rows(FAR)
    for out in (FAR, end - 16, FAR - size + 16):
        assert attend(L, s, q=q, n_q=4, out=out) == -1 and b"out" in L.nsn_last_error(), out
    back = rows(FAR, t=-1024)               # tokens in falling order
    assert attend(L, s, q=back, n_q=4, out=FAR - 3 * 1024 * 2) == -1 and b"out" in L.nsn_last_error()
    w = 2 * s.max_len * 4
    for w_in in (FAKE, FAKE + 2 * w):
        assert attend(L, s, q=q, out=FAR, w_in=w_in, w_out=FAKE + w, batch=2) == -1 and b"overlap" in L.nsn_last_error(), w_in
    for new in (FAKE, FAKE + 4, FAKE - 4):
        assert evict(L, s, new=new, batch=2) == -1 and b"new_lens" in L.nsn_last_error(), new
    for w_out in (FAKE, FAKE + 64, FAKE - w + 64):
        assert evict(L, s, w_out=w_out) == -1 and b"weights" in L.nsn_last_error(), w_out


def test_a_workspace_serves_fewer_and_shorter_sequences(L):
    rng = np.random.default_rng(3)
    for _ in range(300):
        d, kv, ratio = int(rng.choice([64, 128])), int(rng.choice([1, 2, 8, 12, 32])), int(rng.choice([1, 4, 7]))
        s = api.make_q8_shape(d, kv * ratio, kv, 1 << 20)
        n, batch, length = int(np.exp(rng.uniform(0, 8))), int(np.exp(rng.uniform(0, 5))), int(np.exp(rng.uniform(0, 12)))
        size = lambda b, m: api.nsn_q8_workspace_bytes(s, api.NSN_OP_Q8_ATTENTION, b, n, m)  # noqa: E731
        most = size(batch, length)
        for _ in range(8):
            b, m = int(rng.integers(1, batch + 1)), int(rng.integers(0, length + 1))
            assert 0 < size(b, m) <= most, (d, kv, ratio, n, batch, length, b, m)
