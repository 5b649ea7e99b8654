"""Host-only checks of the 8-bit cache's entry points: what is refused before any HIP call, and the binding's own refusals."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2408_01890_amd import lisa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD, HALF = 0x10000, 0x10004, 0x10002


def desc(**kw):
    a = dict(dtype=lisa.BF16, B=2, H=8, Hkv=4, Lq=1, Lk=100, d_k=64, r=11, F=32, write_scores=1, causal=0)
    a.update(kw)
    return lisa.make_desc(**a)


def cache(**kw):
    a = dict(format=0, n_pages=9, max_pages=2, Hkv=4, width=11, d_k=64, k=FAKE, k_scale=FAKE, v=FAKE, v_scale=FAKE, table=FAKE, lens=FAKE)
    a.update(kw)
    return lisa.Cache8Desc(**a)


def pages(**kw):
    a = dict(n_pages=9, n_seqs=4, max_pages=2, reserved=0, table=FAKE, lens=FAKE, refs=FAKE)
    a.update(kw)
    return lisa.PagesDesc(**a)


def ref(x):
    return None if x is None else C.byref(x)


def append(d, c, k=FAKE, v=FAKE, counts=None):
    return lisa.library().lisa_cache8_append(ref(d), ref(c), k, v, counts, None)


def decode(d, c, q=FAKE, prev=FAKE, w1=FAKE, w2=FAKE, out=FAKE, row=2 * FAKE, ws=FAKE, wsb=1 << 40):
    return lisa.library().lisa_attn_decode8(ref(d), ref(c), q, prev, w1, w2, out, row, ws, wsb, None)


def std(d, c, q=FAKE, row=2 * FAKE, out=FAKE, ws=FAKE, wsb=1 << 40):
    return lisa.library().std_attn_decode8(ref(d), ref(c), q, row, out, ws, wsb, None)


def test_structs_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lisa.h")).read(), flags=re.S)
    for name, cls in (("lisa_cache8", lisa.Cache8Desc), ("lisa_pages", lisa.PagesDesc)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
        assert re.findall(r"(?:int32_t|float|void|const int32_t)\s*\*?\s+(\w+);|\*\s*(\w+);", body) != []
        fields = [re.split(r"[\s*]+", line.strip())[-1] for line in body.split(";") if line.strip()]
        assert fields == [f[0] for f in cls._fields_]


BAD_CACHES = [(None, -1), (dict(v=None), -1), (dict(v_scale=None), -1), (dict(k=None), -1), (dict(k_scale=None), -1), (dict(table=None), -1), (dict(lens=None), -1),
              (dict(format=2), -3), (dict(format=-1), -3), (dict(n_pages=0), -2), (dict(max_pages=0), -2), (dict(Hkv=0), -2), (dict(width=-1), -2), (dict(d_k=0), -2),
              (dict(n_pages=(1 << 20) + 1), -3), (dict(width=257), -3), (dict(d_k=257), -3), (dict(v=0x10008), -4), (dict(k=0x10008), -4), (dict(k_scale=HALF), -4),
              (dict(v_scale=HALF), -4), (dict(table=HALF), -4), (dict(lens=HALF), -4)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(kw, status):
    c = None if kw is None else cache(**kw)
    assert append(desc(), c) == status
    assert decode(desc(), c) == status
    assert std(desc(), c if c is None or kw.get("width") or kw.get("k", 1) is None or kw.get("k_scale", 1) is None else cache(**{"width": 64, **kw})) == status
    if kw is not None and not {"table", "lens"} & set(kw):
        arr = (lisa.Cache8Desc * 1)(c)
        assert lisa.library().lisa_pages_copy(arr, 1, FAKE, 3, None) == status


def test_append_refuses():
    assert append(None, cache()) == -1
    assert append(desc(), cache(), k=None) == -1
    assert append(desc(), cache(), v=None) == -1
    assert append(desc(dtype=1, B=0), cache()) == -2
    assert append(desc(Lq=0), cache()) == -2
    assert append(desc(Hkv=2), cache()) == -2
    assert append(desc(r=12), cache()) == -2
    assert append(desc(d_k=32), cache()) == -2
    assert append(desc(B=65536), cache()) == -3
    assert append(desc(), cache(), k=0x10008) == -4
    assert append(desc(), cache(), v=0x10008) == -4
    assert append(desc(), cache(), counts=HALF) == -4
    d = desc()
    d.dtype = 2
    assert append(d, cache()) == -3


def test_decode_refuses():
    c = cache()
    assert decode(None, c) == -1
    for k in ("q", "prev", "w1", "w2", "out", "row"):
        assert decode(desc(), c, **{k: None}) == -1
        assert decode(desc(), c, **{k: 0x10008}) == -4
    assert decode(desc(Lq=2), c) == -2
    assert decode(desc(H=6), c) == -2
    assert decode(desc(Lk=129), c) == -2                     # two pages hold 128 tokens
    assert decode(desc(Lk=0), c) == -2
    assert decode(desc(r=12), c) == -2
    assert decode(desc(d_k=128), c) == -2
    assert decode(desc(Hkv=8), c) == -2
    assert decode(desc(F=0), c) == -2
    assert decode(desc(F=640), c) == -3
    assert decode(desc(mix=9), c) == -3
    assert decode(desc(score_tiled=1), c) == -3
    assert decode(desc(), c, row=FAKE) == -2                 # the row that it shares
    assert decode(desc(), c, ws=None) == -5
    need = lisa.workspace_bytes(desc(), lisa.WS_DECODE8)
    assert need > 0 and decode(desc(), c, wsb=need - 1) == -5
    assert lisa.workspace_bytes(desc(Lq=2), lisa.WS_DECODE8) == 0


def test_std_refuses():
    c, d = cache(width=64), desc(r=0, F=0)
    assert std(None, c) == -1
    assert std(d, c, q=None) == -1
    assert std(d, c, out=None) == -1
    assert std(d, c, q=0x10008) == -4
    assert std(d, c, row=0x10008) == -4
    assert std(d, cache()) == -2                             # K_LR where K is needed
    assert std(desc(r=0, F=0, Lk=129), c) == -2
    assert std(desc(r=0, F=0, score_tiled=1), c) == -3
    assert std(d, c, ws=None) == -5
    assert std(d, c, wsb=lisa.workspace_bytes(d, lisa.WS_STD_DECODE8) - 1) == -5


BAD_PAGES = [(None, -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(refs=None), -1), (dict(n_pages=0), -2), (dict(n_seqs=0), -2), (dict(max_pages=0), -2),
             (dict(reserved=1), -2), (dict(n_pages=(1 << 20) + 1), -3), (dict(n_seqs=1 << 20, max_pages=1 << 12), -3), (dict(table=HALF), -4), (dict(lens=HALF), -4),
             (dict(refs=HALF), -4)]


@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_bad_page_states_are_refused(kw, status):
    p, lib = None if kw is None else pages(**kw), lisa.library()
    assert lib.lisa_pages_workspace_bytes(ref(p)) == 0
    assert lib.lisa_pages_grow(ref(p), FAKE, FAKE, FAKE, 1 << 30, None) == status
    assert lib.lisa_pages_fork(ref(p), FAKE, FAKE, 1, FAKE, FAKE, FAKE, 1 << 30, None) == status
    assert lib.lisa_pages_free(ref(p), FAKE, 1, FAKE, FAKE, 1 << 30, None) == status
    assert lib.lisa_pages_compact(ref(p), FAKE, FAKE, 1 << 30, None) == status


def test_page_calls_refuse():
    lib, p = lisa.library(), pages()
    need = lib.lisa_pages_workspace_bytes(ref(p))
    assert need >= 4 * 2 * (9 + 4)
    grow = lambda add=FAKE, done=FAKE, ws=FAKE, wsb=need: lib.lisa_pages_grow(ref(p), add, done, ws, wsb, None)  # noqa: E731
    assert [grow(add=None), grow(done=None), grow(add=HALF), grow(done=HALF), grow(ws=None), grow(wsb=need - 1), grow(ws=0x10008)] == [-1, -1, -4, -4, -5, -5, -4]
    fork = lambda src=FAKE, dst=FAKE, n=2, done=FAKE, copies=FAKE, wsb=need: lib.lisa_pages_fork(ref(p), src, dst, n, done, copies, FAKE, wsb, None)  # noqa: E731
    assert [fork(src=None), fork(dst=None), fork(done=None), fork(copies=None), fork(n=0), fork(n=5), fork(copies=ODD), fork(wsb=0)] == [-1, -1, -1, -1, -2, -2, -4, -5]
    free = lambda seqs=FAKE, n=2, done=FAKE, wsb=need: lib.lisa_pages_free(ref(p), seqs, n, done, FAKE, wsb, None)  # noqa: E731
    assert [free(seqs=None), free(done=None), free(n=0), free(n=5), free(seqs=HALF), free(wsb=need - 1)] == [-1, -1, -2, -2, -4, -5]
    compact = lambda copies=FAKE, wsb=need: lib.lisa_pages_compact(ref(p), copies, FAKE, wsb, None)  # noqa: E731
    assert [compact(copies=None), compact(copies=ODD), compact(wsb=need - 1)] == [-1, -4, -5]
    arr = (lisa.Cache8Desc * 2)(cache(), cache(n_pages=8))
    copy = lambda a=arr, n=2, copies=FAKE, m=1: lib.lisa_pages_copy(a, n, copies, m, None)  # noqa: E731
    assert [copy(a=None), copy(copies=None), copy(n=0), copy(m=0), copy(), copy(n=1, copies=ODD)] == [-1, -1, -2, -2, -2, -4]


def test_the_binding_refuses_host_tensors():
    z = torch.zeros
    with pytest.raises(ValueError):
        lisa.Pages(z((2, 3), dtype=torch.int32), z(2, dtype=torch.int32), z(5, dtype=torch.int32))
