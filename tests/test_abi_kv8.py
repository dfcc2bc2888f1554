"""Host-side checks of the 8-bit cache's calls and of attention over shared
prefixes, without a GPU: every call below stops at a check, before the first
CUDA call."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module", params=["release", "debug"])
def lib(request):
    from paper_2609_27233_gb300 import build, _lib
    path = _lib.LIB_PATH if request.param == "release" else _lib.DEBUG_LIB_PATH
    if not os.path.exists(path):
        build.build(variants=(request.param,))
    return _lib.load(path)


null = ctypes.c_void_p(0)
fake = ctypes.c_void_p(1 << 20)      # never dereferenced
odd = ctypes.c_void_p((1 << 20) + 4)


def pool(values=4096, scales=8192, layers=2, pages=4, heads=2, page=16, D=128):
    from paper_2609_27233_gb300._lib import PagedKV8C
    return ctypes.byref(PagedKV8C(values, scales, layers, pages, heads, page, D))


def refuses_the_pool(call):
    assert call(kv=pool(values=0)) == 1 and call(kv=pool(scales=0)) == 1
    assert call(kv=pool(values=4096 + 8)) == 1 and call(kv=pool(scales=4096 + 8)) == 1
    assert call(kv=pool(layers=0)) == 1 and call(kv=pool(pages=0)) == 1 and call(kv=pool(heads=0)) == 1
    assert call(kv=pool(page=8)) == 2 and call(kv=pool(D=96)) == 2 and call(kv=pool(heads=65)) == 2


@pytest.mark.parametrize("name", ["umim_kv8_write", "umim_kv8_read"])
def test_rows(lib, name):
    def call(kv=None, layer=0, bt=fake, cols=4, start=fake, cu=fake, B=3, k=fake, v=fake, stride=0, T=40):
        return getattr(lib, name)(kv or pool(), layer, bt, cols, start, cu, B, k, v, stride, T, null, null)
    refuses_the_pool(call)
    assert call(layer=2) == 1 and call(layer=-1) == 1
    assert call(B=-1) == 1 and call(cols=-1) == 1 and call(T=-1) == 1 and call(stride=-8) == 1
    assert call(cu=null) == 1                    # one row a sequence, but not as many rows
    assert call(stride=248) == 1                 # rows overlap
    assert call(stride=260) == 1                 # not a multiple of 8
    assert call(T=(1 << 24) + 1) == 2
    assert call(B=1 << 16, cols=1 << 12) == 2
    assert call(bt=null) == 1 and call(start=null) == 1 and call(k=null) == 1 and call(v=null) == 1
    assert call(k=odd) == 1 and call(v=odd) == 1
    assert call(B=0) == 0 and call(T=0) == 0 and call(B=0, T=0, cu=null) == 0


def test_append_merge(lib):
    def call(kv=None, bt=fake, cols=4, lens=fake, B=3, nk=fake, nv=fake, mk=null, row=null, n=0, sk=null, sv=null):
        return lib.umim_kv8_append_merge(kv or pool(), bt, cols, lens, B, nk, nv, null, mk, row, n, sk, sv, null, null,
                                         null)
    refuses_the_pool(call)
    assert call(B=-1) == 1 and call(cols=-1) == 1 and call(n=-1) == 1
    assert call(B=1 << 16, cols=1 << 12) == 2
    assert call(bt=null) == 1 and call(lens=null) == 1 and call(nk=null) == 1 and call(nv=odd) == 1
    assert call(mk=fake, n=2) == 1               # merges without surrogates
    assert call(mk=fake, n=2, row=fake, sk=odd, sv=fake) == 1
    assert call(B=0) == 0


def test_attention(lib):
    def call(kv=None, q=fake, Hq=8, layer=0, bt=fake, cols=4, lens=fake, B=3, out=fake, ws=null, size=1 << 30):
        return lib.umim_decode_attention_kv8(q, Hq, kv or pool(), layer, bt, cols, lens, B, 0.0, out, ws, size, null,
                                             null)
    size = lib.umim_decode_attention_kv8_workspace_size
    assert size(16, 32, 8, 128) > 0 and size(16, 32, 8, 96) == 0 and size(-1, 32, 8, 128) == 0 and size(1, 0, 8, 64) == 0
    refuses_the_pool(call)
    assert call(Hq=0) == 1 and call(Hq=7) == 2 and call(Hq=34) == 2
    assert call(layer=2) == 1 and call(B=-1) == 1 and call(cols=-1) == 1
    assert call(B=1 << 24) == 2 and call(B=1 << 20, cols=1 << 10) == 2
    assert call(q=null) == 1 and call(q=odd) == 1 and call(out=null) == 1 and call(bt=null) == 1 and call(lens=null) == 1
    assert call() == 5 and call(ws=ctypes.c_void_p((1 << 20) + 16)) == 5 and call(ws=fake, size=4096) == 5
    assert call(B=0) == 0


@pytest.mark.parametrize("bits", [16, 8])
def test_shared_attention(lib, bits):
    from paper_2609_27233_gb300._lib import PagedKVC
    name = "umim_decode_attention_shared" + ("_kv8" if bits == 8 else "")

    def call(kv=None, q=fake, Hq=8, layer=0, pt=fake, pcols=4, pl=fake, po=fake, n=2, bt=fake, cols=4, lens=fake, B=3,
             out=fake, ws=null, size=1 << 30):
        kv = kv or (pool() if bits == 8 else ctypes.byref(PagedKVC(4096, 2, 4, 2, 16, 128)))
        return getattr(lib, name)(q, Hq, kv, layer, pt, pcols, pl, po, n, bt, cols, lens, B, 0.0, out, ws, size, null,
                                  null)
    size = lib.umim_decode_attention_shared_workspace_size
    assert size(16, 1, 32, 8, 128) > 0 and size(16, 0, 32, 8, 128) == 0 and size(16, 1, 32, 8, 80) == 0
    assert size(4096, 512, 1024, 64, 128) > 4096 * 64 * 16 * 128 * 4
    if bits == 8:
        refuses_the_pool(call)
    else:
        assert call(kv=ctypes.byref(PagedKVC(0, 2, 4, 2, 16, 128))) == 1
        assert call(kv=ctypes.byref(PagedKVC(4096, 2, 4, 2, 16, 96))) == 2
    assert call(Hq=0) == 1 and call(Hq=7) == 2 and call(Hq=34) == 2
    assert call(layer=2) == 1 and call(B=-1) == 1 and call(cols=-1) == 1 and call(pcols=-1) == 1
    assert call(n=0) == 1 and call(n=513) == 2 and call(B=4097) == 2
    assert call(po=null) == 1                    # whose sequences are whose?
    assert call(B=4096, cols=1 << 18) == 2 and call(pcols=1 << 30) == 2
    assert call(q=null) == 1 and call(q=odd) == 1 and call(out=null) == 1 and call(bt=null) == 1 and call(lens=null) == 1
    assert call(pt=null) == 1 and call(pl=null) == 1
    assert call() == 5 and call(ws=ctypes.c_void_p((1 << 20) + 16)) == 5 and call(ws=fake, size=4096) == 5
    assert call(n=1, po=null) == 5               # one prefix for all: as far as the workspace
    assert call(B=0) == 0


def test_binding_refuses_tensors_of_other_kinds():
    import paper_2609_27233_gb300 as umim
    values = torch.zeros((1, 2, 2, 1, 16, 64), dtype=torch.uint8)
    scales = torch.zeros((1, 2, 2, 1, 16), dtype=torch.uint8)
    v8, s8 = values.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)
    for v, s in ((values, s8), (v8, scales), (v8[0], s8), (v8, s8[:, :1]), (v8[:, :, :1], s8), (v8, s8)):
        with pytest.raises(ValueError):          # (the last: not on a GPU)
            umim.Kv8Pool(v, s)
