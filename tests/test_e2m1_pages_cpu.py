"""Host side of the 4-bit cache, several axes and the pages without a GPU: argument checks, all made before any launch."""
import ctypes
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2608_09160_b200 import attn, binding, pages
from tests.test_abi import ROOT, declared_functions

A, B, C, D, E, F, G, H = (0x10000000 + i * 0x4000000 for i in range(8))
CPU = not torch.cuda.is_available()
LEGAL = binding.QKNORM_ERR_CUDA              # a legal call without a GPU gets as far as asking CUDA for the device


@pytest.fixture(scope="module")
def lib(libqknorm):
    pages.lib()
    return attn.lib()


def test_header_and_binding_agree_on_exports(lib):
    assert declared_functions(os.path.join(ROOT, "include", "qknorm_pages.h")) == sorted(pages.EXPORTS)
    for name in pages.EXPORTS:
        assert hasattr(lib, name), name


# ---- several axes -------------------------------------------------------------------------------------------------------

def axes(positions=G, ld=0, inv_freq=G + 0x100000, axis=G + 0x200000, n=3, rot_dim=64, interleaved=0, mscale=1.0):
    return attn.CRotationAxes(positions, ld, inv_freq, axis, n, rot_dim, interleaved, mscale)


def test_axes_argument_errors(lib):
    b = binding

    def rope(rot, fn="qknorm_rope_axes", oq=C):
        return getattr(lib, fn)(A, B, ctypes.byref(rot) if rot else None, 4, 256, 128, 64, 0, 0, 0, oq, D, 0, 0, None)

    for fn in ("qknorm_rope_axes", "qknorm_rope_axes_e4m3"):
        assert rope(None, fn) == b.QKNORM_ERR_NULL
        assert rope(axes(n=0), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(n=9), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(ld=3), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(ld=-1), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(rot_dim=63), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(rot_dim=66), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(mscale=math.nan), fn) == b.QKNORM_ERR_SHAPE
        assert rope(axes(positions=None), fn) == b.QKNORM_ERR_NULL
        assert rope(axes(positions=G + 4), fn) == b.QKNORM_ERR_ALIGN
        assert rope(axes(), fn, oq=G + 0x200000) == b.QKNORM_ERR_ALIAS           # on top of axis
        assert rope(axes(ld=1 << 20), fn, oq=G + (1 << 23)) == b.QKNORM_ERR_ALIAS  # on top of the second axis' positions
        if CPU:
            assert rope(axes(axis=None), fn) == LEGAL
            assert rope(axes(), fn) == LEGAL


# ---- the 4-bit cache ----------------------------------------------------------------------------------------------------

def cache(pages_=8, page=16, heads=2, hd=64, k=E, v=F, ks=E + 0x1000000, vs=F + 0x1000000, k_scale=1.0, v_scale=1.0, **kw):
    code, sc = hd // 2, hd // 16
    c = attn.CPagedCacheE2m1(k, v, ks, vs, heads * page * code, code, page * code, heads * page * code, code, page * code,
                             heads * page * sc, sc, page * sc, heads * page * sc, sc, page * sc, pages_, page, heads, hd, k_scale, v_scale)
    for n, x in kw.items():
        setattr(c, n, x)
    return c


BAD_CACHES = [
    (dict(pages_=-1), "SHAPE"), (dict(page=0), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(hd=0), "HEADS"), (dict(hd=24), "HEADS"),
    (dict(hd=272), "HEADS"), (dict(k=None), "NULL"), (dict(vs=None), "NULL"), (dict(k=E + 4), "ALIGN"), (dict(v_token=36), "SHAPE"), (dict(v_page=1028), "ALIGN"),
    (dict(ks=E + 0x1000002), "ALIGN"), (dict(k_scale=0.0), "SHAPE"), (dict(v_scale=math.inf), "SHAPE"), (dict(k_scale=math.nan), "SHAPE"),
    (dict(k_token=16), "SHAPE"), (dict(ks_head=2), "SHAPE"), (dict(k_page=8), "SHAPE"), (dict(v_head=-32), "SHAPE"),
]


def append(lib, c, rot=None, T=4, dq=256, q=A, k=B, v=C, gq=G, gk=G + 0x10000, norm=1, eps=1e-6, slots=H, oq=D, ldk=0):
    return lib.qknorm_fwd_append_e2m1(q, k, v, gq, gk, norm, eps, ctypes.byref(rot) if rot else None, slots, ctypes.byref(c) if c else None, T, dq, 0,
                                      ldk, 0, oq, 0, None)


def attend(lib, c, q=A, table=G, cols=4, ld=0, lens=G + 0x10000, starts=G + 0x20000, seqs=2, T=2, max_q=1, max_kv=64, hq=4, scale=0.125, causal=1,
           window=0, out=D, lse=None, ws=None, wsb=0):
    return lib.qknorm_attn_paged_e2m1(q, 0, ctypes.byref(c) if c else None, table, cols, ld, lens, starts, seqs, T, max_q, max_kv, hq, scale, causal,
                                      window, out, 0, lse, ws, wsb, None)


@pytest.mark.parametrize("bad,error", BAD_CACHES)
def test_caches_that_are_refused(lib, bad, error):
    want = getattr(binding, "QKNORM_ERR_" + error)
    assert append(lib, cache(**bad)) == want
    assert attend(lib, cache(**bad)) == want


def test_append_argument_errors(lib):
    b = binding
    assert append(lib, None) == b.QKNORM_ERR_NULL
    assert append(lib, cache(), T=0) == b.QKNORM_OK
    assert append(lib, cache(), T=-1) == b.QKNORM_ERR_SHAPE
    assert append(lib, cache(), dq=100) == b.QKNORM_ERR_HEADS
    assert append(lib, cache(), norm=3) == b.QKNORM_ERR_SHAPE
    assert append(lib, cache(), eps=-1.0) == b.QKNORM_ERR_EPS
    assert append(lib, cache(), k=None) == b.QKNORM_ERR_NULL
    assert append(lib, cache(), slots=None) == b.QKNORM_ERR_NULL
    assert append(lib, cache(), gk=None) == b.QKNORM_ERR_NULL
    assert append(lib, cache(), slots=H + 4) == b.QKNORM_ERR_ALIGN
    assert append(lib, cache(), ldk=100) == b.QKNORM_ERR_SHAPE
    assert append(lib, cache(k_scale=1e-39)) == b.QKNORM_ERR_SHAPE               # no finite reciprocal
    assert append(lib, cache(), rot=axes(rot_dim=128)) == b.QKNORM_ERR_SHAPE
    assert append(lib, cache(), oq=E) == b.QKNORM_ERR_ALIAS                      # the output in the cache
    assert append(lib, cache(), oq=F + 0x1000000) == b.QKNORM_ERR_ALIAS          # and in its scales
    assert append(lib, cache(v=E)) == b.QKNORM_ERR_ALIAS                         # K on V
    assert append(lib, cache(vs=E + 0x1000000)) == b.QKNORM_ERR_ALIAS            # scales on scales
    assert append(lib, cache(ks=E + 64)) == b.QKNORM_ERR_ALIAS                   # scales in the codes
    if CPU:
        assert append(lib, cache()) == LEGAL
        assert append(lib, cache(), rot=axes()) == LEGAL
        assert append(lib, cache(), oq=A, dq=0, q=None, gq=None) == LEGAL
        # codes and scales of a page beside one another in one buffer
        page = 2 * 16 * 32 + 2 * 16 * 4
        assert append(lib, cache(ks=E + 2 * 16 * 32, k_page=page, ks_page=page)) == LEGAL


def test_attention_argument_errors(lib):
    b = binding
    assert attend(lib, None) == b.QKNORM_ERR_NULL
    assert attend(lib, cache(), seqs=0) == b.QKNORM_OK
    assert attend(lib, cache(), T=0) == b.QKNORM_OK
    assert attend(lib, cache(), seqs=-1) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(), max_kv=0x7fffffff) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(), hq=3) == b.QKNORM_ERR_HEADS
    assert attend(lib, cache(), scale=0.0) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(k_scale=1e38), scale=1e10) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(), causal=2) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(), window=-1) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(), ld=3) == b.QKNORM_ERR_SHAPE
    assert attend(lib, cache(), q=None) == b.QKNORM_ERR_NULL
    assert attend(lib, cache(), table=None) == b.QKNORM_ERR_NULL
    assert attend(lib, cache(), q=A + 1) == b.QKNORM_ERR_ALIGN
    assert attend(lib, cache(), lens=G + 0x10002) == b.QKNORM_ERR_ALIGN
    n = ctypes.c_int64(-1)
    ws = lambda *a: lib.qknorm_attn_paged_e2m1_workspace(*a, ctypes.byref(n))
    assert ws(2, 2, 1, 64, 4, 2, 24, 0) == b.QKNORM_ERR_HEADS
    assert ws(2, 2, 1, 64, 4, 2, 512, 0) == b.QKNORM_ERR_HEADS
    assert ws(2, 2, 1, 64, 4, 3, 64, 0) == b.QKNORM_ERR_HEADS
    assert ws(0, 2, 1, 64, 4, 2, 64, 0) == b.QKNORM_OK and n.value == 0
    assert lib.qknorm_attn_paged_e2m1_workspace(2, 2, 1, 64, 4, 2, 64, 0, None) == b.QKNORM_ERR_NULL
    if CPU:
        assert attend(lib, cache()) == LEGAL


# ---- pages --------------------------------------------------------------------------------------------------------------

def pool(base=A, page=4096, c0=1, c1=1, s0=0, s1=0, n=4096):
    return pages.CPagePool(base, page, (ctypes.c_int64 * 2)(c0, c1), (ctypes.c_int64 * 2)(s0, s1), n)


def array(*pools_):
    return (pages.CPagePool * len(pools_))(*pools_)


BAD_POOLS = [
    (dict(base=None), "NULL"), (dict(page=-1), "SHAPE"), (dict(c0=0), "SHAPE"), (dict(n=0), "SHAPE"), (dict(s0=-8, c0=2), "SHAPE"), (dict(n=4097), "SHAPE"),
    (dict(c1=2, s1=2048), "SHAPE"), (dict(c0=2, s0=0), "SHAPE"), (dict(page=1 << 58, n=8), "SHAPE"),
]


@pytest.mark.parametrize("bad,error", BAD_POOLS)
def test_pools_that_are_refused(lib, bad, error):
    want = getattr(binding, "QKNORM_ERR_" + error)
    assert lib.qknorm_pages_copy(array(pool(**bad)), 1, 100, G, H, 3, None) == want
    assert fork(lib, pools=array(pool(**bad))) == want
    assert compact(lib, pools=array(pool(**bad))) == want


def fork(lib, pools=None, k=1, N=100, refs=B, table=C, cols=8, ld=0, lens=D, rows=4, page=16, parents=E, children=F, n=2, ok=None, ws=G, wsb=1 << 20):
    return lib.qknorm_pages_fork(array(pool()) if pools is None else pools, k, N, refs, table, cols, ld, lens, rows, page, parents, children, n, ok, ws,
                                 wsb, None)


def free(lib, refs=B, N=100, table=C, cols=8, ld=0, lens=D, rows=4, page=16, list_=E, n=2):
    return lib.qknorm_pages_free(refs, N, table, cols, ld, lens, rows, page, list_, n, None)


def compact(lib, pools=None, k=1, N=100, refs=B, table=C, cols=8, ld=0, lens=D, rows=4, page=16, live=E, ws=G, wsb=1 << 20):
    return lib.qknorm_pages_compact(array(pool()) if pools is None else pools, k, N, refs, table, cols, ld, lens, rows, page, live, ws, wsb, None)


def test_pages_argument_errors(lib):
    b = binding
    copy = lambda src=G, dst=H, n=3, k=1, N=100: lib.qknorm_pages_copy(array(pool()), k, N, src, dst, n, None)
    assert copy(n=0) == b.QKNORM_OK and copy(k=0) == b.QKNORM_OK
    assert copy(n=-1) == b.QKNORM_ERR_SHAPE and copy(N=0) == b.QKNORM_ERR_SHAPE and copy(k=-1) == b.QKNORM_ERR_SHAPE
    assert copy(src=None) == b.QKNORM_ERR_NULL and copy(dst=H + 2) == b.QKNORM_ERR_ALIGN
    assert copy(src=A + 4096 * 99) == b.QKNORM_ERR_ALIAS                         # the list inside the last page
    assert lib.qknorm_pages_copy(None, 1, 100, G, H, 3, None) == b.QKNORM_ERR_NULL
    assert lib.qknorm_pages_copy(array(pool()), 1025, 100, G, H, 3, None) == b.QKNORM_ERR_SHAPE
    for fn in (fork, free, compact):
        assert fn(lib, refs=None) == b.QKNORM_ERR_NULL
        assert fn(lib, table=None) == b.QKNORM_ERR_NULL
        assert fn(lib, lens=None) == b.QKNORM_ERR_NULL
        assert fn(lib, refs=B + 2) == b.QKNORM_ERR_ALIGN
        assert fn(lib, page=0) == b.QKNORM_ERR_SHAPE
        assert fn(lib, ld=7) == b.QKNORM_ERR_SHAPE
        assert fn(lib, cols=-1) == b.QKNORM_ERR_SHAPE
        assert fn(lib, rows=-1) == b.QKNORM_ERR_SHAPE
        assert fn(lib, N=1 << 31) == b.QKNORM_ERR_SHAPE
        assert fn(lib, lens=C + 16) == b.QKNORM_ERR_ALIAS                        # inside the table: one of the two is written
        assert fn(lib, refs=D) == b.QKNORM_ERR_ALIAS
        if CPU:
            assert fn(lib) == LEGAL
    assert fork(lib, n=0) == b.QKNORM_OK and free(lib, n=0) == b.QKNORM_OK
    assert fork(lib, n=-1) == b.QKNORM_ERR_SHAPE and free(lib, n=-1) == b.QKNORM_ERR_SHAPE
    assert fork(lib, parents=None) == b.QKNORM_ERR_NULL and free(lib, list_=None) == b.QKNORM_ERR_NULL and compact(lib, live=None) == b.QKNORM_ERR_NULL
    assert fork(lib, ok=F) == b.QKNORM_ERR_ALIAS and fork(lib, table=A + 64) == b.QKNORM_ERR_ALIAS and compact(lib, live=A) == b.QKNORM_ERR_ALIAS
    for fn in (fork, compact):
        assert fn(lib, ws=None) == b.QKNORM_ERR_SCRATCH
        assert fn(lib, wsb=16) == b.QKNORM_ERR_SCRATCH
        assert fn(lib, ws=G + 4) == b.QKNORM_ERR_SCRATCH
        assert fn(lib, ws=C) == b.QKNORM_ERR_SCRATCH                             # on the table
        assert fn(lib, ws=A) == b.QKNORM_ERR_SCRATCH                             # on the pages
    if CPU:
        assert fork(lib, parents=E, children=E + 4) == LEGAL                     # lists that are only read may overlap
        assert fork(lib, parents=E, children=E) == LEGAL
    n = ctypes.c_int64(0)
    assert lib.qknorm_pages_workspace(100, 4, 2, None) == b.QKNORM_ERR_NULL
    assert lib.qknorm_pages_workspace(0, 4, 2, ctypes.byref(n)) == b.QKNORM_ERR_SHAPE
    assert lib.qknorm_pages_workspace(100, 4, 2, ctypes.byref(n)) == b.QKNORM_OK and n.value > 0 and n.value % 16 == 0


def test_how_a_page_lies():
    """What the binding makes of a tensor's shape and strides."""
    f = lambda t, d: pages._pieces(tuple(t.shape), t.stride(), t.element_size(), d)
    t = torch.zeros((3, 2, 24, 4, 2, 16), dtype=torch.bfloat16)
    assert f(t, 2) == (256, 1, 6, 0, 24 * 256, 256)                              # layers and K, V are one axis
    assert f(t[:, 0], 1) == (256, 1, 3, 0, 2 * 24 * 256, 256)
    assert f(t[..., :8], 2) == (256, 6, 8, 24 * 256, 32, 16)
    assert f(t[:, :, :, :, 0, :8], 2) == (256, 6, 4, 24 * 256, 64, 16)
    assert f(t[:2, 0, :, :, :, :8], 1) == (256, 2, 8, 2 * 24 * 256, 32, 16)
    assert f(t.permute(2, 0, 1, 5, 4, 3), 0) == (256, 1, 6, 0, 24 * 256, 256)    # whatever the order of its axes
    assert f(t[:, :1, :, ::2, :, :8], 2) is None                                 # three axes of pieces
    assert f(torch.zeros((5, 7), dtype=torch.uint8), 0) == (7, 1, 1, 0, 0, 7)
    assert f(torch.zeros((5, 1, 1)), 0) == (4, 1, 1, 0, 0, 4)


def test_a_torch_without_a_4_bit_type_will_do():
    """Everything but tensors of that type works there: bf16 and FP8 calls need no more than before."""
    code = ("import torch\n"
            "del torch.float4_e2m1fn_x2\n"
            "from paper_2608_09160_b200 import attn, pages\n"
            "assert attn._F4 is None\n")
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)
