"""Host side of include/qknorm_attn.h without a GPU: exports, argument checks (all made before any launch), the frequency helper."""
import ctypes
import math
import os

import pytest

from paper_2608_09160_b200 import attn, binding
from tests.test_abi import ROOT, declared_functions

HEADER_ATTN = os.path.join(ROOT, "include", "qknorm_attn.h")
A, B, C, D, E, F, G, H = (0x10000000 + i * 0x4000000 for i in range(8))


@pytest.fixture(scope="module")
def lib(libqknorm):
    return attn.lib()


def test_header_and_binding_agree_on_exports(lib):
    assert declared_functions(HEADER_ATTN) == sorted(attn.EXPORTS)
    for name in attn.EXPORTS:
        assert hasattr(lib, name), name


def rotation(rot_dim=64, positions=G, inv_freq=G + 0x100000, interleaved=0, mscale=1.0):
    return attn.CRotation(positions, inv_freq, rot_dim, interleaved, mscale)


def rope(lib, q=A, k=B, rot=None, T=4, dq=256, dk=128, hd=64, ldq=0, ldk=0, inverse=0, oq=C, ok=D, ldoq=0, ldok=0, fn="qknorm_rope"):
    r = rotation() if rot is None else rot
    return getattr(lib, fn)(q, k, ctypes.byref(r) if r else None, T, dq, dk, hd, ldq, ldk, inverse, oq, ok, ldoq, ldok, None)


def test_rope_argument_errors(lib):
    b = binding
    assert rope(lib, T=0) == b.QKNORM_OK
    assert rope(lib, T=-1) == b.QKNORM_ERR_SHAPE
    assert rope(lib, dq=-64) == b.QKNORM_ERR_SHAPE
    assert rope(lib, dq=0, dk=0) == b.QKNORM_ERR_SHAPE
    assert rope(lib, dq=65536 + 64) == b.QKNORM_ERR_SHAPE
    assert rope(lib, hd=0) == b.QKNORM_ERR_HEADS
    assert rope(lib, hd=96) == b.QKNORM_ERR_HEADS
    assert rope(lib, hd=1024, dq=1024, dk=1024) == b.QKNORM_ERR_HEADS
    assert rope(lib, rot=False) == b.QKNORM_ERR_NULL
    assert rope(lib, rot=rotation(rot_dim=63)) == b.QKNORM_ERR_SHAPE
    assert rope(lib, rot=rotation(rot_dim=66)) == b.QKNORM_ERR_SHAPE
    assert rope(lib, rot=rotation(rot_dim=-2)) == b.QKNORM_ERR_SHAPE
    assert rope(lib, rot=rotation(interleaved=2)) == b.QKNORM_ERR_SHAPE
    assert rope(lib, rot=rotation(mscale=math.inf)) == b.QKNORM_ERR_SHAPE
    assert rope(lib, rot=rotation(positions=None)) == b.QKNORM_ERR_NULL
    assert rope(lib, rot=rotation(inv_freq=None)) == b.QKNORM_ERR_NULL
    assert rope(lib, rot=rotation(positions=G + 4)) == b.QKNORM_ERR_ALIGN
    assert rope(lib, inverse=2) == b.QKNORM_ERR_SHAPE
    assert rope(lib, q=None) == b.QKNORM_ERR_NULL
    assert rope(lib, ok=None) == b.QKNORM_ERR_NULL
    assert rope(lib, q=A + 1) == b.QKNORM_ERR_ALIGN
    assert rope(lib, ldq=255) == b.QKNORM_ERR_SHAPE
    assert rope(lib, ldok=-1) == b.QKNORM_ERR_SHAPE
    assert rope(lib, oq=A + 64) == b.QKNORM_ERR_ALIAS
    assert rope(lib, oq=B) == b.QKNORM_ERR_ALIAS
    assert rope(lib, oq=C, ok=C + 64) == b.QKNORM_ERR_ALIAS
    assert rope(lib, oq=G) == b.QKNORM_ERR_ALIAS                 # on top of the positions
    assert rope(lib, oq=A, ldoq=512) == b.QKNORM_ERR_ALIAS       # same base, another pitch
    assert rope(lib, fn="qknorm_rope_e4m3", T=0) == b.QKNORM_OK
    import torch
    if not torch.cuda.is_available():                            # legal: gets as far as asking CUDA for the device
        assert rope(lib, oq=A, ok=B) == b.QKNORM_ERR_CUDA
        assert rope(lib, q=A, k=A + 512, ldq=512, ldk=512, oq=A, ok=A + 512, ldoq=512, ldok=512, fn="qknorm_rope") == b.QKNORM_ERR_CUDA
        assert rope(lib, q=A + 1, k=B, oq=A + 1, ok=B, fn="qknorm_rope_e4m3") == b.QKNORM_ERR_CUDA


def cache(k=E, v=F, pages=8, page=16, heads=2, hd=64, e4m3=0, ks=1.0, vs=1.0, **kw):
    c = attn.CPagedCache(k, v, page * heads * hd, heads * hd, hd, page * heads * hd, heads * hd, hd, pages, page, heads, hd, e4m3, ks, vs)
    for n, x in kw.items():
        setattr(c, n, x)
    return c


BAD_CACHES = [
    (dict(pages=-1), "SHAPE"), (dict(page=0), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(hd=0), "HEADS"), (dict(hd=1024), "HEADS"),
    (dict(e4m3=2), "SHAPE"), (dict(e4m3=1, ks=0.0), "SHAPE"), (dict(e4m3=1, vs=math.nan), "SHAPE"), (dict(k=None), "NULL"),
    (dict(k=E + 1), "ALIGN"), (dict(k_token=-1), "SHAPE"),
    (dict(k_head=32), "SHAPE"),                       # heads overlap
    (dict(v_token=64), "SHAPE"),                      # tokens overlap heads
    (dict(k_page=8), "SHAPE"),                        # pages overlap
    (dict(k_page=1 << 60), "SHAPE"),                  # beyond any memory
]


def append(lib, c=None, q=A, k=B, v=B + 0x1000000, gq=C, gk=C + 0x100000, norm=1, eps=1e-6, rot=None, slots=H, T=4, dq=256, ldq=0, ldk=0,
           ldv=0, oq=D, ldo=0):
    c = cache() if c is None else c
    return lib.qknorm_fwd_append(q, k, v, gq, gk, norm, eps, ctypes.byref(rot) if rot else None, slots, ctypes.byref(c) if c else None, T,
                                 dq, ldq, ldk, ldv, oq, ldo, None)


def test_append_argument_errors(lib):
    b = binding
    assert append(lib, T=0) == b.QKNORM_OK
    assert append(lib, c=False) == b.QKNORM_ERR_NULL
    for kw, name in BAD_CACHES:
        assert append(lib, c=cache(**kw)) == getattr(b, "QKNORM_ERR_" + name), kw
    assert append(lib, T=-1) == b.QKNORM_ERR_SHAPE
    assert append(lib, dq=200) == b.QKNORM_ERR_HEADS
    assert append(lib, norm=3) == b.QKNORM_ERR_SHAPE
    assert append(lib, eps=-1.0) == b.QKNORM_ERR_EPS
    assert append(lib, eps=math.nan) == b.QKNORM_ERR_EPS
    assert append(lib, rot=rotation(rot_dim=66)) == b.QKNORM_ERR_SHAPE
    for n in ("q", "k", "v", "gq", "gk", "slots", "oq"):
        assert append(lib, **{n: None}) == b.QKNORM_ERR_NULL, n
    assert append(lib, slots=H + 4) == b.QKNORM_ERR_ALIGN
    assert append(lib, gk=C + 1) == b.QKNORM_ERR_ALIGN
    assert append(lib, ldk=100) == b.QKNORM_ERR_SHAPE
    assert append(lib, oq=A + 128) == b.QKNORM_ERR_ALIAS
    assert append(lib, oq=E + 64) == b.QKNORM_ERR_ALIAS          # q's output inside the K pool
    assert append(lib, c=cache(v=E + 256)) == b.QKNORM_ERR_ALIAS  # K and V pools overlap
    assert append(lib, k=E) == b.QKNORM_ERR_ALIAS                # k comes out of the pool it goes to
    import torch
    if not torch.cuda.is_available():
        assert append(lib, norm=0, gq=None, gk=None, eps=-1.0) == b.QKNORM_ERR_CUDA
        assert append(lib, q=None, oq=None, gq=None, dq=0) == b.QKNORM_ERR_CUDA
        # K and V side by side: in one page, in one token, heads before tokens
        assert append(lib, c=cache(v=E + 2 * 2048, k_page=4096, v_page=4096)) == b.QKNORM_ERR_CUDA
        assert append(lib, c=cache(v=E + 256, k_page=4096, v_page=4096, k_token=256, v_token=256)) == b.QKNORM_ERR_CUDA
        assert append(lib, c=cache(k_head=1024, k_token=64, v_head=1024, v_token=64)) == b.QKNORM_ERR_CUDA


def attention(lib, c=None, q=A, ldq=0, table=G, cols=4, ldt=0, lens=G + 0x100000, starts=G + 0x200000, B_=2, T=4, max_q=2, max_kv=64, hq=4,
              scale=0.125, causal=1, window=0, out=D, ldo=0, lse=None, ws=H, ws_bytes=1 << 24):
    c = cache() if c is None else c
    return lib.qknorm_attn_paged(q, ldq, ctypes.byref(c) if c else None, table, cols, ldt, lens, starts, B_, T, max_q, max_kv, hq, scale,
                                 causal, window, out, ldo, lse, ws, ws_bytes, None)


def test_attention_argument_errors(lib):
    b = binding
    for kw in (dict(T=0), dict(B_=0), dict(max_q=0)):
        assert attention(lib, **kw) == b.QKNORM_OK, kw
    assert attention(lib, c=False) == b.QKNORM_ERR_NULL
    for kw, name in BAD_CACHES:
        assert attention(lib, c=cache(**kw)) == getattr(b, "QKNORM_ERR_" + name), kw
    for kw in (dict(T=-1), dict(B_=-1), dict(max_q=-1), dict(max_kv=-1), dict(max_kv=0x7fffffff), dict(window=-1), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(causal=2), dict(cols=-1), dict(ldt=3), dict(ldq=100),
               dict(ldo=-4), dict(T=1 << 31)):
        assert attention(lib, **kw) == b.QKNORM_ERR_SHAPE, kw
    assert attention(lib, hq=3) == b.QKNORM_ERR_HEADS
    assert attention(lib, hq=0) == b.QKNORM_ERR_HEADS
    for n in ("q", "out", "table", "lens", "starts"):
        assert attention(lib, **{n: None}) == b.QKNORM_ERR_NULL, n
    for kw in (dict(q=A + 1), dict(out=D + 1), dict(table=G + 2), dict(lens=G + 2), dict(starts=G + 1), dict(lse=C + 2)):
        assert attention(lib, **kw) == b.QKNORM_ERR_ALIGN, kw
    import torch
    if not torch.cuda.is_available():
        assert attention(lib) == b.QKNORM_ERR_CUDA                     # everything but the device is in order
        assert attention(lib, cols=0, table=None) == b.QKNORM_ERR_CUDA  # no page at all: every row is empty


def test_workspace_argument_errors(lib):
    out = ctypes.c_int64(-1)
    ask = lambda seqs=4, T=8, mq=2, mk=64, hq=8, hk=2, hd=64, w=0: lib.qknorm_attn_paged_workspace(seqs, T, mq, mk, hq, hk, hd, w, ctypes.byref(out))
    assert lib.qknorm_attn_paged_workspace(1, 1, 1, 1, 1, 1, 64, 0, None) == binding.QKNORM_ERR_NULL
    assert ask(T=0) == binding.QKNORM_OK and out.value == 0
    assert ask(hq=7) == binding.QKNORM_ERR_HEADS
    assert ask(hd=513) == binding.QKNORM_ERR_HEADS
    assert ask(w=-1) == binding.QKNORM_ERR_SHAPE
    assert ask(mk=-1) == binding.QKNORM_ERR_SHAPE


def frequencies(rot_dim, theta, scaling, factor=1.0, orig=0.0, low=1.0, high=32.0):
    """The scalings of the header, written from their definitions."""
    out = []
    for i in range(rot_dim // 2):
        f = theta ** (-2.0 * i / rot_dim)
        if scaling == "linear":
            f /= factor
        elif scaling == "base":
            f = (theta * factor ** (rot_dim / (rot_dim - 2))) ** (-2.0 * i / rot_dim)
        elif scaling == "ramp":
            at = lambda n: rot_dim * math.log(orig / (n * 2 * math.pi)) / (2 * math.log(theta))
            a, z = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot_dim - 1)
            ramp = min(max((i - a) / ((z - a) or 0.001), 0.0), 1.0)
            f = f / factor * ramp + f * (1 - ramp)
        elif scaling == "bands":
            turns = orig * f / (2 * math.pi)
            if turns <= low:
                f /= factor
            elif turns < high:
                t = (turns - low) / (high - low)
                f = (1 - t) * f / factor + t * f
        out.append(f)
    return out


@pytest.mark.parametrize("rot_dim,theta,scaling,kw", [
    (128, 10000.0, "plain", {}), (2, 500000.0, "plain", {}), (64, 10000.0, "linear", dict(factor=4.0)),
    (128, 10000.0, "base", dict(factor=8.0)), (128, 10000.0, "ramp", dict(factor=16.0, original_len=4096, low=1.0, high=32.0)),
    (96, 500000.0, "ramp", dict(factor=2.0, original_len=100.0, low=1.0, high=2.0)),
    (128, 500000.0, "bands", dict(factor=8.0, original_len=8192, low=1.0, high=4.0)), (128, 10000.0, "linear", dict(factor=1.0)),
])
def test_frequencies_against_their_definitions(lib, rot_dim, theta, scaling, kw):
    got, mscale = attn.rope_frequencies(rot_dim, theta, scaling, device="cpu", **kw)
    want = frequencies(rot_dim, theta, scaling, kw.get("factor", 1.0), kw.get("original_len", 0.0), kw.get("low", 1.0), kw.get("high", 32.0))
    assert got.shape == (rot_dim // 2,)
    for g, w in zip(got.tolist(), want):
        assert abs(g - w) <= 1e-13 * w
    assert abs(mscale - (0.1 * math.log(kw["factor"]) + 1 if scaling == "ramp" else 1.0)) < 1e-7


def test_frequency_refusals(lib):
    bad = [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=514), dict(rot_dim=64, theta=1.0), dict(rot_dim=64, theta=math.nan),
           dict(rot_dim=64, scaling="linear", factor=0.5), dict(rot_dim=2, scaling="base", factor=2.0),
           dict(rot_dim=64, scaling="ramp", factor=2.0), dict(rot_dim=64, scaling="bands", factor=2.0, original_len=64, low=4.0, high=4.0)]
    for kw in bad:
        with pytest.raises(binding.QKNormError):
            attn.rope_frequencies(device="cpu", **kw)
    with pytest.raises(binding.QKNormError):
        attn.rope_frequencies(64, scaling="spiral", device="cpu")


def test_reference_inverse_rotation_is_the_gradient():
    """The reference the GPU tests use: rotating back undoes a rotation, and is its gradient by differences."""
    import torch
    from tests import attn_reference as R
    g = torch.Generator().manual_seed(3)
    x, y = torch.randn(3, 32, generator=g, dtype=torch.float64), torch.randn(3, 32, generator=g, dtype=torch.float64)
    pos, f = torch.tensor([0, 5, -1000]), torch.tensor([1.0, 0.1, 0.01], dtype=torch.float64)
    for inter in (False, True):
        fwd = lambda z: R.rotate(z, pos, f, 16, inter, False, 1.5)[0]
        assert torch.allclose(R.rotate(fwd(x), pos, f, 16, inter, True, 1 / 1.5)[0][:, :6], x[:, :6], atol=1e-12)
        grad = R.rotate(y, pos, f, 16, inter, True, 1.5)[0]
        for e in range(0, 32, 7):
            h = torch.zeros_like(x)
            h[:, e] = 1e-6
            diff = ((fwd(x + h) - fwd(x - h)) * y).sum(1) / 2e-6
            assert torch.allclose(diff, grad[:, e], atol=1e-7)


# K and V in one buffer: axes of the buffer, the side's place among them.  hd = 64, 2 heads, pages of 16, 8 pages unless said.
SHARED_BUFFERS = {
    "tokens, one page": (dict(pages=1), "ptshd"), "heads": ({}, "pthsd"), "heads before tokens": ({}, "phtsd"), "tokens of a head": ({}, "phstd"),
    "layers between": ({}, "pltshd"), "layers, heads before tokens": ({}, "plhtsd"), "pages inside": ({}, "tpshd"), "one token a page": (dict(page=1), "pthsd"),
    "one head": (dict(heads=1), "ptshd"), "side by side in a page": ({}, "psthd"), "apart": ({}, "spthd"),
}


def shared(axes, pages=8, page=16, heads=2, hd=64, layers=3):
    """(K's strides by axis, elements from K to V) of a contiguous buffer [axes]; 's' is K and V, 'l' layers."""
    size = dict(p=pages, t=page, h=heads, d=hd, s=2, l=layers)
    stride, n = {}, 1
    for a in reversed(axes):
        stride[a] = n
        n *= size[a]
    return stride, stride["s"]


@pytest.mark.parametrize("name", SHARED_BUFFERS)
@pytest.mark.parametrize("e4m3", [0, 1])
def test_append_takes_every_order_of_a_shared_buffer(lib, name, e4m3):
    """K and V that do not meet are accepted wherever the axes lie; a V that meets K is refused."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("accepted calls would run on made-up addresses")
    kw, axes = SHARED_BUFFERS[name]
    st, to_v = shared(axes, **kw)
    eb = 1 if e4m3 else 2
    at = dict(k_page=st["p"], k_token=st["t"], k_head=st["h"], v_page=st["p"], v_token=st["t"], v_head=st["h"], e4m3=e4m3, **kw)
    assert append(lib, c=cache(v=E + to_v * eb, **at), dq=0, q=None, oq=None, gq=None) == binding.QKNORM_ERR_CUDA
    for off in (0, 8, -8, *([st["t"]] if kw.get("page") != 1 else []), *([st["h"]] if kw.get("heads") != 1 else [])):
        assert append(lib, c=cache(v=E + off * eb, **at), dq=0, q=None, oq=None, gq=None) == binding.QKNORM_ERR_ALIAS, off


def test_append_finds_every_meeting_of_k_and_v(lib):
    """Small pools of random strides, K and V alike: refused exactly where two elements share a place."""
    import random
    import torch
    if torch.cuda.is_available():
        pytest.skip("accepted calls would run on made-up addresses")
    rng = random.Random(5)
    seen = {binding.QKNORM_ERR_CUDA: 0, binding.QKNORM_ERR_ALIAS: 0}
    for _ in range(4000):
        hd, n = rng.choice([1, 2, 3]), dict(p=rng.randint(1, 3), t=rng.randint(1, 3), h=rng.randint(1, 3))
        order, stride, extent = rng.sample("pth", 3), {}, hd
        for a in order:                                     # nested, with gaps
            stride[a] = extent + rng.choice([0, 0, hd, rng.randint(0, 9)])
            extent = (n[a] - 1) * stride[a] + extent
        k = {p * stride["p"] + t * stride["t"] + h * stride["h"] + d for p in range(n["p"]) for t in range(n["t"]) for h in range(n["h"]) for d in range(hd)}
        off = rng.randint(-extent - 2, extent + 2)
        c = cache(v=E + 2 * off, pages=n["p"], page=n["t"], heads=n["h"], hd=hd, k_page=stride["p"], k_token=stride["t"], k_head=stride["h"],
                  v_page=stride["p"], v_token=stride["t"], v_head=stride["h"])
        want = binding.QKNORM_ERR_ALIAS if any(e + off in k for e in k) else binding.QKNORM_ERR_CUDA
        assert append(lib, c=c, dq=0, q=None, oq=None, gq=None) == want, (n, hd, stride, off)
        seen[want] += 1
    assert min(seen.values()) > 500


def test_python_integers_past_32_bits_are_refused(lib, monkeypatch):
    """ctypes would cut them off without a word: a window of 2^32 + 1 would be one of 1."""
    import torch
    from paper_2608_09160_b200.binding import QKNormError
    monkeypatch.setattr(attn, "_device", lambda: -1)            # CPU tensors pass the checks; no call gets as far as a kernel
    monkeypatch.setattr(attn, "_current", lambda stream: 0)
    monkeypatch.setattr(attn, "_workspace", lambda *sizes: 0)
    calls = []
    monkeypatch.setattr(attn, "_invoke", lambda fn, args, stream, keep: calls.append(args))
    bf, i32 = torch.bfloat16, torch.int32
    q, pool = torch.zeros((4, 128), dtype=bf), torch.zeros((2, 16, 1, 64), dtype=bf)
    table, lens, starts = torch.zeros((2, 1), dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(3, dtype=i32)
    go = lambda max_q=2, max_kv=16, **kw: attn.qknorm_attn_paged(q, pool, pool.clone(), table, lens, starts, max_q, max_kv, **kw)
    go()
    assert len(calls) == 1
    for kw in (dict(window=2 ** 32 + 1), dict(window=2 ** 31), dict(window=-2 ** 40), dict(max_q=2 ** 32), dict(max_kv=2 ** 32 + 16), dict(max_kv=-2 ** 33)):
        with pytest.raises(QKNormError) as e:
            go(**kw)
        assert e.value.status == binding.QKNORM_ERR_SHAPE, kw
    pos, inv = torch.zeros(4, dtype=torch.int64), torch.zeros(32, dtype=torch.float64)
    attn.qknorm_rope(q, None, pos, inv, 64)
    assert len(calls) == 2
    with pytest.raises(QKNormError):
        attn.qknorm_rope(q, None, pos, inv, 2 ** 32 + 64)
    with pytest.raises(QKNormError):
        attn.rope_frequencies(2 ** 32 + 64, device="cpu")
    assert len(calls) == 2
    monkeypatch.undo()
    for i in (0, 2, 3, 4, 5, 6, 7):
        sizes = [4, 8, 2, 64, 8, 2, 64, 0]
        sizes[i] += 2 ** 32
        with pytest.raises(QKNormError) as e:
            attn.attn_paged_workspace(*sizes)
        assert e.value.status == binding.QKNORM_ERR_SHAPE, sizes


def test_scales_whose_product_no_float_holds_are_refused(lib):
    assert attention(lib, c=cache(e4m3=1, ks=1e20), scale=1e30) == binding.QKNORM_ERR_SHAPE
    assert attention(lib, scale=3e38) == binding.QKNORM_ERR_SHAPE            # times log2 e
    import torch
    if not torch.cuda.is_available():
        assert attention(lib, c=cache(ks=1e20), scale=1e30) == binding.QKNORM_ERR_CUDA      # a bf16 cache has no scale
        assert attention(lib, c=cache(e4m3=1, ks=1e-30), scale=1e-30) == binding.QKNORM_ERR_CUDA


def test_append_refuses_scales_without_a_reciprocal(lib):
    """1 / 1e-39 is no fp32 number: zeros would be written as NaN."""
    for kw in (dict(ks=1e-39), dict(vs=1e-39)):
        assert append(lib, c=cache(e4m3=1, **kw)) == binding.QKNORM_ERR_SHAPE, kw
    import torch
    if not torch.cuda.is_available():
        assert append(lib, c=cache(e4m3=1, ks=1e-37)) == binding.QKNORM_ERR_CUDA
        assert append(lib, c=cache(ks=1e-39)) == binding.QKNORM_ERR_CUDA     # a bf16 cache has no scale
        assert attention(lib, c=cache(e4m3=1, ks=1e-39)) == binding.QKNORM_ERR_CUDA   # reading multiplies
