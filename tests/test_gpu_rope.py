"""Rotary positions and the fused norm + rotation + cache write against 64-bit definitions."""
import numpy as np
import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests import attn_reference as R
from tests.attn_reference import BF16, F8

pytestmark = pytest.mark.gpu
EPS = 1e-6


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=g) * sigma).to(dtype)


def check(got, want, mag, dtype, what, rel32=1e-6, extra=0.0):
    """|got - want| <= half a step of the storage format + rel32 of the pair's magnitude (fp32 cos, sin and products: the
    angle is off by at most 2^-25 turns' worth, cos and sin by an ulp, two products and a sum by half an ulp each)."""
    got = got.detach().cpu().double()
    tol = R.HALF_STEP[dtype] * want.abs() + rel32 * mag + extra
    if dtype is F8:
        tol = tol + R.F8_TINY
        want = want.clamp(-448, 448)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


CASES = [
    # T, heads_q, heads_k, head_dim, rot_dim, interleaved, inverse
    (1, 1, 1, 64, 64, False, False),
    (3, 2, 1, 128, 128, True, False),
    (65, 5, 1, 128, 64, False, True),
    (65, 7, 1, 96, 96, True, True),
    (300, 4, 2, 80, 32, False, False),
    (700, 2, 2, 64, 64, True, False),       # short rows: tokens share a CTA
    (5, 40, 8, 128, 128, False, False),
    (2, 3, 1, 50, 20, False, False),        # general kernel
    (301, 2, 1, 34, 34, True, True),
    (4, 1, 1, 512, 512, False, False),
    (3, 128, 0, 512, 256, True, False),     # the widest row, Q alone
    (3, 0, 3, 256, 16, False, True),        # K alone
    (2, 256, 64, 16, 16, False, False),
    (2, 512, 512, 128, 128, True, False),   # more units than one CTA takes
]


@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,hq,hk,hd,rot,inter,inverse", CASES)
def test_rope(libqknorm, T, hq, hk, hd, rot, inter, inverse, dtype):
    g = gen(T + hd)
    inv, mscale = attn.rope_frequencies(rot, 10000.0, "ramp", factor=4.0, original_len=4096)
    pos = torch.randint(-5, 1_000_000, (T,), generator=g)
    x = {"q": randn(g, (T, hq * hd), dtype), "k": randn(g, (T, hk * hd), dtype)}
    dev = {n: t.cuda() if t.shape[1] else None for n, t in x.items()}
    got = attn.qknorm_rope(dev["q"], dev["k"], pos.cuda(), inv, hd, interleaved=inter, inverse=inverse, mscale=mscale)
    torch.cuda.synchronize()
    for n, y in zip(("q", "k"), got):
        if dev[n] is None:
            continue
        want, mag = R.rotate(R.widen(x[n]), pos, inv.cpu(), hd, inter, inverse, mscale)
        check(y, want, mag, dtype, n)
        assert torch.equal(dev[n].cpu().view(torch.uint8), x[n].view(torch.uint8))    # inputs as they were


@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("hd,rot,skew", [(128, 128, 0), (128, 64, 0), (128, 128, 1), (40, 24, 0)])
def test_rope_in_place_inside_a_fused_buffer(libqknorm, hd, rot, skew, dtype):
    """Q and K as column blocks of one projection output, rotated in place; V's columns and the rows behind stay."""
    g = gen(hd + skew)
    T, hq, hk = 130, 6, 2
    width = (hq + 2 * hk) * hd
    whole = randn(g, (T + 2, width + 16), dtype)
    dev = whole.cuda()
    q, k = dev[:T, skew:skew + hq * hd], dev[:T, skew + hq * hd:skew + (hq + hk) * hd]
    inv, _ = attn.rope_frequencies(rot)
    pos = torch.arange(T) + 100_000
    attn.qknorm_rope(q, k, pos.cuda(), inv, hd, q, k)
    torch.cuda.synchronize()
    n = (hq + hk) * hd
    want, mag = R.rotate(R.widen(whole[:T, skew:skew + n]), pos, inv.cpu(), hd, False)
    check(dev[:T, skew:skew + n], want, mag, dtype, "q, k")
    after, before = dev.cpu().view(torch.uint8), whole.view(torch.uint8)
    e = whole.element_size()
    assert torch.equal(after[:, (skew + n) * e:], before[:, (skew + n) * e:])
    assert torch.equal(after[:, :skew * e], before[:, :skew * e]) and torch.equal(after[T:], before[T:])


def test_rope_far_positions_keep_their_angle(libqknorm):
    """Position 10^9 at frequency 1: fp32 would be off by dozens of radians."""
    hd = 64
    pos = torch.tensor([10 ** 9, -10 ** 9, 2 ** 31 + 7, 123456789])
    inv, _ = attn.rope_frequencies(hd)
    x = torch.ones((4, hd), dtype=BF16)
    y, _ = attn.qknorm_rope(x.cuda(), None, pos.cuda(), inv, hd)
    want, mag = R.rotate(R.widen(x), pos, inv.cpu(), hd, False)
    check(y, want, mag, BF16, "far", rel32=3e-6)     # the 64-bit reference's own angle: 10^9 * 2^-53 * 2 pi = 7e-7


def test_rope_backward_is_the_gradient(libqknorm):
    """inverse=True against autograd of the 64-bit definition, and against differences of the kernel's own forward."""
    hd, rot, T = 64, 32, 9
    g = gen(5)
    inv, _ = attn.rope_frequencies(rot)
    pos = torch.randint(0, 5000, (T,), generator=g)
    x, up = randn(g, (T, 2 * hd), BF16), randn(g, (T, 2 * hd), BF16)
    for inter in (False, True):
        leaf = R.widen(x).requires_grad_()
        h = leaf.reshape(T, 2, hd)
        i = torch.arange(rot // 2)
        ia, ib = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        ang = pos.double()[:, None, None] * inv.cpu()
        z = torch.complex(h[..., ia], h[..., ib]) * torch.polar(torch.full_like(ang, 1.25), ang)
        w = R.widen(up).reshape(T, 2, hd)
        loss = (z.real * w[..., ia]).sum() + (z.imag * w[..., ib]).sum() + (h[..., rot:] * w[..., rot:]).sum()
        loss.backward()
        got, _ = attn.qknorm_rope(up.cuda(), None, pos.cuda(), inv, hd, interleaved=inter, inverse=True, mscale=1.25)
        _, mag = R.rotate(R.widen(up), pos, inv.cpu(), hd, inter, True, 1.25)
        check(got, leaf.grad, mag, BF16, "gradient")
        # the kernel's forward is linear: <up, F(e)> for unit vectors e, within two roundings
        for e in (0, 1, rot // 2, rot - 1, rot, hd + 3):
            unit = torch.zeros((T, 2 * hd), dtype=BF16)
            unit[:, e] = 1.0
            y, _ = attn.qknorm_rope(unit.cuda(), None, pos.cuda(), inv, hd, interleaved=inter, mscale=1.25)
            diff = (y.cpu().double() * R.widen(up)).sum(1)
            tol = 2 * 2.0 ** -8 * (y.cpu().double().abs() * R.widen(up).abs()).sum(1) + 2.0 ** -8 * diff.abs() + 1e-5
            assert ((got.cpu().double()[:, e] - diff).abs() <= tol).all()


def test_rope_special_values(libqknorm):
    """NaN and infinities stay in their pair; the pass-through part is copied bit for bit."""
    hd, rot = 64, 32
    x = torch.ones((2, 2 * hd), dtype=BF16)
    x[0, 3], x[1, hd + 1], x[0, 40], x[0, 41] = float("nan"), float("inf"), float("nan"), float("-inf")
    inv, _ = attn.rope_frequencies(rot)
    y, _ = attn.qknorm_rope(x.cuda(), None, torch.tensor([7, 9]).cuda(), inv, hd)
    y = y.cpu()
    bad = ~torch.isfinite(y)
    where = {tuple(v) for v in bad.nonzero().tolist()}
    assert where == {(0, 3), (0, 19), (1, hd + 1), (1, hd + 17), (0, 40), (0, 41)}
    assert y[0, 41] == float("-inf")


# ---- norm + rotation + cache write ------------------------------------------------------------------

def pools(g, pages, page, heads, hd, dtype, order="nhd"):
    """K and V pools filled with values, as strided views of `order`; also the whole buffers."""
    shape = {"nhd": (2, pages, page, heads, hd), "hnd": (2, pages, heads, page, hd), "paired": (pages, 2, page, heads, hd),
             "inner": (pages, page, 2, heads, hd)}[order]
    buf = randn(g, shape, dtype).cuda()
    k, v = {"nhd": lambda: (buf[0], buf[1]), "hnd": lambda: (buf[0].transpose(1, 2), buf[1].transpose(1, 2)),
            "paired": lambda: (buf[:, 0], buf[:, 1]), "inner": lambda: (buf[:, :, 0], buf[:, :, 1])}[order]()
    return k, v, buf


APPEND = [
    # T, heads_q, heads, head_dim, rot_dim, interleaved, norm, cache, page, order
    (1, 2, 1, 64, 64, False, "layerwise", BF16, 16, "nhd"),
    (7, 5, 1, 128, 128, True, "headwise", BF16, 16, "hnd"),
    (64, 40, 8, 128, 128, False, "layerwise", BF16, 16, "paired"),
    (333, 8, 2, 96, 48, True, "headwise", F8, 24, "inner"),
    (333, 7, 1, 64, 64, False, "layerwise", F8, 1, "nhd"),
    (600, 4, 4, 80, 80, False, "headwise", BF16, 7, "nhd"),
    (5, 3, 2, 50, 20, False, "layerwise", BF16, 5, "hnd"),        # general kernel
    (301, 3, 2, 34, 16, True, "headwise", F8, 16, "inner"),
    (17, 2, 2, 128, 0, False, "layerwise", F8, 16, "nhd"),        # no rotation
    (17, 4, 2, 128, 128, False, None, BF16, 16, "nhd"),           # no norm
    (9, 0, 2, 64, 64, False, "layerwise", BF16, 16, "nhd"),       # no q
    (3, 480, 16, 128, 128, False, "layerwise", BF16, 16, "nhd"),  # more units than one CTA takes
    (310, 64, 8, 128, 128, False, "layerwise", BF16, 64, "nhd"),
]


@pytest.mark.parametrize("T,hq,hk,hd,rot,inter,norm,cdt,page,order", APPEND)
def test_append(libqknorm, T, hq, hk, hd, rot, inter, norm, cdt, page, order):
    g = gen(T + hq + hd)
    dq, dk = hq * hd, hk * hd
    qkv = randn(g, (T, dq + 2 * dk), BF16)
    gq, gk = ((torch.rand(n, generator=g) + 0.5).to(BF16) for n in (dq, dk))
    pos = torch.randint(0, 100_000, (T,), generator=g)
    inv = attn.rope_frequencies(rot)[0] if rot else None
    pages = T // page + 3
    k_pool, v_pool, buf = pools(g, pages, page, hk, hd, cdt, order)
    before = buf.clone()
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 4:
        slots[1], slots[3], slots[4] = -1, pages * page, -2 ** 40      # padded tokens
    ks, vs = (0.25, 0.5) if cdt is F8 else (1.0, 1.0)
    dev = qkv.cuda()
    q, k, v = dev[:, :dq], dev[:, dq:dq + dk], dev[:, dq + dk:]
    out = attn.qknorm_fwd_append(q if hq else None, k, v, gq.cuda() if norm and hq else None, gk.cuda() if norm else None,
                                 pos.cuda() if rot else None, inv, slots.cuda(), k_pool, v_pool, EPS, headwise=norm == "headwise",
                                 interleaved=inter, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    assert torch.equal(dev.cpu(), qkv)
    f = inv.cpu() if rot else torch.zeros(0, dtype=torch.float64)

    def want(x, gamma, d):
        x = R.widen(x)
        if norm:
            x = R.norm(x, R.widen(gamma), EPS, hd if norm == "headwise" else d)
        return R.rotate(x, pos, f, hd, inter)
    # on top of the rotation's 1e-6: the fp32 sum of squares over a row, 40 steps of 2^-24 through the sqrt, and two products
    rel = 1e-6 + 3e-6
    if hq:
        w, mag = want(qkv[:, :dq], gq, dq)
        check(out, w, mag, BF16, "q", rel)
    w, mag = want(qkv[:, dq:dq + dk], gk, dk)
    ok = (slots >= 0) & (slots < pages * page)
    rows = slots[ok]
    at = (rows // page, rows % page)
    check(k_pool.cpu()[at].reshape(-1, dk), w[ok] / ks, mag[ok] / ks, cdt, "k", rel)
    wv = R.widen(qkv[:, dq + dk:])[ok]
    check(v_pool.cpu()[at].reshape(-1, dk), wv / vs, wv.abs() / vs, cdt, "v", 1e-6)
    if cdt is BF16:
        assert torch.equal(v_pool.cpu()[at].reshape(-1, dk), qkv[:, dq + dk:][ok])
    # every other slot as it was
    k_pool[at[0].cuda(), at[1].cuda()] = 0
    v_pool[at[0].cuda(), at[1].cuda()] = 0
    k0, v0, _ = {"nhd": lambda b: (b[0], b[1], b), "hnd": lambda b: (b[0].transpose(1, 2), b[1].transpose(1, 2), b),
                 "paired": lambda b: (b[:, 0], b[:, 1], b), "inner": lambda b: (b[:, :, 0], b[:, :, 1], b)}[order](before)
    k0[at[0].cuda(), at[1].cuda()] = 0
    v0[at[0].cuda(), at[1].cuda()] = 0
    assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))


def test_append_q_in_place_and_agrees_with_the_separate_steps(libqknorm):
    """The fused call against qknorm_fwd, qknorm_rope and a copy: apart by the roundings in between."""
    g = gen(11)
    T, hq, hk, hd = 200, 8, 2, 128
    q, k, v = randn(g, (T, hq * hd), BF16).cuda(), randn(g, (T, hk * hd), BF16).cuda(), randn(g, (T, hk * hd), BF16).cuda()
    gq, gk = ((torch.rand(n, generator=g) + 0.5).to(BF16).cuda() for n in (hq * hd, hk * hd))
    inv, _ = attn.rope_frequencies(hd)
    pos = torch.arange(T, device="cuda")
    nq, nk = binding.qknorm_fwd(q, k, gq, gk, EPS)
    rq, rk = attn.qknorm_rope(nq, nk, pos, inv, hd)
    kp, vp = (torch.zeros((20, 16, hk, hd), dtype=BF16, device="cuda") for _ in range(2))
    attn.qknorm_fwd_append(q, k, v, gq, gk, pos, inv, pos + 16, kp, vp, EPS, q)
    torch.cuda.synchronize()
    for a, b in ((q, rq), (kp.view(-1, hk * hd)[16:16 + T], rk)):
        # two roundings of 2^-8 on each element of a pair
        assert ((a.double() - b.double()).abs() <= 3 * 2.0 ** -8 * b.double().abs().amax()).all()
        assert ((a.double() - b.double()).norm() <= 2.0 ** -8 * b.double().norm())
    assert torch.equal(vp.view(-1, hk * hd)[16:16 + T], v)
    assert binding.last_variant() == "append"


def test_empty_pool_and_no_tokens(libqknorm):
    hd = 64
    inv, _ = attn.rope_frequencies(hd)
    none = torch.empty((0, 2, 1, hd), dtype=BF16, device="cuda")
    x, g = torch.ones((3, hd), dtype=BF16, device="cuda"), torch.ones(hd, dtype=BF16, device="cuda")
    pos = torch.zeros(3, dtype=torch.int64, device="cuda")
    out = attn.qknorm_fwd_append(x, x.clone(), x.clone(), g, g, pos, inv, pos, none, none, EPS)
    torch.cuda.synchronize()
    assert torch.equal(out, torch.ones_like(out))
    n0 = binding.launch_count()
    attn.qknorm_rope(x[:0], None, pos[:0], inv, hd)
    assert binding.launch_count() == n0


def test_python_refusals(libqknorm):
    hd = 64
    inv, _ = attn.rope_frequencies(hd)
    x = torch.ones((3, hd), dtype=BF16, device="cuda")
    pos = torch.zeros(3, dtype=torch.int64, device="cuda")
    pool = torch.zeros((2, 16, 1, hd), dtype=BF16, device="cuda")
    bad = [
        lambda: attn.qknorm_rope(x, None, pos.int(), inv, hd),
        lambda: attn.qknorm_rope(x, None, pos[:2], inv, hd),
        lambda: attn.qknorm_rope(x, None, pos, inv.float(), hd),
        lambda: attn.qknorm_rope(x.float(), None, pos, inv, hd),
        lambda: attn.qknorm_rope(x, x[:2], pos, inv, hd),
        lambda: attn.qknorm_rope(None, None, pos, inv, hd),
        lambda: attn.qknorm_rope(x, None, None, None, hd),
        lambda: attn.qknorm_rope(x, None, pos, inv, 32),                       # rot_dim beyond head_dim
        lambda: attn.qknorm_rope(x, None, pos, inv, hd, x[:, :32]),
        lambda: attn.qknorm_fwd_append(x, x, x, None, None, pos, inv, pos, pool, pool, EPS),   # K and V in one place
        lambda: attn.qknorm_fwd_append(x, x, x, None, None, pos, inv, pos, pool, pool.clone()[..., :32], EPS),
        lambda: attn.qknorm_fwd_append(x, x[:, :32], x, None, None, pos, inv, pos, pool, pool.clone(), EPS),
        lambda: attn.qknorm_fwd_append(x, x, x, None, None, pos, inv, pos.int(), pool, pool.clone(), EPS),
        lambda: attn.qknorm_fwd_append(x, x, x, None, None, pos, inv, pos, pool.float(), pool.float(), EPS),
    ]
    n0 = binding.launch_count()
    for i, f in enumerate(bad):
        with pytest.raises(binding.QKNormError):
            f()
            pytest.fail(f"call {i} was accepted")
    assert binding.launch_count() == n0


def test_captured_and_replayed_on_new_inputs(libqknorm):
    hd, T = 128, 33
    g = gen(2)
    inv, _ = attn.rope_frequencies(hd)
    x = randn(g, (T, 4 * hd), BF16).cuda()
    pos = torch.arange(T, device="cuda")
    out = torch.empty_like(x)
    attn.qknorm_rope(x, None, pos, inv, hd, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.qknorm_rope(x, None, pos, inv, hd, out)
    for step in range(3):
        new = randn(g, (T, 4 * hd), BF16)
        x.copy_(new)
        pos.add_(1000)
        graph.replay()
        torch.cuda.synchronize()
        want, mag = R.rotate(R.widen(new), pos.cpu(), inv.cpu(), hd, False)
        check(out, want, mag, BF16, f"replay {step}")


@pytest.mark.parametrize("cdt", [BF16, F8], ids=["bf16", "e4m3"])
def test_append_tokens_with_one_slot(libqknorm, cdt):
    """Several tokens of a call name a slot: every value there is one of theirs, all other slots and q are as they would be."""
    g = gen(17)
    T, hq, hk, hd = 300, 4, 2, 64
    q, k, v = (randn(g, (T, n * hd), BF16).cuda() for n in (hq, hk, hk))
    slots = torch.arange(T, device="cuda")
    slots[1::3] = 450
    kp, vp = (torch.zeros((32, 16, hk, hd), dtype=cdt, device="cuda") for _ in range(2))
    out = attn.qknorm_fwd_append(q, k, v, None, None, None, None, slots, kp, vp, EPS)
    torch.cuda.synchronize()
    assert torch.equal(out, q)
    for pool, x in ((kp, k), (vp, v)):
        rows, want = pool.view(-1, hk * hd).float(), x.to(cdt).float()
        alone = slots != 450
        assert torch.equal(rows[slots[alone]], want[alone])
        assert (rows[450] == want[~alone]).any(0).all()
        untouched = torch.ones(len(rows), dtype=torch.bool, device="cuda")
        untouched[slots] = False
        assert (rows[untouched] == 0).all()


@pytest.mark.parametrize("cdt", [BF16, F8], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("pages,shape,order", [
    # a buffer's axes: p pages, t tokens, s K and V, h heads, d head_dim, l layers (the second is used)
    (1, (1, 64, 2, 2, 64), "ptshd"), (5, (5, 16, 2, 2, 64), "pthsd"), (5, (5, 2, 16, 2, 64), "phtsd"), (5, (5, 2, 2, 16, 64), "phstd"),
    (5, (5, 3, 16, 2, 2, 64), "pltshd"), (5, (5, 3, 2, 16, 2, 64), "plhtsd"), (5, (16, 5, 2, 2, 64), "tpshd"),
])
def test_append_into_every_order_of_a_shared_buffer(libqknorm, pages, shape, order, cdt):
    """K and V between one another in one buffer: what separate pools get, nothing else in the buffer touched; attention reads it."""
    g = gen(len(order) + pages)
    T, hq, hk, hd = 40, 4, 2, 64
    buf = randn(g, shape, cdt).cuda()
    raw = torch.uint8 if cdt is F8 else torch.int16
    before = buf.view(raw).clone()

    def side(b, which):
        view = b.select(order.index("l"), 1) if "l" in order else b
        axes = order.replace("l", "")
        view, axes = view.select(axes.index("s"), which), axes.replace("s", "")
        return view.permute([axes.index(a) for a in "pthd"])
    kp, vp = side(buf, 0), side(buf, 1)
    k2, v2 = kp.contiguous(), vp.contiguous()
    q, k, v = (randn(g, (T, n * hd), BF16).cuda() for n in (hq, hk, hk))
    gq, gk = torch.ones(hq * hd, dtype=BF16, device="cuda"), torch.ones(hk * hd, dtype=BF16, device="cuda")
    inv, _ = attn.rope_frequencies(hd)
    pos = torch.arange(T, device="cuda")
    slots = torch.randperm(kp.shape[0] * kp.shape[1], generator=g)[:T].cuda()
    for a, b in ((kp, vp), (k2, v2)):
        attn.qknorm_fwd_append(q, k, v, gq, gk, pos, inv, slots, a, b, EPS, k_scale=0.5, v_scale=0.25)
    torch.cuda.synchronize()
    assert torch.equal(kp.contiguous().view(raw), k2.view(raw)) and torch.equal(vp.contiguous().view(raw), v2.view(raw))
    want = before.clone()
    for which, pool in ((0, k2), (1, v2)):
        side(want, which).copy_(pool.view(raw))
    assert torch.equal(buf.view(raw), want)
    page = kp.shape[1]
    table = torch.arange(kp.shape[0], dtype=torch.int32, device="cuda")[None]
    lens, starts = torch.tensor([T], dtype=torch.int32, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda")
    outs = [attn.qknorm_attn_paged(q, a, b, table, lens, starts, T, page * kp.shape[0], k_scale=0.5, v_scale=0.25) for a, b in ((kp, vp), (k2, v2))]
    torch.cuda.synchronize()
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
