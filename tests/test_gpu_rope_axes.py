"""Rotary positions with several axes against their 64-bit definition: forward, backward, FP8, the fused cache write."""
import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests import attn_reference as R
from tests.attn_reference import BF16, F8

pytestmark = pytest.mark.gpu


def turn(x, pos, inv_freq, axis, hd, inter, inverse=False, mscale=1.0):
    """(rotated, magnitude of every element's pair): the one-axis definition, pair by pair with the positions of its axis."""
    y, mag = x.clone().reshape(x.shape[0], -1, hd), x.abs().clone().reshape(x.shape[0], -1, hd)
    n = len(inv_freq)
    for i in range(n):
        a = int(axis[i])
        p = pos[a] if a < pos.shape[0] else torch.zeros_like(pos[0])
        only = torch.zeros(n, dtype=torch.float64)
        only[i] = inv_freq[i]
        yi, mi = R.rotate(x, p, only, hd, inter, inverse, mscale)
        at = [2 * i, 2 * i + 1] if inter else [i, i + n]
        y[:, :, at], mag[:, :, at] = yi.view(y.shape)[:, :, at], mi.view(y.shape)[:, :, at]
    return y.reshape(x.shape), mag.reshape(x.shape)


def check(got, want, mag, dtype):
    """As for one axis: half a step of the storage format, and 1e-6 of the pair for cos, sin and two products in fp32."""
    tol = R.HALF_STEP[dtype] * want.abs() + 1e-6 * mag + (R.F8_TINY if dtype is F8 else 0.0)
    if dtype is F8:
        want = want.clamp(-448, 448)
    bad = ~((got.detach().cpu().double() - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first {bad.nonzero()[0].tolist()}"


CASES = [
    # T, heads_q, heads_k, head_dim, rot_dim, interleaved, inverse, axes
    (1, 1, 1, 64, 64, False, False, 3), (65, 5, 1, 128, 128, False, True, 3), (65, 7, 1, 96, 48, True, False, 2), (700, 2, 2, 64, 64, True, True, 4),
    (300, 4, 2, 80, 32, False, False, 8), (5, 40, 8, 128, 64, False, False, 1), (2, 3, 1, 50, 20, False, True, 3), (301, 2, 1, 34, 34, True, False, 3),
    (3, 0, 3, 256, 16, False, True, 2), (3, 128, 0, 512, 256, True, False, 3),
]


@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,hq,hk,hd,rot,inter,inverse,axes", CASES)
def test_rope_axes(libqknorm, T, hq, hk, hd, rot, inter, inverse, axes, dtype):
    g = torch.Generator().manual_seed(T + hd)
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    pos = torch.randint(-5, 1_000_000, (axes, T), generator=g)
    axis = torch.randint(0, axes + 1, (rot // 2,), generator=g).to(torch.uint8)     # one beyond: position 0
    x = {"q": torch.randn((T, hq * hd), generator=g).to(dtype), "k": torch.randn((T, hk * hd), generator=g).to(dtype)}
    wide = torch.full((axes, T + 3), 10 ** 9)
    wide[:, :T] = pos
    got = attn.qknorm_rope(*(x[n].cuda() if x[n].shape[1] else None for n in "qk"), wide.cuda()[:, :T], inv.cuda(), hd, interleaved=inter,
                           inverse=inverse, mscale=1.25, axis=axis.cuda())
    torch.cuda.synchronize()
    for n, y in zip("qk", got):
        if x[n].shape[1]:
            check(y, *turn(x[n].double(), pos, inv, axis, hd, inter, inverse, 1.25), dtype)


def test_equal_axes_give_the_bits_of_one(libqknorm):
    g = torch.Generator().manual_seed(1)
    q, k = torch.randn((200, 512), generator=g).to(BF16).cuda(), torch.randn((200, 256), generator=g).to(BF16).cuda()
    inv, _ = attn.rope_frequencies(128)
    pos = torch.randint(0, 10 ** 6, (200,), generator=g).cuda()
    one = attn.qknorm_rope(q, k, pos, inv, 128)
    axis = attn.rope_axes([16, 24, 24])
    many = attn.qknorm_rope(q, k, pos.expand(3, -1).contiguous(), inv, 128, axis=axis)
    for a, b in zip(one, many):
        assert torch.equal(a, b)


def test_backward_is_the_gradient(libqknorm):
    """inverse=True on dL/dy against the formula's gradient and against differences of a loss in 64 bits."""
    g = torch.Generator().manual_seed(2)
    T, hd, axes = 6, 64, 3
    inv = 10000.0 ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
    pos, axis = torch.randint(0, 5000, (axes, T), generator=g), attn.rope_axes([8, 12, 12], turns=True, device="cpu")
    x = torch.randn((T, 2 * hd), generator=g).to(BF16).double().requires_grad_()
    w = torch.randn((T, 2 * hd), generator=g).to(BF16)
    loss = lambda v: (turn(v, pos, inv, axis, hd, False)[0] * w.double()).sum()
    want, = torch.autograd.grad(loss(x), x)
    got, _ = attn.qknorm_rope(w.cuda(), None, pos.cuda(), inv.cuda(), hd, inverse=True, axis=axis.cuda())
    check(got, want, turn(w.double(), pos, inv, axis, hd, False, True)[1], BF16)
    for r, c in ((0, 3), (5, 100), (2, 64)):
        d = torch.zeros_like(x)
        d[r, c] = 1e-4
        slope = float((loss(x.detach() + d) - loss(x.detach() - d)) / 2e-4)
        assert abs(slope - float(got[r, c])) <= 2.0 ** -8 * abs(slope) + 1e-5


@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
def test_append_with_axes(libqknorm, dtype):
    """Norm, rotation and cache write in one, against the norm and then the rotation on their own."""
    g = torch.Generator().manual_seed(3)
    T, hq, hk, hd, page = 70, 4, 2, 128, 16
    q, k, v = (torch.randn((T, h * hd), generator=g).to(BF16) for h in (hq, hk, hk))
    gq, gk = ((torch.rand(h * hd, generator=g) + 0.5).to(BF16) for h in (hq, hk))
    inv = 10000.0 ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
    pos, axis = torch.randint(0, 20000, (3, T), generator=g), attn.rope_axes([16, 24, 24], device="cpu")
    slots = torch.randperm(6 * page, generator=g)[:T]
    pools = [torch.zeros((6, page, hk, hd), dtype=dtype, device="cuda") for _ in range(2)]
    c = lambda t: t.cuda()
    out = attn.qknorm_fwd_append(c(q), c(k), c(v), c(gq), c(gk), c(pos), c(inv), c(slots), *pools, 1e-6, axis=c(axis), k_scale=0.5, v_scale=0.5)
    assert binding.last_variant() == "append"
    torch.cuda.synchronize()
    scale = 0.5 if dtype is F8 else 1.0
    for got, x, gamma, d, s in ((out.cpu(), q, gq, BF16, 1.0), (pools[0].cpu().view(-1, hk * hd)[slots], k, gk, dtype, scale)):
        y = R.norm(x.double(), gamma.double(), 1e-6, x.shape[1])
        want, mag = turn(y, pos, inv, axis, hd, False)
        check(got, want / s, mag / s * 4, d)        # the norm's statistic and products add as much again, twice over


def test_captured_and_replayed_on_new_positions(libqknorm):
    g = torch.Generator().manual_seed(4)
    q = torch.randn((9, 256), generator=g).to(BF16).cuda()
    inv, _ = attn.rope_frequencies(128)
    pos, axis = torch.zeros((3, 9), dtype=torch.int64, device="cuda"), attn.rope_axes([16, 24, 24])
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.qknorm_rope(q, None, pos, inv, 128, out, axis=axis)
    for seed in (5, 6):
        pos.copy_(torch.randint(0, 9999, (3, 9), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        want = attn.qknorm_rope(q, None, pos, inv, 128, axis=axis)[0]
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_python_refusals(libqknorm):
    q = torch.zeros((4, 128), dtype=BF16, device="cuda")
    inv = torch.ones(64, dtype=torch.float64, device="cuda")
    pos, axis = torch.zeros((3, 4), dtype=torch.int64, device="cuda"), torch.zeros(64, dtype=torch.uint8, device="cuda")
    for bad in (dict(positions=pos[0]), dict(positions=pos.int()), dict(positions=pos[:, :3]), dict(positions=pos.T.contiguous().T),
                dict(positions=pos.cpu()), dict(positions=pos.expand(3, 4)[:0]), dict(positions=torch.zeros((9, 4), dtype=torch.int64, device="cuda")),
                dict(axis=axis[:32]), dict(axis=axis.int()), dict(axis=axis.cpu()), dict(inv_freq=inv.float()), dict(inv_freq=None)):
        kw = dict(positions=pos, inv_freq=inv, axis=axis) | bad
        with pytest.raises(binding.QKNormError):
            attn.qknorm_rope(q, None, kw["positions"], kw["inv_freq"], 128, axis=kw["axis"])
    for sections in ([], [-1, 3], [1] * 9):
        with pytest.raises(binding.QKNormError):
            attn.rope_axes(sections)
