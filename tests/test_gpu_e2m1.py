"""The 4-bit cache: what is written into it and attention over it, against 64-bit definitions (tests/e2m1_reference.py,
tests/attn_reference.py)."""
import math

import numpy as np
import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests import attn_reference as R
from tests import e2m1_reference as E
from tests.e2m1_reference import BF16, F8

pytestmark = pytest.mark.gpu

# A normalised and rotated fp32 value is off by a few steps of 2^-24: the statistic, two products and the rotation of a pair, whose
# other element may be as large as the block's largest is small.
OFF = 2.0 ** -19


def lay(t, order):
    """t [pages, page, heads, n] on the GPU with its axes in memory in that order."""
    perm = {"nhd": (0, 1, 2, 3), "hnd": (0, 2, 1, 3), "thd": (1, 0, 2, 3)}[order]
    inv = [perm.index(i) for i in range(4)]
    raw = t.view(torch.uint8)
    return raw.permute(perm).contiguous().cuda().permute(inv)


class Layer:
    def __init__(self, T, hq, hk, hd, page=16, order="hnd", seed=0, rot=None, axes=0, sigma=1.0):
        g = torch.Generator().manual_seed(seed)
        self.T, self.hq, self.hk, self.hd, self.page = T, hq, hk, hd, page
        rnd = lambda n: (torch.randn((T, n * hd), generator=g) * sigma).to(BF16)
        self.q, self.k, self.v = rnd(hq), rnd(hk), rnd(hk)
        self.gq, self.gk = ((torch.rand(n * hd, generator=g) + 0.5).to(BF16) for n in (hq, hk))
        self.rot = hd if rot is None else rot
        self.inv_freq = 10000.0 ** (-torch.arange(0, self.rot, 2, dtype=torch.float64) / max(1, self.rot))
        self.axis = (torch.arange(self.rot // 2) % axes).to(torch.uint8) if axes else None
        self.pos = torch.randint(-5000, 100000, (axes, T) if axes else (T,), generator=g)
        self.pages = T // page + 3
        ids = torch.randperm(self.pages * page, generator=g)[:T]
        self.slots = ids.clone()
        pool = lambda n: torch.randint(0, 256, (self.pages, page, hk, n), generator=g, dtype=torch.uint8)
        self.codes, self.scales = [pool(hd // 2) for _ in range(2)], [pool(hd // 16) for _ in range(2)]
        self.dcodes, self.dscales = [lay(t, order) for t in self.codes], [lay(t, order).view(F8) for t in self.scales]

    def expect(self, norm, inter, eps=1e-6, mscale=1.0):
        out = {}
        for n, x, gamma in (("q", self.q, self.gq), ("k", self.k, self.gk)):
            x = x.double()
            if norm:
                x = R.norm(x, gamma.double(), eps, self.hd if norm == "headwise" else x.shape[1])
            if self.rot:
                x = turn(x, self.pos, self.inv_freq, self.axis, self.hd, inter, mscale=mscale)
            out[n] = x
        out["v"] = self.v.double()
        return out

    def call(self, norm, inter, **kw):
        c = lambda t: None if t is None else t.cuda()
        out = attn.qknorm_fwd_append_e2m1(c(self.q), c(self.k), c(self.v), c(self.gq) if norm else None, c(self.gk) if norm else None,
                                          c(self.pos) if self.rot else None, c(self.inv_freq) if self.rot else None, c(self.slots),
                                          *self.dcodes, *self.dscales, 1e-6, headwise=norm == "headwise", interleaved=inter,
                                          axis=c(self.axis) if self.rot else None, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, out, want, units):
        T, hd = self.T, self.hd
        q = want["q"].view(T, -1, hd)
        assert ((out.cpu().double().view(T, -1, hd) - q).abs() <= 2.0 ** -8 * q.abs() + OFF * q.abs().amax(-1, keepdim=True)).all()
        page, token = self.slots // self.page, self.slots % self.page
        ok = (self.slots >= 0) & (self.slots < self.pages * self.page)
        for side, n in enumerate("kv"):
            codes, scales = self.dcodes[side].cpu(), self.dscales[side].cpu().view(torch.uint8)
            E.check_written(want[n].view(T, self.hk, hd)[ok], codes[page[ok], token[ok]], scales[page[ok], token[ok]].view(F8), units[side],
                            OFF if n == "k" else 0.0)
            left = torch.ones((self.pages, self.page), dtype=torch.bool)
            left[page[ok], token[ok]] = False
            assert torch.equal(codes[left], self.codes[side][left]) and torch.equal(scales[left], self.scales[side][left])


def turn(x, pos, inv_freq, axis, hd, inter, inverse=False, mscale=1.0):
    """R.rotate with every pair at the positions of its axis."""
    if axis is None:
        return R.rotate(x, pos, inv_freq, hd, inter, inverse, mscale)[0]
    T = x.shape[0]
    x = x.reshape(T, -1, hd)
    y = x.clone()
    for i, f in enumerate(inv_freq.tolist()):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + len(inv_freq))
        n = int(axis[i])
        p = pos[n].double() if n < pos.shape[0] else torch.zeros(T, dtype=torch.float64)
        ang = p * f * (-1.0 if inverse else 1.0)
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        y[:, :, a] = (x[:, :, a] * c - x[:, :, b] * s) * mscale
        y[:, :, b] = (x[:, :, b] * c + x[:, :, a] * s) * mscale
    return y.reshape(T, -1)


@pytest.mark.parametrize("norm", [None, "layerwise", "headwise"])
@pytest.mark.parametrize("inter", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("T,hq,hk,hd,rot,page,order", [
    (1, 5, 1, 128, 128, 16, "hnd"), (37, 4, 2, 64, 32, 16, "nhd"), (700, 2, 1, 128, 64, 24, "hnd"), (65, 3, 3, 96, 96, 7, "thd"),
    (33, 2, 1, 80, 48, 16, "nhd"), (20, 2, 2, 16, 16, 16, "nhd"), (9, 1, 1, 256, 256, 16, "hnd"), (400, 8, 8, 32, 0, 1, "nhd"),
    (310, 16, 4, 208, 160, 5, "hnd"),
])
def test_append(libqknorm, T, hq, hk, hd, rot, page, order, inter, norm):
    a = Layer(T, hq, hk, hd, page, order, seed=T + hd, rot=rot)
    a.slots[T // 2] = -1                     # padded tokens: nothing is written for them
    a.slots[-1] = a.pages * page
    want = a.expect(norm, inter)
    units = (2.0 ** -6, 2.0 ** -7)
    out = a.call(norm, inter, k_scale=units[0], v_scale=units[1])
    vec = rot % (16 if inter else 32) == 0
    assert binding.last_variant() == ("append" if vec else "append_general")
    a.check(out, want, units)


def test_append_general_writes_what_the_vector_kernel_does(libqknorm, monkeypatch):
    one, two = Layer(50, 4, 2, 128, seed=3), Layer(50, 4, 2, 128, seed=3)
    one.call(None, False)
    monkeypatch.setenv("QKNORM_FORCE_VARIANT", "general")
    two.call(None, False)
    assert binding.last_variant() == "append_general"
    for x, y in zip(one.dcodes + one.dscales, two.dcodes + two.dscales):       # without a norm both round the same fp32 values ...
        same = (x.view(torch.uint8) == y.view(torch.uint8)).float().mean()
        assert same > 0.999                                                    # ... but for the order of a rotation's two products


@pytest.mark.parametrize("axes", [1, 2, 3, 8])
def test_append_with_several_axes(libqknorm, axes):
    a = Layer(45, 4, 2, 128, seed=axes, axes=axes)
    a.check(a.call("layerwise", False), a.expect("layerwise", False), (1.0, 1.0))


def test_ties_extremes_and_nan(libqknorm):
    """V goes in as it is: its blocks come out bit for bit as the definition has them."""
    a = Layer(64, 1, 1, 128, seed=5)
    x = torch.randn((64, 8, 16), generator=torch.Generator().manual_seed(6)).double()
    f = E.VALUES[:8].double()
    x[0, 0] = torch.cat((torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]), -torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]))) * 1.125
    x[1] = 0.0
    x[2] *= 1e-30                                    # scale rounds to zero
    x[3] *= 1e30                                     # saturates
    x[4, 2, 5], x[4, 3, 1], x[4, 4, 7] = float("nan"), float("inf"), -float("inf")
    x[5, 0] = f.repeat(2) * 448.0
    x[6] *= 2.0 ** -9
    for i in range(7, 64):                           # ties of every scale: a multiple of half a code times an E4M3 value
        sc = torch.tensor([0x20 + i], dtype=torch.uint8).view(F8).double()
        x[i, 0] = torch.tensor([6.0] + [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] * 2 + [4.0]) * sc
    a.v = x.reshape(64, 128).to(BF16)
    a.call(None, False)
    v = a.v.double().view(64, 1, 128)
    codes, scales = E.quantise(v.nan_to_num(posinf=1e38, neginf=-1e38, nan=0.0), 1.0)
    page, token = a.slots // 16, a.slots % 16
    got_c, got_s = E.codes_of(a.dcodes[1].cpu()[page, token]), a.dscales[1].cpu().view(torch.uint8)[page, token]
    nan = v.isnan().unflatten(-1, (-1, 16)).any(-1)
    assert ((got_s[nan] & 0x7F) == 0x7F).all()
    assert torch.equal(got_s[~nan], scales.view(torch.uint8)[~nan])
    keep = (~nan).repeat_interleave(16, -1)
    assert torch.equal(E.VALUES[got_c[keep]], E.VALUES[codes[keep]])


class Batch:
    """As tests/test_gpu_attn.py has it, over a 4-bit pool whose unused slots hold NaN."""

    def __init__(self, new, kv, hq, hk, hd, page=16, seed=0, order="hnd", guard=2, sigma=1.0, pad_cols=0, unit=(0.25, 0.5)):
        g = torch.Generator().manual_seed(seed)
        self.new, self.kv, self.hq, self.hk, self.hd, self.page, self.unit = list(new), list(kv), hq, hk, hd, page, unit
        need = [-(-max(n, 0) // page) for n in kv]
        self.pages, cols = sum(need) + 3, max(need + [1]) + pad_cols
        ids = torch.randperm(self.pages, generator=g).tolist()
        self.table = [[ids.pop() for _ in range(n)] + [10 ** 6] * (cols - n) for n in need]
        self.k, self.ks = E.random_pool(g, (self.pages, page, hk, hd), sigma, unit[0])
        self.v, self.vs = E.random_pool(g, (self.pages, page, hk, hd), 1.0, unit[1])
        used = torch.zeros((self.pages, page), dtype=torch.bool)
        for row, n in zip(self.table, kv):
            for j in range(max(n, 0)):
                used[row[j // page], j % page] = True
        for t in (self.ks, self.vs):
            t.view(torch.uint8)[~used] = 0x7F
        self.T = sum(new) + guard
        self.q = torch.randn((self.T, hq * hd), generator=g).to(BF16)
        self.q[sum(new):] = float("nan")
        self.starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        self.order = order
        self.dq = self.q.cuda()
        self.dtable = torch.tensor(self.table, dtype=torch.int32, device="cuda").view(len(new), cols)
        self.dlens = torch.tensor(kv, dtype=torch.int32, device="cuda")
        self.dstarts = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.place()

    def place(self):
        self.pools = [lay(t, self.order) for t in (self.k, self.v)] + [lay(t, self.order).view(F8) for t in (self.ks, self.vs)]

    def call(self, **kw):
        out = torch.full_like(self.dq, 7.0)
        lse = torch.full((self.T, self.hq), 7.0, dtype=torch.float32, device="cuda")
        kw.setdefault("max_q", max(self.new + [1]))
        kw.setdefault("max_kv", max(self.kv + [1]))
        attn.qknorm_attn_paged_e2m1(self.dq, *self.pools, self.dtable, self.dlens, self.dstarts, kw.pop("max_q"), kw.pop("max_kv"),
                                    k_scale=self.unit[0], v_scale=self.unit[1], out=out, lse=lse, **kw)
        torch.cuda.synchronize()
        assert binding.device_error_word() == 0
        return out.cpu(), lse.cpu()

    def reference(self, scale=None, causal=True, window=0, max_kv=None):
        scale = 1.0 / math.sqrt(self.hd) if scale is None else scale
        return R.attention(R.widen(self.q), E.widen(self.k, self.ks), E.widen(self.v, self.vs), self.table, self.kv, self.starts, self.hq,
                           scale=scale, causal=causal, window=window, k_scale=self.unit[0], v_scale=self.unit[1], max_kv=max_kv)

    def compare(self, out, lse, ref, fp16):
        n = self.starts[-1]
        got, z = out.double().numpy().reshape(self.T, self.hq, self.hd), lse.double().numpy()
        tol, tol_lse = R.attention_bounds(ref, self.hd, fp16)
        for r in range(n):
            bad = ~((np.abs(got[r] - ref["out"][r]) <= tol[r]) | (np.isnan(got[r]) & np.isnan(ref["out"][r])))
            assert not bad.any(), (f"row {r}: {int(bad.sum())} of {bad.size} off, first {np.argwhere(bad)[0]}: {got[r][bad][0]} for "
                                   f"{ref['out'][r][bad][0]} (tolerance {tol[r][bad][0]:.3g})")
            empty = np.isneginf(ref["lse"][r])
            assert (np.isneginf(z[r]) == empty).all(), f"row {r}: lse {z[r]} for {ref['lse'][r]}"
            some = ~empty & ~np.isnan(ref["lse"][r])
            assert (np.abs(z[r][some] - ref["lse"][r][some]) <= tol_lse[r][some]).all(), f"row {r}: lse {z[r]} for {ref['lse'][r]}"
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()     # rows of no sequence: not written

    def check(self, variant="attn_e2m1", **kw):
        ref = self.reference(**{k: v for k, v in kw.items() if k in ("scale", "causal", "window", "max_kv")})
        out, lse = self.call(**kw)
        assert binding.last_variant() == variant
        self.compare(out, lse, ref, variant == "attn_e2m1")
        return out, lse


@pytest.fixture(params=["tma", "cp.async"])
def copies(request, monkeypatch):
    """Both ways of bringing tiles in, whichever the sizes would choose; a layout that TMA cannot bring takes the other."""
    monkeypatch.setenv("QKNORM_E2M1_TMA", "1" if request.param == "tma" else "0")
    attn._workspace_e2m1.cache_clear()       # the two need different sizes
    yield
    attn._workspace_e2m1.cache_clear()


@pytest.mark.parametrize("order", ["hnd", "nhd"])
@pytest.mark.parametrize("hq,hk,hd", [(1, 1, 128), (1, 1, 64), (8, 1, 128), (5, 1, 64), (8, 8, 128), (7, 1, 96), (40, 8, 128), (6, 2, 32),
                                      (3, 1, 16), (16, 1, 128), (9, 1, 64), (32, 1, 128), (4, 2, 256), (12, 1, 208), (2, 1, 80), (2, 2, 112)])
def test_single_tokens(libqknorm, copies, hq, hk, hd, order):
    Batch([1, 1, 1, 1], [1, 130, 33, 128], hq, hk, hd, order=order, seed=hd).check()


@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 128, 256])
def test_pages_and_lengths(libqknorm, copies, page):
    Batch([1, 2, 1, 3, 1], [127, 129, 255, 257, 384], 4, 2, 64, page=page, seed=page).check()


@pytest.mark.parametrize("hq,hk,hd,new,kv", [
    (4, 2, 128, [16, 3, 1], [300, 129, 1]), (8, 1, 64, [7, 6, 4], [500, 16, 130]), (1, 1, 96, [50], [400]), (32, 1, 128, [2], [700]),
    (7, 1, 64, [9, 0, 2], [3000, 0, 5]), (3, 1, 256, [20, 11, 0], [2000, 11, 5]), (40, 8, 128, [5, 5], [1000, 5]), (2, 1, 160, [17], [40]),
])
def test_several_new_tokens(libqknorm, copies, hq, hk, hd, new, kv):
    Batch(new, kv, hq, hk, hd, seed=len(new)).check()


@pytest.mark.parametrize("hq,hk,hd,new,kv", [
    (5, 1, 128, [60, 3, 26], [60, 200, 27]), (8, 2, 64, [16, 17, 33], [300, 17, 129]), (3, 1, 96, [100, 1, 0], [256, 300, 9]), (1, 1, 128, [300], [300]),
    (2, 2, 16, [70], [500]), (128, 1, 64, [2, 1], [130, 140]),
])
def test_chunks(libqknorm, hq, hk, hd, new, kv):
    """More than 96 rows of a sequence and key head: over a widened cache."""
    Batch(new, kv, hq, hk, hd, seed=len(new)).check("attn_tc" if max(new) * hq // hk > 96 else "attn_e2m1")


@pytest.mark.parametrize("new,variant", [([1, 1, 1], "attn_e2m1"), ([9, 4, 2], "attn_e2m1"), ([80, 1, 33], "attn_tc")])
@pytest.mark.parametrize("window", [1, 31, 100, 1000])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(libqknorm, copies, causal, window, new, variant):
    Batch(new, [400, 257, 90], 4, 2, 128, seed=window).check(variant, causal=causal, window=window)


@pytest.mark.parametrize("new,kv,variant", [([3, 5], [1, 3], "attn_e2m1"), ([100, 4], [40, 0], "attn_tc"), ([1, 1], [0, 7], "attn_e2m1")])
def test_rows_that_see_nothing(libqknorm, copies, new, kv, variant):
    """More new tokens than keys: the first rows stand before key 0."""
    out, lse = Batch(new, kv, 2, 1, 64, seed=1).check(variant)


def test_long_rows_are_cut_and_joined(libqknorm, copies):
    b = Batch([1, 4], [20000, 5001], 8, 1, 128, seed=2)
    assert attn.attn_paged_e2m1_workspace(2, b.T, 4, 20000, 8, 1, 128) > 0
    out, lse = b.check()
    again, _ = b.call()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("hq,hk,hd,new,kv", [
    (8, 8, 64, [1] * 40, [3000 - 70 * i for i in range(40)]),             # many units, ragged, some without a key
    (16, 4, 128, [1, 3, 0, 2], [9000, 17, 40, 2500]),                     # units over one share, several in one
    (4, 1, 64, [1] * 300, [(37 * i) % 400 for i in range(300)]),          # more sequences than threads look for a share
    (6, 2, 256, [1, 2], [5000, 700]), (5, 1, 96, [1, 1], [6000, 1500]), (24, 2, 64, [4], [70000]),
])
def test_shares(libqknorm, copies, hq, hk, hd, new, kv):
    """Units cut wherever equal shares end, in every way that they can be."""
    Batch(new, kv, hq, hk, hd, seed=len(kv), pad_cols=3).check(max_kv=max(kv) + 5000)


def test_bounds_smaller_than_the_batch(libqknorm):
    Batch([1, 1], [300, 150], 4, 1, 128, seed=3).check(max_kv=200)
    b = Batch([4, 2], [90, 50], 4, 1, 128, seed=4)
    out, _ = b.call(max_q=3)
    assert (out[3] == 7.0).all() and not (out[2] == 7.0).all()


def test_bad_pages_read_as_zeros(libqknorm, copies):
    b = Batch([1, 2], [100, 70], 8, 2, 128, seed=5)
    for row, j, e in ((0, 1, -1), (0, 3, 2 ** 31 - 1), (1, 2, b.pages)):
        b.table[row][j] = e
    b.dtable = torch.tensor(b.table, dtype=torch.int32, device="cuda")
    b.check()
    c = Batch([70, 2], [100, 70], 8, 2, 128, seed=5)
    for row, j, e in ((0, 1, -1), (0, 3, 2 ** 31 - 1), (1, 2, c.pages)):
        c.table[row][j] = e
    c.dtable = torch.tensor(c.table, dtype=torch.int32, device="cuda")
    c.check("attn_tc")


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_values_not_seen_do_not_matter(libqknorm, copies, hd):
    """NaN in K and V blocks that only some rows of a tile see: those rows have it, the others are as they were."""
    b = Batch([6], [200], 2, 1, hd, seed=6)
    page, token = b.table[0][197 // 16], 197 % 16                # seen by rows 3, 4, 5
    b.vs.view(torch.uint8)[page, token, 0, hd // 16 - 1] = 0xFF
    page, token = b.table[0][198 // 16], 198 % 16                # seen by rows 4, 5
    b.ks.view(torch.uint8)[page, token, 0, 0] = 0x7F
    b.place()
    out, lse = b.call()
    ref = b.reference()
    got = out.double().numpy().reshape(b.T, 2, hd)
    tol, _ = R.attention_bounds(ref, hd, True)
    for r in range(3):
        assert (np.abs(got[r] - ref["out"][r]) <= tol[r]).all()
    assert np.isnan(got[3][:, hd - 16:]).all() and (np.abs(got[3] - ref["out"][3]) <= tol[3])[:, :hd - 16].all()
    assert np.isnan(got[4:6]).all()


def test_extreme_queries_and_scales(libqknorm):
    b = Batch([1, 1, 1, 1], [64, 64, 64, 64], 4, 2, 128, seed=7)
    b.q[0] *= 2.0 ** 100                     # one key takes all
    b.q[1] *= 2.0 ** -100
    b.q[2] *= 2.0 ** -130                    # subnormal bf16 values
    b.dq = b.q.cuda()
    b.check(scale=2.0 ** -3)
    b.check(scale=1e-38)


def test_small_weights_are_kept(libqknorm, copies):
    """One key far above the rest: 30000 others share 2^-20 of its weight each."""
    b = Batch([1], [30000], 1, 1, 64, seed=8)
    b.k[:], b.ks.view(torch.uint8)[:] = 0, 0x38
    first = b.table[0][0]
    b.k[first, 0, 0, 0] = 0x04               # code 4 of element 0: a key of 2
    b.q[:] = 0
    b.q[0, 0] = 20 * math.log(2) / (2 * 0.25) * math.sqrt(64)
    b.dq = b.q.cuda()
    b.place()
    b.check()


def test_strided_rows_and_other_streams(libqknorm):
    b = Batch([1, 3], [77, 300], 5, 1, 128, seed=9)
    ref = b.reference()
    wide = torch.full((b.T, 3 * b.hq * b.hd + 1), float("nan"), dtype=BF16, device="cuda")
    wide[:, 1:1 + b.hq * b.hd] = b.dq        # rows at odd addresses
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.full((b.T, 2 * b.hq * b.hd), 7.0, dtype=BF16, device="cuda")[:, :b.hq * b.hd]
    lse = torch.full((b.T, b.hq), 7.0, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    attn.qknorm_attn_paged_e2m1(wide[:, 1:1 + b.hq * b.hd], *b.pools, b.dtable, b.dlens, b.dstarts, 3, 300, k_scale=b.unit[0], v_scale=b.unit[1],
                                out=out, lse=lse, stream=side)
    torch.cuda.synchronize()
    b.compare(out.cpu(), lse.cpu(), ref, True)


@pytest.mark.parametrize("skew", [0, 16])
@pytest.mark.parametrize("new,kv", [([60, 1], [300, 77]), ([1, 1], [3000, 50])])
def test_workspaces_anywhere(libqknorm, new, kv, skew):
    """A workspace of exactly the bytes asked for, at any multiple of 16: what lies around it stays."""
    b = Batch(new, kv, 8, 2, 128, seed=12)
    n = attn.attn_paged_e2m1_workspace(2, b.T, max(new), max(kv), 8, 2, 128)
    around = torch.full((n + 64,), 77, dtype=torch.uint8, device="cuda")
    b.check("attn_tc" if max(new) > 24 else "attn_e2m1", workspace=around[skew:skew + n]) if n else b.check()
    assert (around[:skew] == 77).all() and (around[skew + n:] == 77).all()


@pytest.mark.parametrize("new,kv", [([1, 1], [700, 900]), ([70, 2], [700, 300])])
def test_capture_and_replay(libqknorm, copies, new, kv):
    b = Batch(new, kv, 8, 2, 128, seed=10)
    want, _ = b.call()
    out = torch.zeros_like(b.dq)
    ws = torch.empty(max(16, attn.attn_paged_e2m1_workspace(2, b.T, max(new), max(kv), 8, 2, 128)), dtype=torch.uint8, device="cuda")
    args = (b.dq, *b.pools, b.dtable, b.dlens, b.dstarts, max(new), max(kv))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.qknorm_attn_paged_e2m1(*args, k_scale=b.unit[0], v_scale=b.unit[1], out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        graph.replay()
    torch.cuda.synchronize()
    n = b.starts[-1]
    assert torch.equal(out.cpu()[:n].view(torch.int16), want[:n].view(torch.int16))


def test_append_then_attend(libqknorm):
    """A prompt and two decode steps through both operators, every row against attention over what the cache then holds."""
    T, hq, hk, hd, page = 40, 8, 2, 128, 16
    g = torch.Generator().manual_seed(11)
    pages = 4
    codes = [torch.zeros((pages, hk, page, hd // 2), dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in range(2)]
    scales = [torch.zeros((pages, hk, page, hd // 16), dtype=torch.uint8, device="cuda").view(F8).transpose(1, 2) for _ in range(2)]
    inv_freq, _ = attn.rope_frequencies(hd)
    gq, gk = ((torch.rand(n * hd, generator=g) + 0.5).to(BF16).cuda() for n in (hq, hk))
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device="cuda")
    unit = (2.0 ** -7, 2.0 ** -7)
    done = 0
    for n in (T, 1, 1):
        q, k, v = (torch.randn((n, m * hd), generator=g).to(BF16).cuda() for m in (hq, hk, hk))
        pos = torch.arange(done, done + n, device="cuda")
        slots = table[0].long()[pos // page] * page + pos % page
        qn = attn.qknorm_fwd_append_e2m1(q, k, v, gq, gk, pos, inv_freq, slots, *codes, *scales, 1e-6, k_scale=unit[0], v_scale=unit[1])
        done += n
        lens, starts = torch.tensor([done], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
        lse = torch.empty((n, hq), device="cuda")
        out = attn.qknorm_attn_paged_e2m1(qn, *codes, *scales, table, lens, starts, n, 64, k_scale=unit[0], v_scale=unit[1], lse=lse)
        torch.cuda.synchronize()
        kp, vp = (E.widen(codes[i].cpu().contiguous(), scales[i].cpu().view(torch.uint8).contiguous()) for i in range(2))
        ref = R.attention(R.widen(qn), kp, vp, table.tolist(), [done], [0, n], hq, scale=1 / math.sqrt(hd), k_scale=unit[0], v_scale=unit[1])
        tol, tol_lse = R.attention_bounds(ref, hd, n == 1)
        assert (np.abs(out.cpu().double().numpy().reshape(n, hq, hd) - ref["out"]) <= tol).all()
        assert (np.abs(lse.cpu().double().numpy() - ref["lse"]) <= tol_lse).all()


@pytest.mark.parametrize("new", [[1, 2], [60, 2]])
def test_no_keys_to_look_at(libqknorm, copies, new):
    """Bounds of 0 keys, tables without columns, a pool without pages: zeros (a page that is none reads as zeros)."""
    b = Batch(new, [50, 40], 4, 2, 64, seed=13)
    n = b.starts[-1]
    out, lse = b.call(max_kv=0)
    assert (out[:n] == 0).all() and torch.isneginf(lse[:n]).all() and (out[n:] == 7.0).all()
    b.dtable = b.dtable[:, :0]
    out, lse = b.call()
    assert (out[:n] == 0).all() and torch.isneginf(lse[:n]).all()
    c = Batch(new, [50, 40], 4, 2, 64, seed=13)
    c.pools = [t[:0] for t in c.pools]
    out, lse = c.call()
    seen = torch.tensor([max(0, L - m + i + 1) for m, L in zip(new, [50, 40]) for i in range(m)]).double()
    assert (out[:n] == 0).all() and ((lse[:n].double() - torch.log(seen)[:, None]).abs()[seen > 0] < 1e-5).all()


@pytest.mark.parametrize("hd", [64, 96, 128, 256])
def test_many_short_sequences(libqknorm, copies, hd):
    """More units than SMs, each taken whole."""
    Batch([1] * 160, [(53 * i) % 290 for i in range(160)], 2, 1, hd, seed=21).check()


def test_more_query_heads_than_the_widened_path_takes(libqknorm):
    Batch([1, 2], [300, 40], 130, 1, 64, seed=14).check()
    Batch([3], [500], 300, 2, 128, seed=15).check()


@pytest.mark.parametrize("hq,hk", [(8, 8), (16, 8), (4, 1)])
def test_results_at_odd_addresses(libqknorm, copies, hq, hk):
    b = Batch([1, 3], [77, 2000], hq, hk, 128, seed=16)
    ref = b.reference()
    wide = torch.full((b.T, hq * 128 + 3), 7.0, dtype=BF16, device="cuda")
    out, lse = wide[:, 1:1 + hq * 128], torch.full((b.T, hq), 7.0, device="cuda")
    attn.qknorm_attn_paged_e2m1(b.dq, *b.pools, b.dtable, b.dlens, b.dstarts, 3, 2000, k_scale=b.unit[0], v_scale=b.unit[1], out=out, lse=lse)
    torch.cuda.synchronize()
    b.compare(out.cpu(), lse.cpu(), ref, True)
    assert (wide[:, 0] == 7.0).all() and (wide[:, 1 + hq * 128:] == 7.0).all()


def test_two_streams_at_once(libqknorm, copies):
    """Calls that run beside one another, each with a workspace of its own, give what they give alone."""
    b, c = Batch([1] * 8, [2500] * 8, 8, 8, 128, seed=17), Batch([1] * 3, [4000, 50, 3000], 16, 2, 64, seed=18)
    want = [x.call()[0] for x in (b, c)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(x.dq) for _ in range(6)] for x in (b, c)]
    torch.cuda.synchronize()
    for i in range(6):
        for x, s, o in zip((b, c), streams, outs):
            attn.qknorm_attn_paged_e2m1(x.dq, *x.pools, x.dtable, x.dlens, x.dstarts, 1, max(x.kv), k_scale=x.unit[0], v_scale=x.unit[1], out=o[i], stream=s)
    torch.cuda.synchronize()
    for x, w, o in zip((b, c), want, outs):
        n = x.starts[-1]
        for y in o:
            assert torch.equal(y.cpu()[:n].view(torch.int16), w[:n].view(torch.int16))


def test_lengths_grow_between_replays(libqknorm, copies):
    b = Batch([1, 1], [700, 3000], 8, 4, 128, seed=19)
    out = torch.zeros_like(b.dq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.qknorm_attn_paged_e2m1(b.dq, *b.pools, b.dtable, b.dlens, b.dstarts, 1, 3000, k_scale=b.unit[0], v_scale=b.unit[1], out=out)
    for lens in ([1, 1], [0, 2999], [700, 3000], [33, 128]):
        b.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        want, _ = b.call(max_kv=3000)
        assert torch.equal(out.cpu()[:2].view(torch.int16), want[:2].view(torch.int16))


def test_python_refusals(libqknorm):
    b = Batch([1], [20], 2, 1, 64, seed=20)
    k, v, ks, vs = b.pools
    bad = [(k[..., :16], v, ks, vs), (k, v, ks[..., :2], vs), (k.view(torch.int8), v, ks, vs), (k, v, ks.view(torch.int8), vs), (k, v.cpu(), ks, vs),
           (k, v, ks, None), (k.transpose(2, 3), v.transpose(2, 3), ks, vs), (k[:1], v, ks, vs), (k, v, ks.view(torch.uint8), vs), (k[0], v[0], ks[0], vs[0])]
    for pools in bad:
        with pytest.raises(binding.QKNormError):
            attn.qknorm_attn_paged_e2m1(b.dq, *pools, b.dtable, b.dlens, b.dstarts, 1, 20)
    x = torch.zeros((2, 64), dtype=BF16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    for pools in bad:
        with pytest.raises(binding.QKNormError):
            attn.qknorm_fwd_append_e2m1(None, x, x, None, None, None, None, slots, *pools, 1e-6)
    four = torch.zeros((1, 16, 1, 32), dtype=torch.uint8, device="cuda").view(torch.float4_e2m1fn_x2)     # torch's own type for two codes
    byte = torch.zeros((1, 16, 1, 4), dtype=torch.uint8, device="cuda")
    x[0], x[1] = 3.0, -1.5
    attn.qknorm_fwd_append_e2m1(None, x, x, None, None, None, None, torch.tensor([4, 7], device="cuda"), four, torch.zeros_like(four.view(torch.uint8)).view(four.dtype),
                                byte, torch.zeros_like(byte), 1e-6)
    torch.cuda.synchronize()
    assert (four.view(torch.uint8)[0, 4] == 0x77).all() and (four.view(torch.uint8)[0, 7] == 0xFF).all() and (byte[0, [4, 7]] != 0).all()
