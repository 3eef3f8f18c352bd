"""Attention over a paged cache against its 64-bit definition (tests/attn_reference.py says how the bounds come about)."""
import math

import numpy as np
import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests import attn_reference as R
from tests.attn_reference import BF16, F8

pytestmark = pytest.mark.gpu


class Batch:
    """A seeded batch: lists of new tokens and keys per sequence, a shuffled page pool (unused slots hold NaN), guard rows."""

    def __init__(self, new, kv, hq, hk, hd, page=16, dtype=BF16, seed=0, order="nhd", guard=2, sigma=1.0, pad_cols=0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.kv, self.hq, self.hk, self.hd, self.page, self.dtype = list(new), list(kv), hq, hk, hd, page, dtype
        need = [-(-max(n, 0) // page) for n in kv]
        self.pages, cols = sum(need) + 3, max(need + [1]) + pad_cols
        ids = torch.randperm(self.pages, generator=g).tolist()
        self.table = [[ids.pop() for _ in range(n)] + [10 ** 6] * (cols - n) for n in need]
        self.ks, self.vs = (0.25, 0.5) if dtype is F8 else (1.0, 1.0)
        self.k = (torch.randn((self.pages, page, hk, hd), generator=g) * sigma / self.ks).to(dtype)
        self.v = (torch.randn((self.pages, page, hk, hd), generator=g) / self.vs).to(dtype)
        used = torch.zeros((self.pages, page), dtype=torch.bool)
        for row, n in zip(self.table, kv):
            for j in range(max(n, 0)):
                used[row[j // page], j % page] = True
        nan = torch.tensor([0x7F], dtype=torch.uint8).view(F8)[0] if dtype is F8 else torch.tensor(float("nan"), dtype=BF16)
        for t in (self.k, self.v):
            raw = t.view(torch.uint8 if dtype is F8 else torch.int16)
            raw[~used] = nan.view(raw.dtype)
        self.T = sum(new) + guard
        self.q = torch.randn((self.T, hq * hd), generator=g).to(BF16)
        self.q[sum(new):] = float("nan")          # rows of no sequence: not read
        self.starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        perm = {"nhd": (0, 1, 2, 3), "hnd": (0, 2, 1, 3), "thd": (1, 0, 2, 3)}[order]
        inv = [perm.index(i) for i in range(4)]
        raw = torch.uint8 if dtype is F8 else torch.int16
        place = lambda t: t.view(raw).permute(perm).contiguous().cuda().permute(inv).view(dtype)
        self.dk, self.dv = place(self.k), place(self.v)
        self.dq = self.q.cuda()
        self.dtable = torch.tensor(self.table, dtype=torch.int32, device="cuda").view(len(new), cols)
        self.dlens = torch.tensor(kv, dtype=torch.int32, device="cuda")
        self.dstarts = torch.tensor(self.starts, dtype=torch.int32, device="cuda")

    def call(self, **kw):
        out = torch.full_like(self.dq, 7.0)
        lse = torch.full((self.T, self.hq), 7.0, dtype=torch.float32, device="cuda")
        kw.setdefault("max_q", max(self.new + [1]))
        kw.setdefault("max_kv", max(self.kv + [1]))
        attn.qknorm_attn_paged(self.dq, self.dk, self.dv, self.dtable, self.dlens, self.dstarts, kw.pop("max_q"), kw.pop("max_kv"),
                               k_scale=self.ks, v_scale=self.vs, out=out, lse=lse, **kw)
        torch.cuda.synchronize()
        assert binding.device_error_word() == 0
        return out.cpu(), lse.cpu()

    def reference(self, scale=None, causal=True, window=0, max_kv=None):
        scale = 1.0 / math.sqrt(self.hd) if scale is None else scale
        return R.attention(R.widen(self.q), R.widen(self.k), R.widen(self.v), self.table, self.kv, self.starts, self.hq, scale=scale,
                           causal=causal, window=window, k_scale=self.ks, v_scale=self.vs, max_kv=max_kv)

    def compare(self, out, lse, ref, rows=None):
        n = self.starts[-1]
        rows = range(n) if rows is None else rows
        got, z = out.double().numpy().reshape(self.T, self.hq, self.hd), lse.double().numpy()
        tol, tol_lse = R.attention_bounds(ref, self.hd, self.dtype is F8)
        for r in rows:
            bad = ~(np.abs(got[r] - ref["out"][r]) <= tol[r])
            assert not bad.any(), (f"row {r}: {int(bad.sum())} of {bad.size} off, first {np.argwhere(bad)[0]}: {got[r][bad][0]} for "
                                   f"{ref['out'][r][bad][0]} (tolerance {tol[r][bad][0]:.3g})")
            empty = np.isneginf(ref["lse"][r])
            assert (np.isneginf(z[r]) == empty).all(), f"row {r}: lse {z[r]} for {ref['lse'][r]}"
            assert (np.abs(z[r][~empty] - ref["lse"][r][~empty]) <= tol_lse[r][~empty]).all(), f"row {r}: lse {z[r]} for {ref['lse'][r]}"
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()     # rows of no sequence: not written

    def check(self, variant=None, **kw):
        ref = self.reference(**{k: v for k, v in kw.items() if k in ("scale", "causal", "window", "max_kv")})
        out, lse = self.call(**kw)
        if variant:
            assert binding.last_variant() == variant
        self.compare(out, lse, ref)


BOTH = pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])


@BOTH
@pytest.mark.parametrize("hq,hk,hd", [(1, 1, 128), (1, 1, 64), (8, 1, 128), (5, 1, 64), (8, 8, 128), (7, 1, 96), (40, 8, 128)])
def test_single_tokens(libqknorm, hq, hk, hd, dtype):
    Batch([1, 1, 1, 1], [1, 130, 33, 128], hq, hk, hd, dtype=dtype).check("attn_tc")


@BOTH
@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 128, 256])
def test_pages_and_lengths(libqknorm, page, dtype):
    Batch([1, 2, 1, 3, 1], [127, 129, 255, 257, 384], 4, 2, 64, page=page, dtype=dtype, seed=page).check("attn_tc")


@BOTH
@pytest.mark.parametrize("hq,hk,hd,new,kv", [
    (1, 1, 128, [128], [128]), (1, 1, 128, [129], [129]), (1, 1, 64, [300], [300]), (5, 1, 128, [60, 3, 26], [60, 200, 27]),
    (8, 2, 64, [16, 17, 33], [300, 17, 129]), (3, 1, 96, [100], [256]), (128, 1, 64, [2, 1], [130, 140]), (2, 2, 128, [257, 1], [500, 129]),
])
def test_chunks(libqknorm, hq, hk, hd, new, kv, dtype):
    Batch(new, kv, hq, hk, hd, dtype=dtype, seed=len(new)).check("attn_tc")


@BOTH
@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("hq,hk,hd,new,kv", [
    (4, 2, 128, [20, 3, 1], [300, 129, 1]), (8, 1, 64, [9, 16, 4], [500, 16, 130]), (1, 1, 96, [100], [400]), (64, 1, 128, [2], [700]),
    (7, 1, 64, [18], [3000]), (3, 1, 128, [42, 11, 0], [2000, 11, 5]),
])
def test_short_chunks(libqknorm, hq, hk, hd, new, kv, page, dtype):
    """33 to 128 rows per sequence and key head: one query tile, key tiles alternating between the warpgroups."""
    assert 32 < max(new) * hq // hk <= 128
    b = Batch(new, kv, hq, hk, hd, page=page, dtype=dtype, seed=hd)
    b.check("attn_tc")
    b.check("attn_tc", causal=False)
    b.check("attn_tc", window=100)


@BOTH
@pytest.mark.parametrize("rows", [1, 5, 31, 32])
def test_up_to_32_rows(libqknorm, rows, dtype):
    """The four-quarter form at its edges: keys that end in each quarter of a tile."""
    for kv in (31, 32, 33, 64, 65, 96, 97, 128, 129, 225):
        Batch([rows], [max(kv, 1)], 2, 2, 64, dtype=dtype, seed=kv).check("attn_tc")
    Batch([rows, 1, rows // 2], [300, 260, 40], 2, 2, 128, page=24, dtype=dtype).check("attn_tc", window=50)


@BOTH
@pytest.mark.parametrize("window", [1, 5, 64, 128, 200])
def test_windows(libqknorm, window, dtype):
    b = Batch([1, 40, 150], [400, 300, 150], 4, 2, 64, dtype=dtype)
    b.check("attn_tc", window=window)
    Batch([1, 1], [300, 77], 4, 2, 64, dtype=dtype).check("attn_tc", window=window)


@BOTH
@pytest.mark.parametrize("one", [True, False])
def test_not_causal(libqknorm, one, dtype):
    new = [5, 2] if one else [140, 3]
    Batch(new, [130, 259], 2, 1, 128, dtype=dtype).check("attn_tc", causal=False)
    Batch(new, [130, 259], 2, 1, 128, dtype=dtype).check("attn_tc", causal=False, window=30)


@BOTH
def test_rows_without_keys(libqknorm, dtype):
    """Fewer keys than new tokens (the first rows stand before the first key), no keys at all, an empty sequence between."""
    Batch([6, 0, 3, 2], [4, 40, 0, 1], 4, 2, 64, dtype=dtype).check("attn_tc")
    Batch([200, 0, 140], [70, 0, 0], 4, 2, 64, dtype=dtype).check("attn_tc")
    Batch([1], [0], 4, 2, 64, dtype=dtype).check("attn_tc")


@BOTH
def test_split_keys(libqknorm, dtype):
    """Long contexts, few rows: parts joined by the second launch; ragged, so that some sequences have fewer parts."""
    b = Batch([1, 1, 1], [5000, 128, 1], 4, 2, 64, dtype=dtype)
    n0 = binding.launch_count()
    b.check("attn_tc")
    assert binding.launch_count() - n0 == 2
    Batch([3, 90], [4000, 3000], 2, 1, 128, dtype=dtype).check("attn_tc")
    Batch([2, 5], [3000, 3], 2, 1, 128, dtype=dtype).check("attn_tc", window=1000)
    Batch([2, 5], [3000, 0], 2, 1, 128, dtype=dtype).check("attn_tc", max_kv=4000)


@BOTH
def test_large_scores_and_growing_maxima(libqknorm, dtype):
    """Scores in the hundreds, the maximum rising from tile to tile: the accumulators have to be rescaled."""
    for new, hd in (([1, 1], 64), ([150], 128)):
        b = Batch(new, [700] * len(new), 2, 1, hd, dtype=dtype, sigma=1.0)
        grow = torch.linspace(0.05, 4.0, 700)
        for row in b.table:
            for j in range(700):
                b.k[row[j // 16], j % 16] = (b.k[row[j // 16], j % 16].float() * grow[j]).to(dtype)
        b.dk.copy_(b.k.cuda())
        b.check("attn_tc", scale=0.5)


@BOTH
@pytest.mark.parametrize("order", ["hnd", "thd"])
def test_other_orders_of_the_pool(libqknorm, order, dtype):
    Batch([1, 70], [200, 150], 4, 2, 128, dtype=dtype, order=order).check("attn_tc")


@BOTH
@pytest.mark.parametrize("hq,hk,hd", [(2, 1, 36), (2, 1, 256), (3, 1, 512), (1, 1, 1), (200, 1, 64), (2, 1, 7)])
def test_general_kernel(libqknorm, hq, hk, hd, dtype):
    Batch([1, 9], [50, 20], hq, hk, hd, page=5, dtype=dtype).check("attn_general")
    Batch([3, 4], [2, 33], hq, hk, hd, page=5, dtype=dtype).check("attn_general", window=7)


@BOTH
def test_unaligned_rows_take_the_general_kernel(libqknorm, dtype):
    b = Batch([1, 9], [50, 20], 2, 1, 64, dtype=dtype)
    wide = torch.zeros((b.T, 2 * 64 + 1), dtype=BF16, device="cuda")
    wide[:, 1:] = b.dq
    b.dq = wide[:, 1:]
    ref = b.reference()
    out = torch.full((b.T, 130), 7.0, dtype=BF16, device="cuda")[:, 1:129]
    lse = torch.full((b.T, 2), 7.0, device="cuda")
    attn.qknorm_attn_paged(b.dq, b.dk, b.dv, b.dtable, b.dlens, b.dstarts, 9, 50, k_scale=b.ks, v_scale=b.vs, out=out, lse=lse)
    torch.cuda.synchronize()
    assert binding.last_variant() == "attn_general"
    b.compare(out.cpu().contiguous(), lse.cpu(), ref)


@BOTH
@pytest.mark.parametrize("new,kv,kw", [([40], [40], {}), ([3, 2], [200, 90], {}), ([150], [150], dict(window=20)), ([1], [300], dict(window=9)),
                                       ([2, 2], [2500, 2500], {}), ([20], [300], {}), ([25], [25], dict(window=3)), ([2, 2], [2500, 2500], dict(window=140))])
def test_unseen_values_do_not_matter(libqknorm, new, kv, kw, dtype):
    """NaN and infinities in K and V at keys that the rows checked do not see -- later tokens of the chunk, keys that left the
    window -- inside the same tile."""
    b = Batch(new, kv, 4, 2, 64, dtype=dtype)
    rows, poison = [], float("nan") if dtype is F8 else float("inf")
    k, v = b.k.clone(), b.v.clone()
    for s, row in enumerate(b.table):
        last = kv[s] - 1                                        # seen by the last new token only (if it is not its own)
        places = [last] if new[s] > 1 else []
        if kw.get("window"):
            places += [kv[s] - new[s] - kw["window"]] if kv[s] > new[s] + kw["window"] else [0]
        for j in places:
            for t in (b.k, b.v):
                t[row[j // b.page], j % b.page] = poison
        rows += [r for r in range(b.starts[s], b.starts[s + 1])
                 if not any(R.sees(kv[s] - new[s] + r - b.starts[s], kv[s], True, kw.get("window", 0))[j] for j in places)]
    b.dk.copy_(b.k.cuda())
    b.dv.copy_(b.v.cuda())
    out, lse = b.call(**kw)
    b.k, b.v = k, v                                             # the rows' own result never involves those keys
    assert rows
    b.compare(out, lse, b.reference(**kw), rows)


@BOTH
def test_seen_nan_reaches_the_row(libqknorm, dtype):
    b = Batch([1, 1], [200, 200], 2, 1, 64, dtype=dtype)
    b.v[b.table[0][5], 3, 0, 11] = float("nan")
    b.k[b.table[1][5], 3, 0, 11] = float("nan")
    b.dk.copy_(b.k.cuda())
    b.dv.copy_(b.v.cuda())
    out, lse = b.call()
    o = out[:2].view(2, 2, 64)
    assert torch.isnan(o[0, :, 11]).all() and torch.isfinite(o[0, :, :11]).all() and torch.isfinite(lse[0]).all()
    assert torch.isnan(o[1]).all() and torch.isnan(lse[1]).all()


@BOTH
def test_bad_table_entries_are_pages_of_zeros(libqknorm, dtype):
    b = Batch([1, 40], [100, 90], 4, 2, 64, dtype=dtype)
    for s, col, e in ((0, 2, -1), (1, 0, b.pages), (1, 3, 2 ** 31 - 1)):
        b.table[s][col] = e
        b.dtable[s, col] = e
    b.check("attn_tc")


def test_lengths_beyond_their_bounds(libqknorm):
    """kv_lens past the table or max_kv, more new tokens than max_q, q_starts outside the rows: nothing out of the buffers."""
    b = Batch([1, 4, 2], [100, 60, 40], 4, 2, 64)
    ref = b.reference(max_kv=48)
    out, lse = b.call(max_kv=48)
    b.compare(out, lse, ref)
    out, lse = b.call(max_q=2)
    keep = [0, 1, 2, 5, 6]
    b.compare(out, lse, b.reference(), keep)
    assert (out[3:5] == 7.0).all() and (lse[3:5] == 7.0).all()
    b.dlens[1] = -5
    b.dstarts.copy_(torch.tensor([0, 1, 5, 10 ** 9], dtype=torch.int32))
    out, lse = b.call(max_q=4)
    assert (out[1:5] == 0).all() and torch.isneginf(lse[1:5]).all()
    b.dstarts.copy_(torch.tensor([5, 1, -7, 2], dtype=torch.int32))
    b.dlens[1] = 60
    b.call(max_q=4)


def test_workspace_is_checked_and_shared_pools_are_safe(libqknorm):
    b = Batch([1, 1], [4000, 3000], 4, 2, 64)
    need = attn.attn_paged_workspace(2, b.T, 1, 4000, 4, 2, 64)
    assert need > 0
    with pytest.raises(binding.QKNormError) as e:
        b.call(workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == binding.QKNORM_ERR_SCRATCH
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN everywhere
    out, lse = b.call(workspace=ws[:need])
    b.compare(out, lse, b.reference())
    assert (ws[need:] == 0xFF).all()


def test_same_bits_every_time(libqknorm):
    b = Batch([3, 70], [4000, 300], 8, 2, 128)
    first = b.call()
    for _ in range(5):
        again = b.call()
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16))
        assert torch.equal(first[1].view(torch.int32), again[1].view(torch.int32))


def test_refusals(libqknorm):
    b = Batch([2, 1], [50, 20], 4, 2, 64)
    go = lambda q=b.dq, k=b.dk, v=b.dv, t=b.dtable, n=b.dlens, s=b.dstarts, **kw: attn.qknorm_attn_paged(q, k, v, t, n, s, 2, 50, **kw)
    out = torch.empty_like(b.dq)
    bad = [
        lambda: go(q=b.dq.float()), lambda: go(q=b.dq[:, :100]), lambda: go(q=b.dq[:, ::2]), lambda: go(k=b.dk.half()),
        lambda: go(v=b.dv[:-1]), lambda: go(t=b.dtable.long()), lambda: go(t=b.dtable[:1]), lambda: go(n=b.dlens.long()),
        lambda: go(s=b.dstarts[:2]), lambda: go(out=b.dq), lambda: go(out=out[:1]), lambda: go(lse=torch.empty((1, 4), device="cuda")),
        lambda: go(scale=0.0), lambda: go(window=-1), lambda: go(k=b.k, v=b.v), lambda: go(q=b.dq[:, :192]),
    ]
    n0 = binding.launch_count()
    for i, f in enumerate(bad):
        with pytest.raises((binding.QKNormError,)):
            f()
            pytest.fail(f"call {i} was accepted")
    assert binding.launch_count() == n0


def test_captured_and_replayed_while_lengths_grow(libqknorm):
    """One graph of a decode step, replayed as the sequences grow: lengths, tables and queries are read when it runs."""
    b = Batch([1, 1, 1], [600, 40, 10], 4, 2, 64, pad_cols=2)
    out, lse = torch.full_like(b.dq, 7.0), torch.full((b.T, 4), 7.0, device="cuda")
    ws = torch.empty(max(16, attn.attn_paged_workspace(3, b.T, 1, 608, 4, 2, 64)), dtype=torch.uint8, device="cuda")
    go = lambda: attn.qknorm_attn_paged(b.dq, b.dk, b.dv, b.dtable, b.dlens, b.dstarts, 1, 608, out=out, lse=lse, workspace=ws)
    b.dlens.copy_(torch.tensor([500, 3, 1], dtype=torch.int32))
    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for kv in ([500, 3, 1], [600, 40, 10], [129, 16, 0]):
        b.kv = kv
        b.dlens.copy_(torch.tensor(kv, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        b.compare(out.cpu(), lse.cpu(), b.reference())


def test_two_streams_at_once(libqknorm):
    a, b = Batch([1] * 4, [3000] * 4, 8, 2, 128, seed=1), Batch([200], [900], 4, 2, 64, seed=2)
    want = [a.call(), b.call()]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = []
        for x, s, mq, mk in ((a, s1, 1, 3000), (b, s2, 200, 900)):
            with torch.cuda.stream(s):
                got.append(attn.qknorm_attn_paged(x.dq, x.dk, x.dv, x.dtable, x.dlens, x.dstarts, mq, mk))
        torch.cuda.synchronize()
        for x, g, w in zip((a, b), got, want):
            n = x.starts[-1]
            assert torch.equal(g.cpu()[:n], w[0][:n])


def test_stream_argument(libqknorm):
    b = Batch([1, 1], [4000, 3000], 4, 2, 64)
    want = b.call()[0][:2]
    s = torch.cuda.Stream()
    for arg in (s, s.cuda_stream):
        got = attn.qknorm_attn_paged(b.dq, b.dk, b.dv, b.dtable, b.dlens, b.dstarts, 1, 4000, stream=arg)
        s.synchronize()
        assert torch.equal(got.cpu()[:2], want)


@BOTH
def test_append_then_attend(libqknorm, dtype):
    """A layer as it is used: a prompt chunk, then single tokens, each through norm + rotation + cache write and attention; against
    the 64-bit definition of attention on what the cache and q hold."""
    g = torch.Generator().manual_seed(8)
    hq, hk, hd, page = 8, 2, 64, 16
    ks, vs = (0.03125, 0.0625) if dtype is F8 else (1.0, 1.0)
    pool = [torch.zeros((32, page, hk, hd), dtype=dtype, device="cuda") for _ in range(2)]
    lens = [70, 33]
    table = [list(range(0, 10)), list(range(10, 20))]
    dtable = torch.tensor(table, dtype=torch.int32, device="cuda")
    gq, gk = ((torch.rand(n, generator=g) + 0.5).to(BF16).cuda() for n in (hq * hd, hk * hd))
    inv, m = attn.rope_frequencies(hd, 10000.0, "linear", factor=2.0)
    seen = [0, 0]
    for new in (lens, [1, 1], [1, 1], [5, 2]):
        T = sum(new)
        x = torch.randn((T, (hq + 2 * hk) * hd), generator=g).to(BF16).cuda()
        q, k, v = x[:, :hq * hd], x[:, hq * hd:(hq + hk) * hd], x[:, (hq + hk) * hd:]
        pos = torch.cat([torch.arange(s, s + n) for s, n in zip(seen, new)])
        slot = torch.tensor([table[b][p // page] * page + p % page for b in range(2) for p in range(seen[b], seen[b] + new[b])])
        attn.qknorm_fwd_append(q, k, v, gq, gk, pos.cuda(), inv, slot.cuda(), *pool, 1e-6, q, mscale=m, k_scale=ks, v_scale=vs)
        seen = [s + n for s, n in zip(seen, new)]
        starts = [0, new[0], T]
        lse = torch.empty((T, hq), device="cuda")
        out = attn.qknorm_attn_paged(q, *pool, dtable, torch.tensor(seen, dtype=torch.int32, device="cuda"),
                                     torch.tensor(starts, dtype=torch.int32, device="cuda"), max(new), 160, k_scale=ks, v_scale=vs, lse=lse)
        torch.cuda.synchronize()
        ref = R.attention(R.widen(q), R.widen(pool[0]), R.widen(pool[1]), table, seen, starts, hq, scale=1 / 8, k_scale=ks, v_scale=vs)
        tol, tol_lse = R.attention_bounds(ref, hd, dtype is F8)
        assert (np.abs(out.double().cpu().numpy().reshape(T, hq, hd) - ref["out"]) <= tol).all()
        assert (np.abs(lse.double().cpu().numpy() - ref["lse"]) <= tol_lse).all()


def test_starts_that_go_back_stay_inside_the_buffers(libqknorm):
    """q_starts that fall name rows twice: more units than the rows allow for, in a call whose lengths need no workspace."""
    one = Batch([1100], [1500], 1, 1, 64, guard=0)
    want, want_lse = one.call()
    seqs = 200
    assert attn.attn_paged_workspace(seqs, 1100, 1100, 1500, 1, 1, 64) == 0
    one.dtable = one.dtable.expand(seqs, -1).contiguous()
    one.dlens = torch.full((seqs,), 1500, dtype=torch.int32, device="cuda")
    one.dstarts = torch.tensor([0, 1100] * (seqs // 2) + [0], dtype=torch.int32, device="cuda")
    out, lse = one.call()
    ref = one.reference()
    one.compare(out, lse, ref)
    one.compare(want, want_lse, ref)


@BOTH
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("hd", [8, 16, 24, 32, 40, 48, 72, 80, 112, 120])
def test_head_sizes(libqknorm, hd, page, dtype):
    """Heads narrower than the tiles' 64 or 128 columns, in each form."""
    variant = "attn_tc" if dtype is BF16 or hd % 16 == 0 else "attn_general"
    Batch([1, 3], [200, 70], 4, 2, hd, page=page, dtype=dtype).check(variant)
    Batch([50, 7], [130, 300], 2, 1, hd, page=page, dtype=dtype).check(variant)
    Batch([150, 20], [150, 260], 2, 2, hd, page=page, dtype=dtype).check(variant)


@BOTH
@pytest.mark.parametrize("hq,hk,new,kv", [
    (2, 1, [1] * 900, [1 + 7 * i % 60 for i in range(900)]),                           # more units than CTAs, none of them cut
    (1, 1, [(i * 5) % 4 for i in range(700)], [(i * 11) % 200 for i in range(700)]),   # some without tokens, without keys, with fewer keys than tokens
    (1, 1, [140 if i % 50 == 7 else 0 for i in range(400)], [200 if i % 50 == 7 else 0 for i in range(400)]),
])
def test_many_sequences(libqknorm, hq, hk, new, kv, dtype):
    Batch(new, kv, hq, hk, 64, dtype=dtype, seed=3).check("attn_tc")


@BOTH
@pytest.mark.parametrize("page", [64, 20])
@pytest.mark.parametrize("hq,hk,new,kv", [(1, 1, [300], [20000]), (1, 1, [100, 2], [30000, 500]), (4, 2, [1], [40000]), (1, 1, [140, 500], [6000, 9000])])
def test_units_cut_into_many_parts(libqknorm, hq, hk, new, kv, page, dtype):
    """Long keys and few rows: a unit's keys over many CTAs, in each form; with a window that leaves whole parts empty too."""
    b = Batch(new, kv, hq, hk, 64, page=page, dtype=dtype, seed=page)
    b.check("attn_tc")
    b.check("attn_tc", causal=False)
    b.check("attn_tc", window=7000)


@BOTH
def test_pages_shared_by_sequences(libqknorm, dtype):
    b = Batch([1, 1, 40], [300, 300, 300], 4, 2, 128, dtype=dtype)
    for row in b.table[1:]:
        row[:10] = b.table[0][:10]                # 160 keys in common
    b.dtable = torch.tensor(b.table, dtype=torch.int32, device="cuda")
    b.check("attn_tc")


@BOTH
@pytest.mark.parametrize("page,hd", [(16, 128), (7, 64), (16, 36)])
def test_offsets_past_32_bits(libqknorm, page, hd, dtype):
    """Pages 2^30 and some elements apart, K and V between one another: the last one starts past 2^32 elements."""
    b = Batch([1, 3], [40, 20], 2, 1, hd, page=page, dtype=dtype)
    stride = 2 ** 30 + 4096
    size = stride * (b.pages - 1) + 2 * page * hd
    assert stride * (b.pages - 1) > 2 ** 32
    pool = torch.empty(size, dtype=dtype, device="cuda")
    views = [torch.as_strided(pool, (b.pages, page, 1, hd), (stride, hd, hd, 1), off) for off in (0, page * hd)]
    for view, src in zip(views, (b.dk, b.dv)):
        view.view(torch.uint8 if dtype is F8 else torch.int16).copy_(src.view(torch.uint8 if dtype is F8 else torch.int16))
    b.dk, b.dv = views
    b.check("attn_general" if hd == 36 else "attn_tc")
    # written by the cache write, too
    x = torch.randn(2, hd, device="cuda").to(BF16)
    slots = torch.tensor([page * (b.pages - 1), 1], device="cuda")
    q = torch.zeros(2, hd, dtype=BF16, device="cuda")
    attn.qknorm_fwd_append(q, x, x, None, None, None, None, slots, b.dk, b.dv, 0.0, k_scale=0.5, v_scale=0.5)
    torch.cuda.synchronize()
    for view in views:
        got = torch.stack([view[b.pages - 1, 0, 0], view[0, 1, 0]]).float()
        want = (x.float() / 0.5).to(F8).float() if dtype is F8 else x.float()
        assert torch.equal(got, want)


def test_first_call_inside_a_capture(libqknorm):
    """A fresh process whose first call of every entry point is captured."""
    import subprocess
    import sys
    code = """
import torch
from paper_2608_09160_b200 import attn
BF16 = torch.bfloat16
q = torch.randn(2, 256, device="cuda").to(BF16); k = torch.randn(2, 128, device="cuda").to(BF16)
kc = torch.zeros(40, 16, 1, 128, dtype=BF16, device="cuda"); vc = torch.zeros_like(kc)
pos = torch.tensor([599, 5], device="cuda"); slots = torch.tensor([16 * 37 + 7, 16 * 39 + 5], device="cuda")
f = attn.rope_frequencies(128, 10000.0)[0].cuda()
gq, gk = torch.ones(256, dtype=BF16, device="cuda"), torch.ones(128, dtype=BF16, device="cuda")
table = torch.stack([torch.arange(38), torch.full((38,), 39)]).int().cuda()
lens = torch.tensor([600, 6], dtype=torch.int32, device="cuda"); starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
def step():
    a = attn.qknorm_rope(q, k, pos, f, 128)
    b = attn.qknorm_fwd_append(q, k, k, gq, gk, pos, f, slots, kc, vc, 1e-6)
    return a[0], b, attn.qknorm_attn_paged(b, kc, vc, table, lens, starts, 1, 600)
with torch.cuda.graph(g):
    got = step()
g.replay(); torch.cuda.synchronize()
got = [t.clone() for t in got]
want = step(); torch.cuda.synchronize()
assert all(torch.equal(x, y) for x, y in zip(got, want)) and bool(want[2].float().abs().sum() > 0)
print("same")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


@BOTH
@pytest.mark.parametrize("hd", [64, 96, 128])
@pytest.mark.parametrize("new,kv", [([1, 3], [900, 130]), ([20, 9], [700, 260]), ([140, 33], [500, 200])])
def test_gathered_rows_are_the_copied_ones(libqknorm, new, kv, hd, dtype):
    """The same keys in pages of 16 tokens (boxes) and of 7 (rows gathered by the loader warps): the same bits, every time."""
    a, b = (Batch(new, kv, 4, 2, hd, page=page, dtype=dtype) for page in (16, 7))
    for s in range(len(kv)):
        for j in range(kv[s]):
            for src, dst in ((a.k, b.k), (a.v, b.v)):
                raw = torch.uint8 if dtype is F8 else torch.int16
                dst.view(raw)[b.table[s][j // 7], j % 7] = src.view(raw)[a.table[s][j // 16], j % 16]
    b.dk.copy_(b.k.cuda())
    b.dv.copy_(b.v.cuda())
    b.q, b.dq = a.q, a.dq
    want, want_lse = a.call()
    for _ in range(10):
        out, lse = b.call()
        assert binding.last_variant() == "attn_tc"
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)


# The tests of the waits lower their limit, but not below a few milliseconds: a whole GPU stands still for 1.8 ms now and then (seen
# once in eight seconds: nothing in any CTA moved for that long), and a wait cannot tell that from something that hangs.


@BOTH
@pytest.mark.parametrize("new", [4, 10, 40])
def test_rows_done_again_outlast_no_wait(libqknorm, monkeypatch, new, dtype):
    """Rows whose tile holds an infinity that they do not see are done again key by key, which takes far longer than the matrix
    path: 30 to 300 ms here.  With the limit of a wait below that: everybody waits on, and the rows of the batch's other sequences come
    out as ever."""
    seqs, keys, hq, hk, hd = 20, 6000, 64, 8, 64
    b = Batch([new] * seqs, [keys] * seqs, hq, hk, hd, dtype=dtype)
    want, want_lse = b.call()
    vmax = b.v.float().nan_to_num(0.0).abs().amax().item() * b.vs     # unused slots are NaN
    b.v[b.table[0][(keys - 1) // 16], (keys - 1) % 16] = float("nan") if dtype is F8 else float("inf")
    b.dv.copy_(b.v.cuda())                                            # seen by the sequence's last token only
    monkeypatch.setenv("QKNORM_ATTN_WAIT_US", "10000")
    out, lse = b.call()                                               # looks at the error word, too
    n = new * seqs
    assert torch.equal(out[new:n].view(torch.int16), want[new:n].view(torch.int16)) and torch.equal(lse[new:n], want_lse[new:n])
    # The rows done again have fp32 weights where the others' are rounded: apart by half a step of bf16 of sum p |v| <= max |v|, half a
    # step of each result, and three times the scores' error on either side (68 2^-24 of 10 at most, as in attention_bounds).
    x, y = out[:new - 1].double(), want[:new - 1].double()
    assert ((x - y).abs() <= 2.0 ** -8 * 1.01 * (x.abs() + y.abs() + vmax) + 6 * 68 * 2.0 ** -24 * 10 * vmax).all()
    # twice 68 2^-24 of 10, and the sum's 6000 / 32 + 16 steps
    assert ((lse[:new - 1] - want_lse[:new - 1]).abs() <= 2 * (680 + 204) * 2.0 ** -24 + 1e-5).all()
    assert not torch.isfinite(out[new - 1].view(hq, hd)).any()


@BOTH
@pytest.mark.parametrize("new,group,seqs", [(1, 8, 450), (10, 8, 450), (40, 8, 450)])
def test_long_items_outlast_no_wait(libqknorm, monkeypatch, new, group, seqs, dtype):
    """Units of 32768 key tiles (three pages over and over), three a CTA: each takes 16 ms or more, and the rows of the one after the
    next wait for it with a limit of five."""
    g = torch.Generator().manual_seed(4)
    keys, page, hd = 1 << 22, 64, 64
    k, v = (torch.randn((3, page, 1, hd), generator=g).to(dtype).cuda() for _ in range(2))
    table = torch.arange(keys // page, dtype=torch.int32).remainder(3).expand(seqs, -1).contiguous().cuda()
    lens = torch.full((seqs,), keys, dtype=torch.int32, device="cuda")
    starts = torch.arange(0, (seqs + 1) * new, new, dtype=torch.int32, device="cuda")
    q = torch.randn((seqs * new, group * hd), generator=g).to(BF16).cuda()
    go = lambda: attn.qknorm_attn_paged(q, k, v, table, lens, starts, new, keys)
    want = go()
    torch.cuda.synchronize()
    monkeypatch.setenv("QKNORM_ATTN_WAIT_US", "5000")
    out = go()
    torch.cuda.synchronize()
    assert binding.device_error_word() == 0
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("new,seqs", [(1, 4_000_000), (300, 400_000)])
def test_sequences_without_rows_outlast_no_wait(libqknorm, monkeypatch, new, seqs):
    """Millions of sequences without new tokens between two that have some: passing by them takes 20 ms, the limit of a wait is five."""
    hd = 64
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((4, 16, 1, hd), generator=g).to(BF16).cuda() for _ in range(2))
    q = torch.randn((2 * new, hd), generator=g).to(BF16).cuda()
    starts = torch.full((seqs + 1,), new, dtype=torch.int32, device="cuda")
    starts[0], starts[-1] = 0, 2 * new
    lens = torch.full((seqs,), 40, dtype=torch.int32, device="cuda")
    table = torch.tensor([2, 0, 3], dtype=torch.int32, device="cuda").expand(seqs, -1).contiguous()
    want = attn.qknorm_attn_paged(q, k, v, table[:2], lens[:2], starts[[0, 1, -1]].contiguous(), new, 40)
    monkeypatch.setenv("QKNORM_ATTN_WAIT_US", "5000")
    out = attn.qknorm_attn_paged(q, k, v, table, lens, starts, new, 40)
    torch.cuda.synchronize()
    assert binding.device_error_word() == 0
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("new", [1, 10, 60])
def test_small_weights_over_an_fp8_cache(libqknorm, new):
    """One key outweighs 1499 others by 2^26 each and holds zeros: what comes out is theirs alone.  A weight keeps at least an absolute
    step of 2^-25 in fp16, where the largest stands for 2^7: 2^-32 of it instead of the 2^-25 that attention_bounds allows."""
    b = Batch([new], [1500], 8, 1, 64, dtype=F8)
    b.q.zero_()
    b.q.view(b.T, 8, 64)[:, :, 0] = 9.0
    b.k[:], b.v[:] = 0.0, 448.0
    first = (b.table[0][0], 0)
    b.k[first][0, 0], b.v[first] = 8.0, 0.0               # 9 * 8 * 0.25 = 18 = 25.97 ln 2
    for dev, host in ((b.dq, b.q), (b.dk, b.k), (b.dv, b.v)):
        dev.copy_(host.cuda())
    kw = dict(scale=1.0, causal=False)
    ref = b.reference(**kw)
    out, lse = b.call(**kw)
    tol, tol_lse = R.attention_bounds(ref, 64, True)
    tol = tol[:new] - (2.0 ** -25 - 2.0 ** -32) * ref["V"][:new]
    want = ref["out"][:new]
    assert (want > 20 * tol).all()
    assert (np.abs(out[:new].double().numpy().reshape(want.shape) - want) <= tol).all()
    assert (np.abs(lse[:new].double().numpy() - ref["lse"][:new]) <= tol_lse[:new]).all()


@BOTH
@pytest.mark.parametrize("new", [1, 10, 60])
def test_scores_beyond_their_own_precision(libqknorm, new, dtype):
    """Scores of tens of millions, apart by less than their own fp32 step and then by far more: weights are coarse there, but finite and
    never past the format they are rounded to."""
    g = torch.Generator().manual_seed(9)
    b = Batch([new], [700], 8, 1, 64, dtype=dtype)
    b.q.fill_(2.0 ** 14)
    grow = 240.0 + 16.0 * torch.arange(44).div(44).repeat_interleave(16)
    for j in range(700):
        b.k[b.table[0][j // 16], j % 16] = (grow[j] + torch.randint(0, 3, (64,), generator=g)).to(dtype)
    b.dq.copy_(b.q.cuda())
    b.dk.copy_(b.k.cuda())
    b.dv.copy_(torch.nan_to_num(b.v.float()).to(dtype).cuda())
    out, lse = b.call(scale=1.0, causal=False)
    vmax = torch.nan_to_num(b.v.float()).abs().max().item() * b.vs
    assert torch.isfinite(out[:new].float()).all() and torch.isfinite(lse[:new]).all()
    assert (out[:new].float().abs() <= vmax * 1.01).all()


@BOTH
def test_window_without_the_causal_edge_is_shared_out(libqknorm, dtype):
    """With causal=False a row sees every key behind its window's start, so the first of several units has all of the sequence: it is
    cut (two launches), and a workspace that was asked for without saying causal or not does for both."""
    b = Batch([2048], [2048], 1, 1, 64, dtype=dtype)
    n0 = binding.launch_count()
    b.check("attn_tc", causal=False, window=64)
    assert binding.launch_count() - n0 == 2
    need = attn.attn_paged_workspace(1, b.T, 2048, 2048, 1, 1, 64, window=64)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for causal in (True, False):
        out, lse = b.call(causal=causal, window=64, workspace=ws)
        b.compare(out, lse, b.reference(causal=causal, window=64))
    Batch([700, 3, 500], [900, 40, 500], 4, 2, 64, dtype=dtype).check("attn_tc", causal=False, window=130)


@pytest.mark.parametrize("variant", ["attn_tc", "attn_general"])
@pytest.mark.parametrize("new", [1, 10, 60])
def test_scales_so_small_that_every_key_counts_alike(libqknorm, new, variant):
    """scale * k_scale below what fp32 holds, or brought there by a tiny query row: the weights of the keys a row sees are equal."""
    b = Batch([new], [200], 8, 1, 64 if variant == "attn_tc" else 56, dtype=F8)
    b.check(variant, scale=1e-45)
    b.q.copy_((b.q.double() * 2.0 ** -112).to(BF16))
    b.dq.copy_(b.q.cuda())
    b.check(variant, scale=1e-10)
    b.check(variant, scale=2.0 ** -30)


@BOTH
@pytest.mark.parametrize("new", [1, 10, 60])
def test_no_keys_at_all(libqknorm, new, dtype):
    """max_kv = 0, and a block table without columns: every row is empty."""
    b = Batch([new, new], [200, 3], 8, 1, 64, dtype=dtype)
    for _ in range(2):
        out, lse = b.call(max_kv=0)
        assert (out[:2 * new] == 0).all() and torch.isneginf(lse[:2 * new]).all() and (out[2 * new:] == 7.0).all()
        b.dtable = b.dtable[:, :0].contiguous()
    out, lse = b.call()
    assert (out[:2 * new] == 0).all() and torch.isneginf(lse[:2 * new]).all() and (out[2 * new:] == 7.0).all()


@BOTH
@pytest.mark.parametrize("new", [[1, 1], [10, 3], [70, 300]])
def test_the_largest_bounds(libqknorm, new, dtype):
    """max_q, max_kv and the window at the ends of their ranges say nothing about the batch: the same results, within the workspace asked for."""
    kv = [300, 500]
    b = Batch(new, kv, 4, 2, 64, dtype=dtype)
    for causal in (True, False):
        for kw in (dict(max_kv=0x7fffff00), dict(max_q=2 ** 31 - 1), dict(window=2 ** 31 - 1), dict(max_q=2 ** 31 - 1, max_kv=0x7fffff00, window=2 ** 31 - 1)):
            out, lse = b.call(causal=causal, **kw)
            b.compare(out, lse, b.reference(causal=causal))
