"""Attention over a 4-bit cache: which way a call goes, and what only some ways meet."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests import attn_reference as R
from tests import e2m1_reference as E
from tests.e2m1_reference import BF16, F8
from tests.test_e2m1_pages_cpu import A, D, attend, cache
from tests.test_gpu_e2m1 import Batch, copies  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [0, 1000])
@pytest.mark.parametrize("seqs", [2 ** 18, 2 ** 20 + 1, 2 ** 21, 2 ** 26 + 12345])
def test_a_widened_cache_beyond_64_bits_is_not_planned(libqknorm, seqs, window):
    """seqs * max_kv elements of K and V whose bytes pass 2^63: the cache is not widened, and the workspace is that of the row tiles --
    8 for each sequence and key head; more than 2^31 - 1 are refused."""
    lib = attn.lib()
    if seqs * 8 * 8 > 2 ** 31 - 1:
        with pytest.raises(binding.QKNormError) as refused:
            attn.attn_paged_e2m1_workspace(seqs, 128, 128, 0x7FFFFF00, 8, 8, 128, window)
        assert refused.value.status == binding.QKNORM_ERR_SHAPE
        return
    need = attn.attn_paged_e2m1_workspace(seqs, 128, 128, 0x7FFFFF00, 8, 8, 128, window)
    assert 0 < need < 2 ** 26
    c = cache(pages_=8, heads=8, hd=128)
    for ws, n in ((None, 0), (0x70000000, need - 16)):      # told before anything is launched
        assert attend(lib, c, seqs=seqs, T=128, max_q=128, max_kv=0x7FFFFF00, hq=8, window=window, ws=ws, wsb=n) == binding.QKNORM_ERR_SCRATCH


@pytest.mark.parametrize("hq,hk,hd,new", [(4, 2, 128, [1, 2]), (4, 2, 64, [1, 2]), (3, 1, 96, [1, 1]), (2, 1, 16, [1, 1]), (8, 2, 256, [9, 2]), (2, 2, 128, [60, 2]),
                                          (4, 1, 128, [60, 2])])
def test_an_empty_pool_beside_queries_at_odd_addresses(libqknorm, copies, hq, hk, hd, new):
    """Nothing of a pool without pages is read, whatever its strides say and wherever q lies: its keys and values are zeros."""
    kv = [300, 40]
    T, g = sum(new), torch.Generator().manual_seed(hd)
    wide = torch.randn((T, hq * hd + 3), generator=g).to(BF16).cuda()
    q = wide[:, 1:1 + hq * hd]                                    # two bytes behind a multiple of 16, rows an odd number of bytes apart
    assert q.data_ptr() % 16 == 2
    store = torch.zeros(64, dtype=torch.uint8, device="cuda")
    pool = lambda n, at: store[at:].as_strided((0, 16, hk, n), (1001 * n, hk * n + 3, n + 1, 1))
    pools = [pool(hd // 2, 1), pool(hd // 2, 3)] + [pool(hd // 16, at).view(F8) for at in (5, 7)]
    table = torch.zeros((2, 19), dtype=torch.int32, device="cuda")
    lens, starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (kv, [0, new[0], T]))
    lse = torch.full((T, hq), 7.0, device="cuda")
    out = torch.full((T, hq * hd), 7.0, dtype=BF16, device="cuda")
    attn.qknorm_attn_paged_e2m1(q, *pools, table, lens, starts, max(new), 300, out=out, lse=lse)
    torch.cuda.synchronize()
    assert binding.device_error_word() == 0
    seen = torch.tensor([L - m + i + 1 for m, L in zip(new, kv) for i in range(m)]).double()
    some = seen > 0
    assert (out == 0).all() and torch.isneginf(lse[~some.cuda()]).all()
    assert ((lse.cpu().double() - torch.log(seen.clamp(min=1))[:, None]).abs()[some] < 1e-5).all()


def weights_in_fp16(b, variant="attn_tc", **kw):
    """The call's rows within the bounds that weights in fp16 have."""
    ref = b.reference(**{k: v for k, v in kw.items() if k in ("scale", "causal", "window", "max_kv")})
    out, lse = b.call(**kw)
    assert binding.last_variant() == variant
    b.compare(out, lse, ref, True)
    return out, lse


@pytest.mark.parametrize("hq,hk,hd,new,kv", [
    (5, 1, 128, [60, 3, 26], [60, 200, 27]), (8, 2, 64, [26, 17, 33], [300, 17, 129]), (3, 1, 96, [100, 1, 0], [256, 300, 9]), (1, 1, 128, [300], [300]),
    (2, 2, 16, [120], [500]), (128, 1, 64, [2, 1], [130, 140]), (4, 2, 80, [80, 130], [80, 130]), (1, 1, 128, [101], [9000]), (6, 2, 64, [40, 1], [40, 20000]),
])
def test_weights_do_not_get_coarser_with_more_rows(libqknorm, hq, hk, hd, new, kv):
    """Short rows among them, where a weight's rounding shows: 2^-9 of a value that others nearly cancel."""
    weights_in_fp16(Batch(new, kv, hq, hk, hd, seed=31 + hd))


@pytest.mark.parametrize("window", [1, 31, 100])
@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_windowed_chunks(libqknorm, causal, window):
    weights_in_fp16(Batch([80, 1, 53], [400, 257, 90], 4, 2, 128, seed=window), causal=causal, window=window)


def test_a_row_is_rounded_the_same_beside_a_chunk(libqknorm):
    """Two decode rows alone, and in a batch with a chunk: both within the bounds of fp16 weights."""
    weights_in_fp16(Batch([1, 1], [5, 40], 8, 2, 128, seed=33), "attn_e2m1")
    weights_in_fp16(Batch([1, 1, 64], [5, 40, 64], 8, 2, 128, seed=33))


def test_extreme_queries_of_a_chunk(libqknorm):
    b = Batch([60, 60], [64, 64], 4, 2, 128, seed=34)
    for row, e in ((0, 10), (3, 14), (5, -100), (9, -112), (11, -120), (20, -130), (21, -126), (60, 9), (61, -133)):
        b.q[row] = (b.q[row].double() * 2.0 ** e).to(BF16)
    b.q[30] = 0
    b.q[31, 5], b.q[32, 7] = float("nan"), float("inf")
    b.dq = b.q.cuda()
    keep = [r for r in range(120) if r not in (31, 32)]
    for scale in (2.0 ** -3, 1e-38, 2.0 ** 100):       # the last: rows so small that without it every score would be 0
        if scale > 1:
            big = torch.ones(b.T, dtype=torch.bool)
            big[[5, 9, 11, 20, 21, 61]] = False
            b.q[big] = 0
            b.dq = b.q.cuda()
            keep = list(range(120))
        ref = b.reference(scale=scale)
        out, lse = b.call(scale=scale)
        assert binding.last_variant() == "attn_tc"
        got, z = out.double().numpy().reshape(b.T, 4, 128), lse.double().numpy()
        tol, tol_lse = R.attention_bounds(ref, 128, True)
        for r in keep:
            assert (np.abs(got[r] - ref["out"][r]) <= tol[r]).all() and (np.abs(z[r] - ref["lse"][r]) <= tol_lse[r]).all(), (scale, r)
        if scale < 1:
            assert np.isnan(got[31, 0]).all() and np.isnan(got[32, 0]).all()     # of the head that has them; the others
            for r in (31, 32):
                assert (np.abs(got[r, 1:] - ref["out"][r, 1:]) <= tol[r, 1:]).all()


def test_small_weights_of_a_chunk_are_kept(libqknorm):
    """One key far above the rest of a long row: 30000 others share 2^-20 of its weight each."""
    b = Batch([100], [30000], 1, 1, 64, seed=35)
    b.k[:], b.ks.view(torch.uint8)[:] = 0, 0x38
    b.k[b.table[0][0], 0, 0, 0] = 0x04
    b.q[:] = 0
    b.q[:100, 0] = 20 * np.log(2) / (2 * 0.25) * 8.0
    b.dq = b.q.cuda()
    b.place()
    weights_in_fp16(b)


@pytest.mark.parametrize("hd", [64, 128])
def test_values_a_chunk_does_not_see_do_not_matter(libqknorm, hd):
    """NaN in blocks of K and V that only the later rows of a chunk see."""
    b = Batch([120], [200], 2, 1, hd, seed=36)
    for pool, key, blk in ((b.vs, 150, hd // 16 - 1), (b.ks, 180, 0)):        # seen from rows 70 and 100 on
        pool.view(torch.uint8)[b.table[0][key // 16], key % 16, 0, blk] = 0xFF
    b.place()
    out, lse = b.call()
    assert binding.last_variant() == "attn_tc"
    ref = b.reference()
    got = out.double().numpy().reshape(b.T, 2, hd)
    tol, _ = R.attention_bounds(ref, hd, True)
    for r in range(100):
        first = 0 if r < 70 else hd - 16
        assert (np.abs(got[r] - ref["out"][r]) <= tol[r])[:, :hd if r < 70 else first].all(), r
        assert r < 70 or np.isnan(got[r][:, hd - 16:]).all()
    assert np.isnan(got[100:120]).all()


@pytest.mark.parametrize("which", ["q", "out", "ld_q", "ld_out"])
@pytest.mark.parametrize("hq,hk,hd,new,kv", [(8, 2, 128, [60, 1], [300, 77]), (3, 1, 64, [200, 40], [700, 2000]), (5, 1, 96, [30], [30])])
def test_chunks_at_odd_addresses(libqknorm, copies, hq, hk, hd, new, kv, which):
    """More than 96 rows whose q or out "attn_tc" cannot take: row tiles, not a row at a time over a widened cache."""
    b = Batch(new, kv, hq, hk, hd, seed=51)
    ref = b.reference()
    n, at = hq * hd, {"q": 1, "out": 1}.get(which, 0)
    gap = 8 if at else 3
    q, out = b.dq, torch.full_like(b.dq, 7.0)
    around = torch.full((b.T, n + gap), 7.0, dtype=BF16, device="cuda")
    if which in ("q", "ld_q"):
        around[:, at:at + n] = q
        q = around[:, at:at + n]
    else:
        out = around[:, at:at + n]
    lse = torch.full((b.T, hq), 7.0, device="cuda")
    need = attn.attn_paged_e2m1_workspace(len(new), b.T, max(new), max(kv), hq, hk, hd)
    ws = torch.full((need + 32,), 77, dtype=torch.uint8, device="cuda")
    attn.qknorm_attn_paged_e2m1(q, *b.pools, b.dtable, b.dlens, b.dstarts, max(new), max(kv), k_scale=b.unit[0], v_scale=b.unit[1], out=out, lse=lse,
                                workspace=ws[:need])
    torch.cuda.synchronize()
    assert binding.last_variant() == "attn_e2m1" and binding.device_error_word() == 0
    b.compare(out.cpu(), lse.cpu(), ref, True)
    assert (ws[need:] == 77).all()
    if which in ("out", "ld_out"):
        assert (around[:, :at] == 7.0).all() and (around[:, at + n:] == 7.0).all()


def test_what_the_second_kernel_refuses_is_refused_before_the_first(libqknorm):
    """More items than "attn_tc" can count: told before the cache is widened."""
    lib, seqs, new = attn.lib(), 2 ** 16, 2 ** 16
    need = attn.attn_paged_e2m1_workspace(seqs, new, new, 16, 128, 1, 64)
    assert need > 2 ** 31
    before = lib.qknorm_launch_count()
    assert attend(lib, cache(pages_=8, heads=1, hd=64), q=0x100000000, out=0x200000000, seqs=seqs, T=new, max_q=new, max_kv=16, cols=1, hq=128,
                  ws=0x300000000, wsb=need) == binding.QKNORM_ERR_SHAPE
    assert lib.qknorm_launch_count() == before


@pytest.mark.parametrize("hq,hk,hd", [(8, 8, 128), (16, 8, 64), (8, 4, 128), (64, 4, 128), (12, 4, 64), (4, 1, 128)])
@pytest.mark.parametrize("page", [16, 64])
def test_shares_of_several_stretches_of_pages(libqknorm, copies, page, hq, hk, hd):
    """Shares of more rounds than pages are looked up for at a time: 160 sequences over the same 20000 keys, the last of them of other lengths.
    (Keys of a round: 32 for 8 / hk heads' warps; pages in runs of 16 or 32 tokens, 256 at a time.)"""
    S, lens = 160, [20000, 19999, 15003, 17]
    b = Batch([1], [20000], hq, hk, hd, page=page, seed=41)
    g = torch.Generator().manual_seed(42)
    q = torch.randn((4, hq * hd), generator=g).to(BF16)
    ref = R.attention(R.widen(q), E.widen(b.k, b.ks), E.widen(b.v, b.vs), b.table * 4, lens, [0, 1, 2, 3, 4], hq, scale=hd ** -0.5, k_scale=b.unit[0],
                      v_scale=b.unit[1])
    tol, tol_lse = R.attention_bounds(ref, hd, True)
    which = torch.tensor([i % 3 if i < S - 8 else i % 4 for i in range(S)])
    out, lse = torch.full((S, hq * hd), 7.0, dtype=BF16, device="cuda"), torch.full((S, hq), 7.0, device="cuda")
    attn.qknorm_attn_paged_e2m1(q[which].cuda(), *b.pools, b.dtable.expand(S, -1).contiguous(), torch.tensor(lens, dtype=torch.int32)[which].cuda(),
                                torch.arange(S + 1, dtype=torch.int32, device="cuda"), 1, 20000, k_scale=b.unit[0], v_scale=b.unit[1], out=out, lse=lse)
    torch.cuda.synchronize()
    assert binding.device_error_word() == 0 and binding.last_variant() == "attn_e2m1"
    got, z = out.cpu().double().numpy().reshape(S, hq, hd), lse.cpu().double().numpy()
    for r, n in enumerate(which.tolist()):
        assert (np.abs(got[r] - ref["out"][n]) <= tol[n]).all() and (np.abs(z[r] - ref["lse"][n]) <= tol_lse[n]).all(), r


@pytest.mark.parametrize("e", [20, 30, 60, 100, 112])
@pytest.mark.parametrize("new,variant", [([1, 2], "attn_e2m1"), ([60, 30], "attn_tc")])
def test_scores_of_any_size(libqknorm, copies, new, variant, e):
    """Queries of 2^e: where the largest score is ahead of the next by more than fp32 sums of D products are off, the result is its key's value."""
    hd = 128
    b = Batch(new, [500, 300], 4, 2, hd, seed=61)
    b.q = (b.q.double() * 2.0 ** e).to(BF16)
    b.dq = b.q.cuda()
    ref = b.reference()
    out, lse = b.call()
    assert binding.last_variant() == variant
    b.compare(out, lse, ref, True)                        # no NaN, and lse
    k, v = (E.widen(c, s).numpy() * u for c, s, u in zip((b.k, b.v), (b.ks, b.vs), b.unit))
    q, got, clear = R.widen(b.q).numpy().reshape(b.T, 4, hd), out.double().numpy().reshape(b.T, 4, hd), 0
    for s, L in enumerate(b.kv):
        kk, vv = (x[b.table[s][:-(-L // b.page)]].reshape(-1, 2, hd) for x in (k, v))
        for r in range(b.starts[s], b.starts[s + 1]):
            seen = L - (b.starts[s + 1] - r) + 1
            for h in range(4):
                score = kk[:seen, h // 2] @ q[r, h] * hd ** -0.5
                top = int(score.argmax())
                second = np.delete(score, top).max()
                if score[top] - second > 2 * (hd + 4) * 2.0 ** -24 * ref["S"][r, h] + 30:
                    clear += 1
                    assert (np.abs(got[r, h] - vv[top, h // 2]) <= 2.0 ** -7 * np.abs(vv[top, h // 2]) + 1e-6).all(), (r, h)
    assert clear > 0


@pytest.mark.parametrize("hq,hk,hd,new,kv", [(8, 2, 128, [60, 1], [300, 77]), (2, 2, 48, [120], [500])])
def test_a_widened_cache_read_a_row_at_a_time(libqknorm, monkeypatch, hq, hk, hd, new, kv):
    """What unaligned rows come to where the row tiles cannot be counted."""
    monkeypatch.setenv("QKNORM_FORCE_VARIANT", "general")
    b = Batch(new, kv, hq, hk, hd, seed=81)
    weights_in_fp16(b, "attn_general")


@pytest.mark.parametrize("hd", [64, 128, 96])
def test_rows_too_far_apart_for_boxes(libqknorm, hd):
    """One row whose stride no tensor map takes: K, V and Q are gathered."""
    b = Batch([1], [700], 128, 1, hd, seed=82, guard=0)
    ref = b.reference()
    lib = attn.lib()
    need = attn.attn_paged_e2m1_workspace(1, 1, 1, 700, 128, 1, hd)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(b.dq, 7.0), torch.full((1, 128), 7.0, device="cuda")
    k, v, ks, vs = b.pools
    strides = [t.stride(d) for t in (k, v, ks, vs) for d in range(3)]
    c = attn.CPagedCacheE2m1(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), *strides, b.pages, b.page, 1, hd, *b.unit)
    rc = lib.qknorm_attn_paged_e2m1(b.dq.data_ptr(), 2 ** 40, ctypes.byref(c), b.dtable.data_ptr(), b.dtable.shape[1], 0, b.dlens.data_ptr(),
                                    b.dstarts.data_ptr(), 1, 1, 1, 700, 128, hd ** -0.5, 1, 0, out.data_ptr(), 0, lse.data_ptr(), ws.data_ptr(), need,
                                    torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == binding.QKNORM_OK and binding.last_variant() == "attn_tc" and binding.device_error_word() == 0
    b.compare(out.cpu(), lse.cpu(), ref, True)


def test_two_chunks_at_once(libqknorm):
    """Chunks on two streams, each with a workspace of its own, give what they give alone; so do chunks beside single tokens."""
    batches = [Batch([80, 33, 1], [900, 33, 2500], 8, 4, 128, seed=83), Batch([130], [4000], 4, 2, 64, seed=84), Batch([1] * 8, [2500] * 8, 8, 8, 128, seed=85)]
    want = [b.call()[0] for b in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    outs = [[torch.zeros_like(b.dq) for _ in range(5)] for b in batches]
    torch.cuda.synchronize()
    for i in range(5):
        for b, s, o in zip(batches, streams, outs):
            attn.qknorm_attn_paged_e2m1(b.dq, *b.pools, b.dtable, b.dlens, b.dstarts, max(b.new), max(b.kv), k_scale=b.unit[0], v_scale=b.unit[1], out=o[i], stream=s)
    torch.cuda.synchronize()
    for b, w, o in zip(batches, want, outs):
        n = b.starts[-1]
        for y in o:
            assert torch.equal(y.cpu()[:n].view(torch.int16), w[:n].view(torch.int16))


def test_lengths_grow_between_replays_of_a_chunk(libqknorm):
    b = Batch([64, 64], [700, 1500], 4, 2, 128, seed=86)
    out = torch.zeros_like(b.dq)
    ws = torch.empty(attn.attn_paged_e2m1_workspace(2, b.T, 64, 1500, 4, 2, 128), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.qknorm_attn_paged_e2m1(b.dq, *b.pools, b.dtable, b.dlens, b.dstarts, 64, 1500, k_scale=b.unit[0], v_scale=b.unit[1], out=out, workspace=ws)
    for lens in ([64, 64], [0, 1499], [700, 1500], [33, 128]):
        b.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        ws.fill_(255)                                   # NaN in every place that nothing is widened into
        graph.replay()
        want, _ = b.call(max_kv=1500)
        assert torch.equal(out.cpu()[:128].view(torch.int16), want[:128].view(torch.int16)) and not torch.isnan(out).any()
