"""Calls of the 4-bit cache, several axes and the pages that are marshalled once and made again and again (binding.prepared)."""
import gc

import pytest
import torch

from paper_2608_09160_b200 import attn, binding, pages
from tests.e2m1_reference import BF16, F8
from tests.test_gpu_e2m1 import Batch, Layer
from tests.test_gpu_pages import I32, Model

pytestmark = pytest.mark.gpu


def again(call, n=3):
    for _ in range(n):
        call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [[1, 2], [60, 3]])
def test_attention(libqknorm, new):
    b = Batch(new, [700, 300], 8, 2, 128, seed=71)
    want, _ = b.call()
    n = b.starts[-1]
    out = torch.zeros_like(b.dq)
    call = binding.prepared(attn.qknorm_attn_paged_e2m1, b.dq, *b.pools, b.dtable, b.dlens, b.dstarts, max(new), 700, k_scale=b.unit[0], v_scale=b.unit[1], out=out)
    assert call.outputs is out and (out == 0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    again(call)
    assert torch.equal(out[:n].cpu().view(torch.int16), want[:n].view(torch.int16))


def test_append_and_rotation_with_several_axes(libqknorm):
    one, two = Layer(45, 4, 2, 128, seed=3, axes=3), Layer(45, 4, 2, 128, seed=3, axes=3)
    out = one.call("layerwise", False)
    c = lambda t: t.cuda()
    call = binding.prepared(attn.qknorm_fwd_append_e2m1, c(two.q), c(two.k), c(two.v), c(two.gq), c(two.gk), c(two.pos), c(two.inv_freq), c(two.slots),
                            *two.dcodes, *two.dscales, 1e-6, axis=c(two.axis))
    gc.collect()                                         # the call keeps what it reads
    junk = [torch.full((1 << 16,), 77, dtype=torch.uint8, device="cuda") for _ in range(64)]
    again(call)
    del junk
    assert torch.equal(call.outputs.view(torch.int16), out.view(torch.int16))
    for x, y in zip(one.dcodes + one.dscales, two.dcodes + two.dscales):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    q, pos, inv, axis = c(one.q), c(one.pos), c(one.inv_freq), c(one.axis)
    want, _ = attn.qknorm_rope(q, None, pos, inv, 128, axis=axis)
    call = binding.prepared(attn.qknorm_rope, q, None, pos, inv, 128, axis=axis)
    again(call)
    assert torch.equal(call.outputs[0].view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("as_", [list, iter], ids=["list", "iterator"])
def test_pages_keep_their_pools(libqknorm, as_):
    """Whatever the pools come in, the tensors are the call's as long as it lives."""
    m = Model(12, 4, 5, seed=9, pools=[torch.randint(0, 256, (12, 64), dtype=torch.uint8, device="cuda") for _ in range(3)])
    src, dst = (torch.tensor(x, dtype=I32, device="cuda") for x in ([1, 2], [5, 6]))
    m.give(0, 20)
    ok = torch.zeros(1, dtype=I32, device="cuda")
    row = lambda r: torch.tensor([r], dtype=I32, device="cuda")
    box = as_(m.pools) if as_ is iter else list(m.pools)
    copy = binding.prepared(pages.qknorm_pages_copy, box, src, dst)
    if as_ is list:
        box.clear()
    fork = binding.prepared(pages.qknorm_pages_fork, as_(m.pools), m.drefs, m.dtable, m.dlens, row(0), row(1), 16, ok=ok)
    free = binding.prepared(pages.qknorm_pages_free, m.drefs, m.dtable, m.dlens, row(1), 16)
    pack = binding.prepared(pages.qknorm_pages_compact, as_(m.pools), m.drefs, m.dtable, m.dlens, 16)
    for call in (copy, fork, pack):
        kept = [t for k in call.keep if isinstance(k, (list, tuple)) for t in k]
        assert [t.data_ptr() for t in kept] == [p.data_ptr() for p in m.pools]
    data = [p.clone() for p in m.pools]
    again(copy)
    for p, d in zip(m.pools, data):
        assert torch.equal(p[5:7], d[1:3]) and torch.equal(p[:5], d[:5]) and torch.equal(p[7:], d[7:])
    for _ in range(3):
        fork()
        torch.cuda.synchronize()
        assert ok.item() == 1 and m.dlens.tolist() == [20, 20, 0, 0] and int((m.drefs > 0).sum()) == 3
        pack()
        assert pack.outputs.item() == 3 and (m.drefs[:3] > 0).all()
        free()
    torch.cuda.synchronize()
    assert m.dlens.tolist() == [20, 0, 0, 0] and int((m.drefs > 0).sum()) == 2
