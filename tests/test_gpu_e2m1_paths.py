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
