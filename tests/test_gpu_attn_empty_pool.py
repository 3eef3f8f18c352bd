"""Attention over a pool without pages whose pointers mean nothing: no key is read, each stands for zeros."""
import ctypes

import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests.e2m1_reference import BF16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [0, 1])
@pytest.mark.parametrize("hd", [64, 96, 128, 256])
@pytest.mark.parametrize("new", [[1, 2], [150, 2]])
def test_an_empty_pool_at_any_address(libqknorm, new, hd, e4m3):
    kv, hq, hk, T = [300, 40], 4, 2, sum(new)
    lib = attn.lib()
    q = torch.randn((T, hq * hd), generator=torch.Generator().manual_seed(hd)).to(BF16).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((T, hq), 7.0, device="cuda")
    store = torch.zeros(64, dtype=torch.uint8, device="cuda")
    c = attn.CPagedCache(store.data_ptr() + 2, store.data_ptr() + 6, 1001, 3, 5, 1003, 7, 9, 0, 16, hk, hd, e4m3, 1.0, 1.0)
    table = torch.zeros((2, 19), dtype=torch.int32, device="cuda")
    lens, starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (kv, [0, new[0], T]))
    n = attn.attn_paged_workspace(2, T, max(new), 300, hq, hk, hd)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    rc = lib.qknorm_attn_paged(q.data_ptr(), 0, ctypes.byref(c), table.data_ptr(), 19, 0, lens.data_ptr(), starts.data_ptr(), 2, T, max(new), 300, hq,
                               0.125, 1, 0, out.data_ptr(), 0, lse.data_ptr(), ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == binding.QKNORM_OK and binding.device_error_word() == 0
    seen = torch.tensor([L - m + i + 1 for m, L in zip(new, kv) for i in range(m)]).double()
    assert (out == 0).all() and ((lse.cpu().double() - torch.log(seen)[:, None]).abs() < 1e-5).all()
