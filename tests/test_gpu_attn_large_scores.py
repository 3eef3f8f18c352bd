"""Attention where scores are so large that fp32 numbers lie far apart there."""
import numpy as np
import pytest
import torch

from paper_2608_09160_b200 import binding
from tests import attn_reference as R
from tests.e2m1_reference import BF16, F8
from tests.test_gpu_attn import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e", [20, 30, 60, 112])
@pytest.mark.parametrize("dtype", [BF16, F8], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("new,hd", [([1, 2], 128), ([20, 9], 128), ([100, 60], 128), ([100, 60], 64), ([2, 40], 256)])
def test_scores_of_any_size(libqknorm, new, hd, dtype, e):
    """Queries of 2^e: where the largest score is ahead of the next by more than fp32 sums of D products are off, the result is its key's value."""
    b = Batch(new, [500, 300], 4, 2, hd, dtype=dtype, seed=61)
    b.q = (b.q.double() * 2.0 ** e).to(BF16)
    b.dq = b.q.cuda()
    k, v = (R.widen(t.nan_to_num(0.0) if dtype is BF16 else t.float().nan_to_num(0.0)).numpy() * u for t, u in ((b.k, b.ks), (b.v, b.vs)))
    out, lse = b.call()
    assert binding.last_variant() == ("attn_tc" if hd <= 128 else "attn_general")
    q, got, z, clear = R.widen(b.q).numpy().reshape(b.T, 4, hd), out.double().numpy().reshape(b.T, 4, hd), lse.double().numpy(), 0
    for s, L in enumerate(b.kv):
        kk, vv = (x[b.table[s][:-(-L // b.page)]].reshape(-1, 2, hd) for x in (k, v))
        for r in range(b.starts[s], b.starts[s + 1]):
            seen = L - (b.starts[s + 1] - r) + 1
            for h in range(4):
                K, V = kk[:seen, h // 2], vv[:seen, h // 2]
                score = K @ q[r, h] * hd ** -0.5
                off = (hd + 4) * 2.0 ** -24 * hd ** -0.5 * (np.abs(K) @ np.abs(q[r, h])).max()
                assert abs(z[r, h] - score.max()) <= 2 * off + 10, (r, h)          # log of at most 500 weights, fp32 products
                assert (np.abs(got[r, h]) <= np.abs(V).max(0) * 1.01).all(), (r, h)
                top = int(score.argmax())
                if score[top] - np.delete(score, top).max() > 2 * off + 30:
                    clear += 1
                    assert (np.abs(got[r, h] - V[top]) <= 2.0 ** -7 * np.abs(V[top]) + 1e-6).all(), (r, h)
    assert clear > 0
