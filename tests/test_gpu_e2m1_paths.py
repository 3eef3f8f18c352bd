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
