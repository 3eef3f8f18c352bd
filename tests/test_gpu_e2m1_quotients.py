"""What goes into a 4-bit cache, bit for bit, over every scale that a block can have: the quotients that choose scales and codes are
correctly rounded fp32 ones, which fp32 divisions on the host are, too."""
import numpy as np
import pytest
import torch

from paper_2608_09160_b200 import attn, binding
from tests import e2m1_reference as E
from tests.e2m1_reference import BF16, F8

pytestmark = pytest.mark.gpu
TIES = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
BLOCKS = 40                                               # of every scale


def values(unit, seed):
    """bf16 [126 * BLOCKS / 8, 128]: blocks whose scale is about each positive E4M3 value, and elements on, beside and between the
    borders of their codes."""
    g = np.random.default_rng(seed)
    scale = torch.arange(1, 127, dtype=torch.uint8).view(F8).double().numpy().repeat(BLOCKS)[:, None] * unit
    x = g.uniform(-6, 6, (len(scale), 16))
    tie = g.random(x.shape) < 0.7
    x[tie] = (g.choice(TIES, x.shape) * g.choice([-1.0, 1.0], x.shape))[tie]
    x[:, 0] = 6.0 * g.uniform(0.97, 1.03, len(x)) * g.choice([-1.0, 1.0], len(x))
    t = torch.from_numpy(x * scale).to(BF16)
    step = torch.from_numpy(g.integers(-1, 2, x.shape)).to(torch.int16)       # the value itself or its neighbour on either side
    return (t.view(torch.int16) + step).view(BF16).reshape(-1, 128)


def expect(x, unit):
    """(values of the codes, bytes of the scales) by fp32 division."""
    y = x.float().numpy() * (np.float32(1) / np.float32(unit))
    y = y.reshape(-1, 8, 16)
    amax = np.abs(y).max(-1)
    f = torch.from_numpy((amax / np.float32(6)).astype(np.float32)).clamp(max=448.0).to(F8)
    w = f.float().numpy()[..., None]
    q = np.where(w > 0, y / np.where(w > 0, w, np.float32(1)), y * np.float32(0))
    assert q.dtype == np.float32
    return E.VALUES[E.nearest(torch.from_numpy(q).double())].reshape(-1, 128), f.view(torch.uint8)


@pytest.mark.parametrize("units", [(1.0, 2.0 ** -7), (0.1, 3e-3), (0.37, 1e-5), (1.0 / 3.0, 7.0)])
@pytest.mark.parametrize("layout", [None, "half", "interleaved"])
@pytest.mark.parametrize("kernel", ["append", "append_general"])
def test_every_scale_bit_for_bit(libqknorm, monkeypatch, kernel, layout, units):
    if kernel == "append_general":
        monkeypatch.setenv("QKNORM_FORCE_VARIANT", "general")
    units = [float(np.float32(u)) for u in units]
    k, v = (values(u, i) for i, u in enumerate(units))
    T = len(k)
    pos = inv = None
    if layout:                                            # position 0: K goes through the rotation and comes out as it was
        pos, inv = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.rand(64, dtype=torch.float64, device="cuda")
    pages = -(-T // 16)
    codes = [torch.zeros((pages, 16, 1, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((pages, 16, 1, 8), dtype=torch.uint8, device="cuda") for _ in range(2)]
    attn.qknorm_fwd_append_e2m1(None, k.cuda(), v.cuda(), None, None, pos, inv, torch.arange(T, device="cuda"), *codes, *scales, 1e-6,
                                interleaved=layout == "interleaved", k_scale=units[0], v_scale=units[1])
    torch.cuda.synchronize()
    assert binding.last_variant() == kernel
    for x, unit, c, s in zip((k, v), units, codes, scales):
        want, byte = expect(x, unit)
        got_s = s.cpu().view(-1, 8)[:T]
        assert torch.equal(got_s, byte), f"unit {unit}: {(got_s != byte).sum()} of {byte.numel()} scales"
        got = E.VALUES[E.codes_of(c).view(-1, 128)[:T]]
        assert torch.equal(got, want), f"unit {unit}: {(got != want).sum()} of {want.numel()} codes"
        assert len(set(byte.flatten().tolist())) >= 120   # the blocks do have nearly every scale
