"""Appending to blocks whose rows were written by something else, with scales that appending never writes: a byte s from 1 to 246 is 2^(s - 127), below 1 as 1, above 246
as 246, and the rows that a block has keep the values that it makes of them."""
import numpy as np
import pytest
import torch

from byte_util import LEAST, Problem8, exponents, numbers, rounded, same_bytes
from gpu_util import TORCH_DT, require_gpu
from test_gpu_byte_append import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,block", [(32, 4), (48, 16), (256, 128)], ids=["16 lanes", "64 lanes", "256 lanes"])
@pytest.mark.parametrize("held", [0, 1, 5, 9, 10, 11, 126, 246, 247, 255])
@pytest.mark.parametrize("size", [0.0, 2.0 ** -116, 1.0, 2.0 ** 100])
def test_rows_keep_their_values(dtype, d, block, held, size):
    """One new token into a block that has some.  2^-116 is below what the least scale of an appended block is for."""
    n = block // 2
    p = Problem8(dtype, [(1, n + 1)], 1, 1, d, block, block, seed=held).on_gpu()
    page = int(p.table[0, 0])
    for name in ("K", "V"):
        scales = getattr(p, name + "_scales")
        scales[page] = held
        p.dev[name + "_scales"].copy_(scales)
    g = torch.Generator().manual_seed(held)
    x = (size * torch.randn((1, 3 * d), generator=g)).to(TORCH_DT[dtype])
    run(p, x, 0, heads=1)
    old = min(max(held, 1), 246) - 127
    for i, name in enumerate("KV"):
        new = x[:, (1 + i) * d:(2 + i) * d].float()
        e = max(int(exponents(new.double().abs().amax().numpy())), LEAST, old)
        want, want_scales = getattr(p, name + "8").clone(), getattr(p, name + "_scales").clone()
        before = want[page, 0, :n].clone()
        if e > old:
            want[page, 0, :n] = rounded(numbers(before), e - old)
        want[page, 0, n] = rounded(new[0], e)
        want_scales[page, 0, 0] = e + 127
        same_bytes(p.dev[name + "8"], want, name)
        assert torch.equal(p.dev[name + "_scales"].cpu(), want_scales), name
        if e - old <= 3:                          # (what the block's rows stand for: in 64 bits, to half of the new scale's least number)
            was, now = (numbers(b).double().numpy() * 2.0 ** s for b, s in ((before, old), (p.dev[name + "8"].cpu()[page, 0, :n], e)))
            both = ~np.isnan(was)
            assert (np.isnan(now) == ~both).all() and (np.abs(now - was)[both] <= np.maximum(2.0 ** (e - 10), np.abs(was)[both] * 2.0 ** -4)).all()
