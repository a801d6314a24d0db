"""Values of a cache in 8 bits near the end of what sums of them can hold: the slots that a row sees times the largest value up to 2^122."""
import pytest
import torch

from byte_util import Problem8
from gpu_util import require_gpu
from test_gpu_byte_attention import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("kernel", ["rows", "tiles"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 96, 128, 160, 256])
@pytest.mark.parametrize("n,block", [(1290, 32), (1322, 2), (40, 8)])
def test_large_values(monkeypatch, kernel, dtype, d, n, block):
    monkeypatch.setenv("ATTNW_PAGED_KERNEL", kernel)
    e = 102 if n > 40 else 107                    # 1322 slots of 448 2^102: 2^121.2; 40 of 448 2^107: 2^121.1
    p = Problem8(dtype, [(min(n, 70), n)], 2, 1, d, 32, block, seed=n + d, sharp=2.0)
    p.Q[3:9] = 0                                  # (the same weight for every slot)
    p.Q[20:24] *= 8                               # (scores that run ahead)
    p.V_scales[:] = 127 + e
    p.V8[..., 2:6] = 0x7e                         # 448
    p.V8[..., 9] = 0xfe
    O, lse = check(p.restate())
    assert bool(torch.isfinite(O[:p.T].float()).all())
    p.V_scales[:] = 246                           # the greatest there is: a single token that sees one slot has its value
    q = Problem8(dtype, [(1, 1)], 2, 1, d, 32, block, seed=n + d)
    q.V_scales[:] = 246
    O, _ = check(q.restate())
    assert bool(torch.isfinite(O.float()).all())
