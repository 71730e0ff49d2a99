"""sl_linear_q4_*: weights at the ends of fp32, and every tile that the product is cut by, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as ref
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_of_a_range_that_fp32_does_not_hold(dtype, group):
    """hi - lo overflows, every weight is finite: the scale is that of hi / 15 - lo / 15, and the weights come back."""
    k = 2 * group + 8
    w = torch.randn(3, k, generator=torch.Generator().manual_seed(2))
    w[1, 3], w[1, 5], w[1, 7] = 3e38, -2.5e38, 1e38                         # first group of one row; the other groups are ordinary
    w = w.to(dtype)
    c = torch.full((3, k // 2), 0xEE, dtype=torch.uint8, device=DEV)
    s, zp = torch.empty(3, 3, dtype=torch.bfloat16, device=DEV), torch.empty(3, 3, dtype=torch.uint8, device=DEV)
    B.sl_linear_q4_quantize(w.to(DEV), group, c, s, zp)
    codes, scales, z = ref.q4_quantize(np.where(np.abs(ref.f64(w)) > 1e30, 0, ref.f64(w)), group, True)
    got = np.stack([c.cpu().numpy() & 15, c.cpu().numpy() >> 4], -1).reshape(3, k)
    keep = np.ones((3, 3), bool)
    keep[1, 0] = False
    assert np.array_equal(ref.f64(s)[keep], scales[keep]) and np.array_equal(zp.cpu().numpy()[keep], z[keep])
    own = ref.f64(w)[1, :group]
    scale = ref.bf16(own.max() / 15 - own.min() / 15)
    assert ref.f64(s)[1, 0] == scale and zp.cpu().numpy()[1, 0] == np.clip(np.rint(-own.min() / scale), 0, 15)
    held = ref.q4_weights(got[1:2, :group], ref.f64(s)[1:2, :1], zp.cpu().numpy()[1:2, :1], group)[0]
    # half a step, half a step of the zero point, and what the scale's rounding leaves out at the ends
    assert (np.abs(held - own) <= scale * (1.0 + 15 * 2.0 ** -8)).all()
