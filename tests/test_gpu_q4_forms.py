"""sl_linear_q4_*: weights at the ends of fp32, and every tile that the product is cut by, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as ref
from tests.gpu_util import DEV, dev
from tests.test_gpu_q4 import check, make, packed_of

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


# ---- every tile ---------------------------------------------------------------------------------
def tile(n, k, m_upper):
    """The rule of slk_q4_linear: rows x columns, waves side by side x waves along the reduction."""
    rows16, tiles_n, blocks_k = -(-m_upper // 16), -(-n // 16), -(-k // 128)
    if rows16 >= 3 and -(-n // 128) * -(-m_upper // 32) >= 192:
        return "32x128,4x2"
    if rows16 >= 3:
        return "32x32,1x8"
    if rows16 == 1 and tiles_n <= 256 and blocks_k >= 16:
        return "16x16,1x16"
    return "16x32,1x8" if tiles_n * rows16 <= 512 else "16x48,1x8"


# n, k, rows, bound: reductions shorter than the waves and not a multiple of them, ends inside a block, row tiles that are full, ragged or
# past the count, columns that end inside a tile and inside a workgroup's
FORMS = {
    "16x48,1x8": [(8200, 136, 1, 1), (12296, 1000, 16, 16), (4120, 8, 19, 32), (8248, 2184, 7, 16), (4300, 648, 32, 32)],
    "32x128,4x2": [(3000, 8, 250, 256), (3500, 136, 199, 224), (4130, 392, 97, 224), (3000, 1160, 256, 256), (6200, 264, 33, 128),
                   (12300, 648, 50, 64), (3500, 904, 1, 224)],
    "16x16,1x16": [(100, 2056, 16, 16), (1, 2184, 1, 1), (1040, 4104, 9, 16), (33, 2048, 3, 5)],
    "32x32,1x8": [(130, 264, 45, 48), (520, 1160, 64, 64), (33, 8, 33, 40), (2900, 136, 100, 250)],
    "16x32,1x8": [(40, 8, 1, 1), (700, 2184, 30, 32), (4100, 2056, 5, 16), (17, 1024, 17, 17)],
}


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("form,n,k,m,m_upper", [(f, *c) for f, cs in FORMS.items() for c in cs])
def test_every_tile(form, n, k, m, m_upper, group, zeros):
    assert tile(n, k, m_upper) == form
    codes, scales, z = make(n, k, group, zeros, n + k + group)
    packed = packed_of(codes, scales, z, zeros, group)
    x = torch.randn(m_upper, k, generator=torch.Generator().manual_seed(m)).bfloat16()
    x[m:] = float("nan")                                          # rows behind the count are not read
    dt = torch.float32 if zeros else torch.bfloat16
    y = torch.full((m_upper, n), -77.0, dtype=dt, device=DEV)
    B.sl_linear_q4_forward(x.to(DEV), packed, dev([m], torch.int32), m_upper, n, k, group, **{"y_f32" if zeros else "y_bf16": y})
    got = ref.f64(y)
    assert (got[m:] == -77.0).all()
    check(got[:m], ref.f64(x[:m]), codes, scales, z, group, dt)


def test_rows_of_a_large_tile_go_where_the_map_says():
    n, k, m, group = 3500, 392, 199, 64
    assert tile(n, k, 224) == "32x128,4x2"
    codes, scales, z = make(n, k, group, True, 3)
    x = torch.randn(224, k, generator=torch.Generator().manual_seed(4)).bfloat16()
    to = torch.randperm(300, generator=torch.Generator().manual_seed(5))[:224].tolist()
    y = torch.full((300, n), -77.0, dtype=torch.bfloat16, device=DEV)
    B.sl_linear_q4_forward(x.to(DEV), packed_of(codes, scales, z, True, group), dev([m], torch.int32), 224, n, k, group, y_bf16=y,
                           row_map=dev(to, torch.int32))
    got = ref.f64(y)
    check(got[to[:m]], ref.f64(x[:m]), codes, scales, z, group, torch.bfloat16)
    assert (got[[r for r in range(300) if r not in to[:m]]] == -77.0).all()
