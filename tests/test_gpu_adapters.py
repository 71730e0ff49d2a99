"""sl_adapters_*: a low-rank adapter for each row beside a shared projection, against its definition in 64 bits (tests/serving_ref.adapters counts the
roundings), plus half a step of the result's type."""
import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import serving_ref as ref
from tests.gpu_util import DEV, dev
from tests.lowbit_ref import f64, half_step

pytestmark = pytest.mark.gpu
F, BF = torch.float32, torch.bfloat16
MARK = -77.0


def bank(n_slots, max_rank, n, k, ranks, seed):
    """A bank with some slots filled: {slot: rank}; the pool starts as NaN, so that nothing unwritten can go unseen."""
    ad = B.Adapters(n_slots, max_rank, n, k)
    ad.bank.fill_(0xFF)
    B.sl_adapters_init(ad)
    g, weights = torch.Generator().manual_seed(seed), {}
    for slot, rank in ranks.items():
        a, b = torch.randn(rank, k, generator=g).to(BF) / 8, torch.randn(n, rank, generator=g).to(BF) / 8
        B.sl_adapters_pack(ad, slot, a.to(DEV), b.to(DEV), 0.5 + slot)
        weights[slot] = (f64(a), f64(b), 0.5 + slot)
    return ad, weights


def forward(ad, x, which, m, m_upper, base, out, y=None):
    y = torch.full((m_upper, ad.n), MARK, dtype=out, device=DEV) if y is None else y
    ws = torch.full((max(256, B.sl_adapters_workspace_bytes(ad, m_upper)),), 0xFF, dtype=torch.uint8, device=DEV)
    B.sl_adapters_forward(ad, x, dev(which, torch.int32), dev([m], torch.int32), m_upper, ws, base=base, splits=1 if base is None else base.shape[0],
                          **{"y_bf16" if out is BF else "y_f32": y})
    return y


def check(y, x, base, which, weights, rows=None):
    want, bound = ref.adapters(f64(x), None if base is None else f64(base), list(which), weights)
    bound = bound + half_step(np.abs(want) + bound, y.dtype) * 1.01
    err = np.abs(f64(y) - want)
    rows = slice(None) if rows is None else rows
    assert (err[rows] <= bound[rows]).all(), (err - bound)[rows].max()


def inputs(m_upper, n, k, splits, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m_upper, k, generator=g).to(BF).to(DEV)
    return x, torch.randn(splits, m_upper, n, generator=g).to(DEV) if splits else None


# rows, bound, outputs, inputs, slots, largest rank, partial sums of the base (0: none), rows of one adapter together
CASES = [
    (1, 1, 1, 8, 1, 1, 1, 1), (1, 1, 64, 64, 4, 16, 1, 1), (1, 2, 33, 40, 2, 3, 0, 1), (3, 3, 688, 256, 5, 8, 1, 1), (16, 16, 256, 688, 16, 16, 2, 1), (17, 20, 100, 1000, 3, 17, 1, 2),
    (40, 40, 130, 520, 7, 64, 1, 5), (64, 64, 512, 4096, 64, 16, 1, 1), (65, 70, 48, 2056, 4, 33, 3, 30), (200, 200, 272, 512, 6, 128, 1, 60), (33, 33, 1040, 136, 2, 256, 0, 16),
    (300, 320, 80, 4096, 9, 16, 1, 1), (5, 5, 4096, 264, 3, 12, 4, 2), (130, 130, 36, 12288, 2, 48, 1, 130), (513, 513, 96, 72, 20, 32, 1, 40),
]


@pytest.mark.parametrize("m,m_upper,n,k,slots,max_rank,splits,run", CASES)
@pytest.mark.parametrize("out", [F, BF])
def test_forward(m, m_upper, n, k, slots, max_rank, splits, run, out):
    rng = np.random.default_rng(m + n)
    ranks = {s: [max_rank, 1, max(1, max_rank - 1), max(1, max_rank // 2)][s % 4] for s in range(slots) if s % 5 != 3}      # (some slots stay empty)
    ad, weights = bank(slots, max_rank, n, k, ranks, n + k)
    which = np.repeat(rng.integers(-1, slots + 1, m_upper), run)[:m_upper]                # -1 and `slots`: no adapter
    x, base = inputs(m_upper, n, k, splits, 3)
    x[m:] = float("nan")
    if base is not None:
        base[:, m:] = float("nan")
    y = forward(ad, x, which, m, m_upper, base, out)
    assert (y[m:] == MARK).all()
    check(y[:m], x[:m], base[:, :m] if base is not None else None, which[:m], weights) if weights else None


# the other forms that sizes choose: more rank tiles a workgroup, more columns a wave
LARGE = [(520, 520, 1041, 72, 6, 256, 1, 9), (700, 703, 801, 136, 5, 80, 0, 11), (1030, 1030, 528, 520, 4, 80, 2, 40), (513, 515, 4099, 264, 7, 16, 1, 50), (520, 520, 4100, 136, 3, 40, 1, 33),
         (2040, 2050, 20, 24, 2, 64, 1, 100), (2040, 2050, 1040, 8, 2, 32, 0, 1)]


@pytest.mark.parametrize("m,m_upper,n,k,slots,max_rank,splits,run", LARGE)
@pytest.mark.parametrize("out", [F, BF])
def test_forward_of_many_rows(m, m_upper, n, k, slots, max_rank, splits, run, out):
    test_forward(m, m_upper, n, k, slots, max_rank, splits, run, out)


@pytest.mark.parametrize("ids", [[-5, 2 ** 31 - 1, 3, -2 ** 31], [1, 1, 1, 1], [0, 1, 0, 1], [2, 2, 2, 0]])
def test_ids_that_name_no_adapter_get_the_base_alone(ids):
    ad, weights = bank(3, 16, 72, 64, {0: 16, 1: 5}, 1)          # slot 2 is empty
    x, base = inputs(4, 72, 64, 2, 4)
    y = forward(ad, x, ids, 4, 4, base, F)
    check(y, x, base, ids, weights)
    for r, i in enumerate(ids):
        if i not in (0, 1):
            assert torch.equal(y[r], base[0, r] + base[1, r])


@pytest.mark.parametrize("m,n", [(1, 40), (37, 96), (37, 97)])
def test_in_place(m, n):
    ad, weights = bank(4, 8, n, 128, {0: 8, 1: 4, 3: 7}, 2)
    which = np.arange(m) % 5 - 1
    x, base = inputs(m, n, 128, 1, 5)
    y = base.clone()
    forward(ad, x, which, m, m, y, F, y=y[0])
    check(y[0], x, base, which, weights)


def test_broken_rows_and_broken_adapters_stay_apart():
    """NaN and infinities in a row, and in an adapter's weights, reach that row, and that adapter's rows, alone."""
    ad, weights = bank(4, 16, 64, 96, {0: 16, 1: 9, 2: 16}, 3)
    a, b = torch.full((16, 96), float("nan"), dtype=BF, device=DEV), torch.full((64, 16), float("inf"), dtype=BF, device=DEV)
    B.sl_adapters_pack(ad, 3, a, b, 1.0)
    which = np.array([0, 1, 2, 3] * 5 + [-1, 1])
    x, base = inputs(22, 64, 96, 1, 6)
    x[5, 7], x[9, 3], x[20, 0] = float("nan"), float("inf"), float("nan")        # row 20 has no adapter: its x is nobody's
    y = forward(ad, x, which, 22, 22, base, F)
    bad = [r for r in range(22) if which[r] == 3 or r in (5, 9)]
    assert torch.isnan(y[bad]).all()
    good = [r for r in range(22) if r not in bad]
    x[[5, 9, 20]] = 0
    check(y, x, base, np.where(which == 3, -1, which), weights, good)
    assert torch.equal(y[20], base[0, 20])


def test_sizes_of_rows_and_scales_far_apart():
    ad, weights = bank(3, 16, 48, 256, {0: 16, 1: 16, 2: 16}, 8)
    a, b, _ = weights[1]
    for slot, scale in ((0, 2.0 ** -60), (1, -(2.0 ** 40)), (2, 0.0)):
        a, b, _ = weights[slot]
        B.sl_adapters_pack(ad, slot, dev(a, BF), dev(b, BF), scale)
        weights[slot] = (a, b, scale)
    which = np.arange(18) % 3
    x, base = inputs(18, 48, 256, 1, 9)
    x[::2] *= 2.0 ** 30
    y = forward(ad, x, which, 18, 18, base, F)
    check(y, x, base, which, weights)


def test_a_slot_taken_over_by_another_adapter_and_emptied():
    ad, weights = bank(2, 16, 40, 64, {0: 16, 1: 16}, 4)
    x, base = inputs(3, 40, 64, 1, 7)
    a, b = torch.randn(3, 64).to(BF), torch.randn(40, 3).to(BF)
    B.sl_adapters_pack(ad, 0, a.to(DEV), b.to(DEV), 2.0)         # of a lower rank than what was there
    weights[0] = (f64(a), f64(b), 2.0)
    check(forward(ad, x, [0, 1, 0], 3, 3, base, F), x, base, [0, 1, 0], weights)
    B.sl_adapters_pack(ad, 0, None, None)
    y = forward(ad, x, [0, 1, 0], 3, 3, base, F)
    check(y, x, base, [-1, 1, -1], weights)
    assert torch.equal(y[0], base[0, 0])


@pytest.mark.parametrize("count", [0, -3, 50])
def test_row_count_from_the_device(count):
    ad, weights = bank(2, 16, 40, 64, {0: 16, 1: 16}, 4)
    x, base = inputs(6, 40, 64, 1, 7)
    y = forward(ad, x, [0, 1, 0, -1, 1, 1], count, 6, base, F)
    if count <= 0:
        assert (y == MARK).all()
    else:
        check(y, x, base, [0, 1, 0, -1, 1, 1], weights)


def test_beside_the_framework_s_products():
    """A k-split projection's planes, and a 4-bit one's result, as the base."""
    m, n, k = 20, 128, 4096
    ad, weights = bank(3, 16, n, k, {0: 16, 1: 8, 2: 3}, 5)
    x, _ = inputs(m, n, k, 0, 8)
    w = (torch.randn(n, k, generator=torch.Generator().manual_seed(1)) / 64).to(BF).to(DEV)
    packed, count = torch.empty_like(w), dev([m], torch.int32)
    B.sl_linear_pack(w, packed)
    splits = B.sl_linear_splits(m, n, k)
    planes = torch.empty(splits, m, n, device=DEV)
    B.sl_linear_forward(x, packed, count, m, n, k, y_f32=planes)
    which = np.arange(m) % 4 - 1
    y = forward(ad, x, which, m, m, planes, BF)
    check(y, x, planes, which, weights)


def test_same_bits_captured_and_on_another_stream():
    ad, weights = bank(5, 32, 512, 2048, {s: 32 - s for s in range(5)}, 6)
    x, base = inputs(50, 512, 2048, 2, 9)
    which, m, ws = dev(np.arange(50) // 7 - 1, torch.int32), dev([50], torch.int32), [
        torch.empty(B.sl_adapters_workspace_bytes(ad, 50), dtype=torch.uint8, device=DEV) for _ in range(2)]
    ys = [torch.zeros(50, 512, dtype=BF, device=DEV) for _ in range(3)]
    call = lambda i, w: B.sl_adapters_forward(ad, x, which, m, 50, ws[w], base=base, splits=2, y_bf16=ys[i])  # noqa: E731
    call(0, 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        call(1, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(2, 1)
    for _ in range(3):
        ys[2].zero_()
        ws[1].fill_(0xFF)
        call(0, 0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


# rows, outputs, largest rank: one, two and four column tiles a wave, and the first product's forms
@pytest.mark.parametrize("m,n,max_rank", [(6, 33, 16), (40, 72, 40), (260, 4100, 16), (520, 4100, 40), (2050, 1040, 64)])
@pytest.mark.parametrize("out", [F, BF])
def test_infinite_weights_of_the_second_product(m, n, max_rank, out):
    """An infinity in B is one in its output (NaN where two of different signs meet), for the rows of its adapter alone, and leaves other outputs as they are."""
    ad, weights = bank(3, max_rank, n, 64, {0: max_rank, 1: max(1, max_rank - 3), 2: 1}, 11)
    a, b, scale = weights[0]
    hit = b.copy()
    hit[3, max_rank // 2], hit[n - 1, 0], hit[17, [0, max_rank - 1]], hit[5, 1] = np.inf, -np.inf, [np.inf, -np.inf], np.nan
    B.sl_adapters_pack(ad, 0, dev(a, BF), dev(hit, BF), scale)
    which = np.arange(m) % 5 - 1
    x, base = inputs(m, n, 64, 1, 12)
    y = forward(ad, x, which, m, m, base, out)
    mine, cols = np.nonzero(which == 0)[0], [3, n - 1, 17, 5]
    with np.errstate(invalid="ignore"):
        want = scale * (f64(x)[mine] @ a.T) @ hit.T[:, cols]
    assert np.array_equal(f64(y)[mine][:, cols], want, equal_nan=True) and np.isinf(want[:, :2]).all() and np.isnan(want[:, 3]).all()
    weights[0] = (a, np.where(np.isfinite(hit), hit, 0), scale)
    y[torch.as_tensor(mine, device=DEV)[:, None], torch.as_tensor(cols, device=DEV)] = 0
    w, bound = ref.adapters(f64(x), f64(base), list(which), weights)
    w[np.ix_(mine, cols)] = 0
    assert (np.abs(f64(y) - w) <= bound + half_step(np.abs(w) + bound, out) * 1.01).all()


@pytest.mark.parametrize("m,n,k,max_rank", [(5, 40, 64, 16), (33, 100, 520, 40), (260, 4100, 64, 16), (520, 4100, 1032, 40), (1030, 48, 136, 64), (2050, 1040, 64, 64)])
def test_all_bits_of_the_first_product_reach_the_second(m, n, k, max_rank):
    """A x is a whole number of 24 bits over 2^16, from three products, and B picks one of its numbers for each output: what comes out may be off by a step of fp32
    (2^-23) for each of the four sums that are not of zeros.  Sixteen of the 24 bits would not do."""
    rng = np.random.default_rng(m + n)
    ad, weights = B.Adapters(3, max_rank, n, k), {}
    for slot, rank in enumerate((max_rank, max_rank - 1, 7)):
        a = rng.choice([-1, 1], (rank, k)) * (129 + 2 * rng.integers(0, 64, (rank, k)))
        b = np.zeros((n, rank))
        b[np.arange(n), np.arange(n) % rank] = rng.choice([-1, 1, 0.5], n)
        B.sl_adapters_pack(ad, slot, dev(a, BF), dev(b, BF), 1.0)
        weights[slot] = (a, b)
    x = np.zeros((m, k))
    for r in range(m):
        x[r, rng.choice(k, 3, replace=False)] = [1, 2.0 ** -8, 2.0 ** -16]
    which = rng.integers(0, 3, m)
    y = f64(forward(ad, dev(x, BF), which, m, m, None, F))
    for slot, (a, b) in weights.items():
        rows = which == slot
        if not rows.any():
            continue
        h = x[rows] @ a.T
        want = h @ b.T
        assert (np.abs(y[rows] - want) <= np.abs(want) * 2.0 ** -21).all()
        high = f64(torch.tensor(h).to(BF))
        cut = (high + f64(torch.tensor(h - high).to(BF))) @ b.T
        assert (np.abs(cut - want) > np.abs(want) * 2.0 ** -21).mean() > 0.5
