"""sl_kv8_attention on values and queries of very different size, against its definition in 64 bits.

The bound (`bound`) goes by what an error does to the result.  With e = 2^-24 and weights P:
  a score s = scale q . k in fp32: at most 3 d + 16 roundings of its sum of absolute terms (`size`), and the distance to a maximum and
  between maxima 8 more; scores off by at most D each move the result by at most D sum P |v - o| to first order (`spread`), 1.2 of that while
  D < 0.1 -- a sharp softmax forgives what a dot product loses;
  sums over slots, exponentials, the join: slots + 64 roundings of sum P |v| (`mass`);
  bf16: a weight goes in with 22 bits, or to 2^-39 of the row's largest weight times its vector's largest number (`peak`), whichever is coarser;
  probabilities below 2^-126 are zero;
  half a step of the result's type."""
import math

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as ref
from tests.gpu_util import DEV
from tests.test_gpu_kv8 import Case, i32

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
E = 2.0 ** -24


def attention(q, K, V, scale, dtype):
    """q [d], K, V [slots, d], float64 -> (o, bound)."""
    n, d = K.shape
    s = scale * (K @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    o, mass = p @ V, p @ np.abs(V)
    D = (3 * d + 24) * E * scale * np.max(np.abs(K) @ np.abs(q))
    assert D < 0.1
    err = 1.2 * D * (p @ np.abs(V - o)) + (n + 64) * E * mass + n * 2.0 ** -126 * np.abs(V).max()
    if dtype is BF:
        err = err + 2.0 ** -22 * mass + n * 2.0 ** -39 * (p * np.abs(V).max(1)).max()
    return o, err + np.abs(o) * torch.finfo(dtype).eps / 2 * 1.01 + 2.0 ** -149


def filled(k, v, page=64):
    """A cache of sequences k[b], v[b] [slots, heads, d]."""
    c = Case([len(x) for x in k], k[0].shape[1], k[0].shape[2], page, k[0].dtype)
    c.k, c.v = list(k), list(v)
    c.write([list(range(len(x))) for x in k])
    c.K, c.V = [ref.kv8_values(ref.f64(x)) for x in k], [ref.kv8_values(ref.f64(x)) for x in v]
    return c


def check(c, q, got, rows):
    """rows: the sequence of each row; every row sees its whole sequence."""
    share = q.shape[1] // c.heads
    for r, b in enumerate(rows):
        for h in range(q.shape[1]):
            want, bound = attention(ref.f64(q[r, h]), c.K[b][:, h // share], c.V[b][:, h // share], 1.0 / math.sqrt(c.d), c.dtype)
            err = np.abs(got[r, h] - want)
            assert (err <= bound).all(), (b, r, h, float(np.nanmax(err / bound)), float(np.abs(want).max()))


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("large", [1e4, 1e8, 1e12, 1e20])
@pytest.mark.parametrize("at", [5, 300, 399])
def test_small_values_that_take_the_weight_from_large_ones(dtype, large, at):
    """One slot far ahead of the others (2^90 in weight), its value ordinary, the others' large: read before, between and after them."""
    d, n = 64, 400
    k, v = 0.01 * randn(1, n, 1, d), large * randn(2, n, 1, d)
    k[at] = 0
    k[at, :, 0] = 90 * math.log(2) * math.sqrt(d)
    v[at] = randn(3, 1, d)
    c = filled([k.to(dtype)], [v.to(dtype)])
    q = torch.zeros(1, 1, d)
    q[..., 0] = 1
    q, got = c.attend([1], 1, q=q.to(dtype))
    check(c, q, got, [0])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("falling", [False, True])
def test_weights_that_rise_step_by_step(dtype, falling):
    """Scores that rise by 5 (in powers of two) from one group of 128 slots to the next, values that fall by 2^10: each group takes the result over."""
    d, n = 64, 512
    group = torch.arange(n) // 128
    k, v = torch.zeros(n, 1, d), randn(4, n, 1, d) * 2.0 ** (-10.0 * group)[:, None, None]
    k[:, 0, 0] = 5 * math.log(2) * math.sqrt(d) * group
    if falling:
        k, v = k.flip(0).contiguous(), v.flip(0).contiguous()
    c = filled([k.to(dtype)], [v.to(dtype)])
    q = torch.zeros(1, 1, d)
    q[..., 0] = 1
    q, got = c.attend([1], 1, q=q.to(dtype))
    check(c, q, got, [0])


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("outlier", [1.0, 1e4, 1e6, 1e12])
def test_fp32_queries_with_one_number_far_above_the_others(d, outlier):
    """The keys hold nothing in that dimension (or little), so the scores are the others'.  fp32 keeps each number's own 24 bits."""
    n, heads, share = 700, 2, 3
    k, v, q = randn(5, n, heads, d), randn(6, n, heads, d), randn(7, 2, heads * share, d)
    k[:, :, 5] = 0
    q[..., 5] = outlier * (1 + torch.arange(2 * heads * share).view(2, -1) / 8)
    c = filled([k], [v])
    q, got = c.attend([2], share, q=q)
    check(c, q, got, [0, 0])


def test_bf16_queries_with_one_number_far_above_the_others():
    """Up to 2^15 times the others' size nothing of theirs is lost."""
    d, n = 128, 300
    k, v, q = randn(5, n, 1, d).to(BF), randn(6, n, 1, d).to(BF), (randn(7, 2, 1, d).sign() * (1 + randn(8, 2, 1, d).abs() / 8)).to(BF)
    k[:, :, 5] = 0
    q[..., 5] = 2.0 ** 14
    c = filled([k], [v])
    q, got = c.attend([2], 1, q=q)
    check(c, q, got, [0, 0])


@pytest.mark.parametrize("outlier", [1e4, 1e18])
@pytest.mark.parametrize("dtype", [BF, F])
def test_scores_of_large_queries_and_small_keys(dtype, outlier):
    """Only the products have to be of ordinary size."""
    d, n = 64, 200
    k, v, q = randn(9, n, 1, d) / outlier, randn(10, n, 1, d), randn(11, 2, 1, d) * outlier
    c = filled([k.to(dtype)], [v.to(dtype)])
    q, got = c.attend([2], 1, q=q.to(dtype))
    check(c, q, got, [0, 0])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 256])
def test_values_near_the_largest_finite_number(dtype, d):
    """A weighted mean of finite values is finite: sums are normalised before they leave their power of two, within a wave, between
    waves and between partial results."""
    lens = [40, 700, 3000]
    k, v = [0.1 * randn(12 + n, n, 1, d) for n in lens], [3e38 * (randn(13, 1, 1, d).sign() * (1 - randn(n, n, 1, 1).abs() / 64)) for n in lens]
    c = filled([x.to(dtype) for x in k], [x.to(dtype) for x in v])
    q, got = c.attend([1, 2, 1], 1, q=randn(14, 4, 1, d).to(dtype))
    assert np.isfinite(got).all()
    check(c, q, got, [0, 1, 1, 2])


@pytest.mark.parametrize("dtype", [BF, F])
def test_values_near_the_smallest_normal_number(dtype):
    d, lens = 64, [40, 3000]
    k, v = [randn(15 + n, n, 1, d) for n in lens], [2.0 ** -112 * randn(n, n, 1, d) for n in lens]
    c = filled([x.to(dtype) for x in k], [x.to(dtype) for x in v])
    q, got = c.attend([1, 1], 1, q=randn(16, 2, 1, d).to(dtype))
    check(c, q, got, [0, 1])


@pytest.mark.parametrize("dtype", [BF, F])
def test_numbers_that_are_not_finite_stay_with_their_rows(dtype):
    """A NaN or an infinity in a query or in a slot that it sees makes that query's result NaN; every other one is exact, and a row that
    sees nothing is zeros whatever its query holds."""
    d, n = 64, 700
    k, v = randn(20, n, 2, d), randn(21, n, 2, d)
    c = filled([k.to(dtype)], [v.to(dtype)])
    broken_k, broken_v = k.clone(), v.clone()
    broken_k[600, 0, 3], broken_v[650, :, 5] = float("nan"), -float("inf")
    B.sl_kv8_write(c.kv, broken_k.to(dtype).to(DEV), broken_v.to(dtype).to(DEV), i32(range(n)), i32([0, n]), n)
    limits = [500, 600, 601, 651, 0, 300, 1]
    q = randn(22, 7, 2, d)
    q[4], q[5, 1, 7] = float("nan"), float("inf")
    q, got = c.attend([7], 1, row_len=limits, q=q.to(dtype))
    assert (got[4] == 0).all()
    assert np.isnan(got[2, 0]).all() and np.isnan(got[3]).all() and np.isnan(got[5, 1]).all()
    for r, h in ((0, 0), (0, 1), (1, 0), (1, 1), (2, 1), (5, 0), (6, 0), (6, 1)):
        want, bound = attention(ref.f64(q[r, h]), c.K[0][:limits[r], h], c.V[0][:limits[r], h], 1.0 / math.sqrt(d), dtype)
        assert (np.abs(got[r, h] - want) <= bound).all(), (r, h)
