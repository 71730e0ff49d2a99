"""sl_rope_*: frequencies and turned rows against their definition in 64 bits (tests/serving_ref.rope_bound counts the roundings)."""
import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import serving_ref as ref
from tests.gpu_util import DEV, dev
from tests.lowbit_ref import f64

pytestmark = pytest.mark.gpu
F, BF = torch.float32, torch.bfloat16
MARK = -77.0


def freqs_on_gpu(rot, theta=10000.0, **kw):
    f = torch.empty(rot // 2, dtype=torch.float64, device=DEV)
    B.sl_rope_freqs(f, theta, **kw)
    return f


@pytest.mark.parametrize("rot", [2, 4, 20, 64, 128, 1024])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "turns"])
def test_freqs(rot, scaling):
    if scaling == "base" and rot == 2:
        return
    got = f64(freqs_on_gpu(rot, 5e5, scaling=scaling, factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=4.0))
    want = ref.rope_freqs(rot, 5e5, scaling, 8.0, 8192.0, 1.0, 4.0)
    assert (np.abs(got / want - 1) < 2.0 ** -47).all()          # a power whose exponent is off by half a step of 14 or so, twice


def rows(m, heads, d, dtype, seed, gap=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, heads * d + gap, generator=g).to(dtype).to(DEV)
    return x[:, :heads * d].view(m, heads, d)


def check(y, x, pos, f, interleaved, amplitude):
    want, mass = ref.rope_rows(f64(x), pos, f64(f), interleaved, amplitude)
    bound = ref.rope_bound(want, mass, torch.finfo(y.dtype).eps)
    err = np.abs(f64(y) - want)
    assert (err <= bound).all(), (err - bound).max()


# rows, bound on them, query heads, key heads, head, turned numbers, most distant position
CASES = [(1, 1, 1, 1, 2, 2, 10), (3, 3, 4, 4, 64, 64, 128), (5, 9, 3, 1, 80, 20, 1 << 20), (17, 17, 32, 8, 128, 64, 1000000), (2, 2, 5, 5, 6, 4, 100), (33, 40, 2, 1, 256, 256, 1 << 30),
         (130, 130, 8, 8, 96, 48, 5000), (1, 1, 1, 1, 1024, 1024, 2 ** 31 - 1), (7, 7, 64, 64, 32, 30, 77), (64, 64, 1, 1, 130, 128, 3000), (9, 9, 6, 3, 24, 8, 4096)]


@pytest.mark.parametrize("m,m_upper,heads,kv,d,rot,most", CASES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("t_in,t_out", [(F, F), (F, BF), (BF, BF), (BF, F)])
def test_rows(m, m_upper, heads, kv, d, rot, most, interleaved, t_in, t_out):
    q, k = rows(m_upper, heads, d, t_in, 1), rows(m_upper, kv, d, t_in, 2)
    q[m:], k[m:] = float("nan"), float("nan")                    # not read
    pos = np.random.default_rng(3).integers(0, most, m_upper)
    pos[0] = most
    f = freqs_on_gpu(rot)
    q_out, k_out = (torch.full(x.shape, MARK, dtype=t_out, device=DEV) for x in (q, k))
    B.sl_rope_rows(q, q_out, k, k_out, f, dev(pos, torch.int32), dev([m], torch.int32), m_upper, interleaved=interleaved, amplitude=1.25)
    for x, y in ((q, q_out), (k, k_out)):
        check(y[:m], x[:m], pos[:m], f, interleaved, 1.25)
        assert (y[m:] == MARK).all()
        assert torch.equal(y[:m, :, rot:], x[:m, :, rot:].to(t_out))


@pytest.mark.parametrize("heads,d,rot,gap", [(4, 64, 64, 0), (4, 64, 64, 8), (4, 64, 32, 3), (3, 128, 128, 1), (2, 80, 20, 5), (8, 128, 64, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F, BF])
def test_in_place_in_a_wider_projection(heads, d, rot, gap, interleaved, dtype):
    """Queries and keys turned where they stand, in rows that lie apart; what is between the rows stays."""
    m, width = 11, heads * d
    whole = torch.randn(m, 2 * width + gap, generator=torch.Generator().manual_seed(5)).to(dtype).to(DEV)
    before = whole.clone()
    q, k = (whole[:, i * width:(i + 1) * width].view(m, heads, d) for i in range(2))
    pos, f = np.arange(m) * 37, freqs_on_gpu(rot)
    B.sl_rope_rows(q, q, k, k, f, dev(pos, torch.int32), dev([m], torch.int32), m, interleaved=interleaved)
    for i, y in enumerate((q, k)):
        x = before[:, i * width:(i + 1) * width].reshape(m, heads, d)
        check(y, x, pos, f, interleaved, 1.0)
        assert torch.equal(y[..., rot:], x[..., rot:])
    assert torch.equal(whole[:, 2 * width:], before[:, 2 * width:])


@pytest.mark.parametrize("offset,gap", [(1, 0), (2, 6), (4, 4), (0, 7)])
@pytest.mark.parametrize("dtype", [F, BF])
def test_rows_that_are_not_aligned(offset, gap, dtype):
    m, heads, d = 6, 4, 64
    store = torch.randn(m * (heads * d + gap) + offset + 8, generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    q = store[offset:offset + m * (heads * d + gap)].view(m, -1)[:, :heads * d].view(m, heads, d)
    out = torch.full((m * (heads * d + gap) + offset,), MARK, dtype=dtype, device=DEV)
    y = out[offset:].view(m, -1)[:, :heads * d].view(m, heads, d)
    pos, f = np.arange(m) + 100, freqs_on_gpu(d)
    B.sl_rope_rows(q, y, None, None, f, dev(pos, torch.int32), dev([m], torch.int32), m)
    check(y, q, pos, f, False, 1.0)
    assert (out[:offset] == MARK).all() and (out[offset:].view(m, -1)[:, heads * d:] == MARK).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_negative_position_turns_back_and_is_the_gradient(interleaved):
    m, heads, d, rot = 8, 4, 64, 48
    x, f, pos = rows(m, heads, d, F, 1), freqs_on_gpu(rot), np.arange(m) * 1001
    y, back = torch.empty_like(x), torch.empty_like(x)
    go = lambda a, b, s: B.sl_rope_rows(a, b, None, None, f, dev(s * pos, torch.int32), dev([m], torch.int32), m, interleaved=interleaved)  # noqa: E731
    go(x, y, 1)
    go(y, back, -1)
    mass = ref.rope_rows(f64(x), pos, f64(f), interleaved, 1.0)[1]
    assert (np.abs(f64(back) - f64(x)) <= 4 * mass * 2.0 ** -24 * 2).all()       # two turns of at most two roundings of a pair, and sine and cosine's
    # d/dx <c, turn(x)> = turn back (c): the turn is linear, so a difference along any direction is exact up to rounding
    c, e = rows(m, heads, d, F, 7), rows(m, heads, d, F, 8)
    ye = torch.empty_like(e)
    go(e, ye, 1)
    go(c, back, -1)
    left, right = (f64(c) * f64(ye)).sum(), (f64(back) * f64(e)).sum()
    assert abs(left - right) <= 2 * 4 * 2.0 ** -24 * (np.abs(f64(c)).sum(-1) * np.abs(f64(e)).sum(-1)).sum()


def test_numbers_that_are_not_finite_stay_in_their_pair():
    m, heads, d = 4, 2, 64
    x = rows(m, heads, d, F, 1).clone()
    x[1, 0, 3], x[2, 1, 40], x[3, 0, 5] = float("nan"), float("inf"), -3e38
    y, f = torch.empty_like(x), freqs_on_gpu(32)
    B.sl_rope_rows(x, y, None, None, f, dev(np.arange(m), torch.int32), dev([m], torch.int32), m)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 0, 3] = bad[1, 0, 19] = True                          # half of 32 apart
    assert torch.isnan(y[bad]).all() and y[2, 1, 40] == float("inf")
    keep = ~bad
    keep[2, 1, 40] = False
    assert torch.isfinite(y[keep]).all()


@pytest.mark.parametrize("count", [0, -4, 99])
def test_row_count_from_the_device(count):
    x, f = rows(5, 2, 32, BF, 1), freqs_on_gpu(32)
    y = torch.full_like(x, MARK)
    B.sl_rope_rows(x, y, None, None, f, dev(np.arange(5), torch.int32), dev([count], torch.int32), 5)
    if count <= 0:
        assert (y == MARK).all()
    else:
        check(y, x, np.arange(5), f, False, 1.0)


def test_same_bits_captured_and_on_another_stream():
    x, f, pos, m = rows(40, 8, 128, BF, 1), freqs_on_gpu(128), dev(np.arange(40) * 99, torch.int32), dev([40], torch.int32)
    ys = [torch.zeros_like(x) for _ in range(3)]
    B.sl_rope_rows(x, ys[0], None, None, f, pos, m, 40)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.sl_rope_rows(x, ys[1], None, None, f, pos, m, 40)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sl_rope_rows(x, ys[2], None, None, f, pos, m, 40)
    for _ in range(3):
        ys[2].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


def turned_exactly(pos, f):
    """cos and sin of 2 pi pos f [rows, pairs], right to 2^-52: f is a fraction over a power of two, so whole turns fall away in whole numbers."""
    turns = np.empty((len(pos), len(f)))
    for j, x in enumerate(f):
        above, below = float(x).as_integer_ratio()
        for i, p in enumerate(pos):
            left = int(p) * above % below
            turns[i, j] = (left if 2 * left <= below else left - below) / below
    return np.cos(2 * np.pi * turns), np.sin(2 * np.pi * turns)


@pytest.mark.parametrize("d", [6, 64])                           # one pair at a time, and four
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("t_in", [F, BF])
def test_sine_and_cosine_are_rounded_once_at_any_position(d, interleaved, t_in):
    """The pairs (1, 0) and (0, 1) turn into sine and cosine alone: half a step of fp32, and 2^-36 for Taylor's sums, whose next terms are below 7e-12."""
    rng = np.random.default_rng(d)
    pos = np.concatenate([[0, 1, -1, 2 ** 31 - 1, -(2 ** 31), 2 ** 28 + 1, -(2 ** 30) - 1], rng.integers(-(2 ** 31), 2 ** 31, 200),
                          rng.integers(2 ** 31 - 10 ** 6, 2 ** 31, 60), rng.integers(-(2 ** 20), 2 ** 20, 60)])
    m, half = len(pos), d // 2
    f = f64(freqs_on_gpu(d))
    f[-1] = 1000.3                                               # a caller's own
    first, second = (slice(0, d, 2), slice(1, d, 2)) if interleaved else (slice(0, half), slice(half, d))
    x = torch.zeros(m, 2, d, dtype=t_in, device=DEV)
    x[:, 0, first] = x[:, 1, second] = 1
    y = torch.empty(m, 2, d, device=DEV)
    B.sl_rope_rows(x, y, None, None, dev(f, torch.float64), dev(pos, torch.int32), dev([m], torch.int32), m, interleaved=interleaved)
    c, s = turned_exactly(pos, f)
    y = f64(y)
    for got, want in ((y[:, 0, first], c), (y[:, 0, second], s), (y[:, 1, first], -s), (y[:, 1, second], c)):
        assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -24 + 2.0 ** -36).all(), np.abs(got - want).max()
