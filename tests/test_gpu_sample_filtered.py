"""sl_sample_filtered against its definition: tokens and counts are whole numbers and compared for equality, probabilities to a rounding.

A weight that the definition rounds may come out one unit (2^-44 of the largest) beside the reference's where exp() is off by its last bit,
so inputs here keep their draws from borders by being what they are: a border within 2^-44 of a uniform number of 24 bits
is one of 2^20; cases that sit on a border on purpose use weights that are exact."""
import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import serving_ref as ref
from tests.gpu_util import DEV, dev
from tests.lowbit_ref import f64

pytestmark = pytest.mark.gpu
F, BF = torch.float32, torch.bfloat16
INF = float("inf")


def draw(logits, u, rows=None, m=None, row_map=None, **filters):
    m_upper = len(u)
    token, kept = (torch.full((m_upper,), -77, dtype=torch.int32, device=DEV) for _ in range(2))
    prob = torch.full((m_upper,), -77.0, device=DEV)
    ws = torch.full((max(256, B.sl_sample_filtered_bytes(m_upper, logits.shape[1])),), 0xFF, dtype=torch.uint8, device=DEV)
    B.sl_sample_filtered(logits, dev([m_upper if m is None else m], torch.int32), m_upper, dev(u, F), token, ws, prob=prob, kept=kept,
                         row_map=None if row_map is None else dev(row_map, torch.int32),
                         **{n: None if v is None else dev(v, torch.int32 if n == "top_k" else F) for n, v in filters.items()})
    return token.tolist(), prob.tolist(), kept.tolist()


def check(logits, u, got, row_map=None, **filters):
    z, u = f64(logits), np.asarray(u, np.float32).astype(np.float64)
    for r in range(len(u)):
        f = {n: float(np.float32(v[r])) if n != "top_k" else int(v[r]) for n, v in filters.items() if v is not None}
        token, prob, kept = ref.sample(z[r if row_map is None else row_map[r]], u[r], **f)
        assert (got[0][r], got[2][r]) == (token, kept), (r, got[0][r], got[2][r], token, kept, f)
        assert abs(got[1][r] - prob) <= prob * 2.0 ** -23 + 2.0 ** -43, r      # its own rounding; the token's weight and the sum a unit off


def bell(m, vocab, dtype, seed, spread=2.0):
    """Most of the vocabulary in a bell, a few tokens far above, some forbidden."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(m, vocab, generator=g) * spread
    z.scatter_add_(1, torch.randint(0, vocab, (m, 8), generator=g), torch.rand(m, 8, generator=g) * 9)
    z[:, vocab // 2:vocab // 2 + vocab // 50] = -INF
    return z.to(dtype).to(DEV)


KINDS = {
    "plain": {}, "cold": dict(temperature=[0.3]), "greedy": dict(temperature=[0.0]), "k1": dict(top_k=[1]), "k5": dict(top_k=[5]), "k50": dict(top_k=[50, 40, 7]),
    "k1000": dict(top_k=[1000]), "k1500": dict(top_k=[1500, 1024, 1025]), "k_all": dict(top_k=[1 << 30, -1, 0]), "p9": dict(top_p=[0.9, 0.5]),
    "p_low": dict(top_p=[1e-6, 0.0, -1.0]), "p_high": dict(top_p=[0.999999, 1.0, 2.0]), "min": dict(min_p=[0.05, 0.0, 1.0, 3.0]), "nan": dict(temperature=[float("nan"), 1], top_p=[float("nan")], min_p=[float("nan")]),
    "kp": dict(top_k=[50], top_p=[0.9], temperature=[1.0, 0.7]), "all": dict(top_k=[0, 300], top_p=[0.95, 0.8], min_p=[0.01, 0.0], temperature=[1.0, 1.4, 0.6, 0.0, INF]),
    "pm": dict(top_p=[0.97], min_p=[0.001], temperature=[2.0]),
}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 1000, 1024, 8197, 33001])
@pytest.mark.parametrize("dtype", [F, BF])
def test_draws(kind, vocab, dtype):
    m = 12
    logits = bell(m, vocab, dtype, vocab)
    u = np.random.default_rng(vocab).random(m).astype(np.float32)
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    filters = {n: np.resize(np.array(v, dtype=np.float64), m) for n, v in KINDS[kind].items()}
    check(logits, u, draw(logits, u, **filters), **filters)


@pytest.mark.parametrize("vocab,dtype", [(126464, BF), (126464, F), (1 << 18, BF), (262143, F), (126463, BF)])
def test_large_vocabularies(vocab, dtype):
    m = 10
    logits = bell(m, vocab, dtype, 3)
    u = np.random.default_rng(1).random(m).astype(np.float32)
    filters = dict(top_k=np.array([0, 50, 0, 5000, 0, 1000, 0, 0, 70000, 0]), top_p=np.array([.9, .9, 1, .8, .99, 1, .5, .95, .9, .2]),
                   min_p=np.array([0, 0, .01, 0, .001, 0, .3, 0, 0, 0]), temperature=np.array([1, 1, 1, .7, 2, 1, 1, .25, 1.5, 20]))
    check(logits, u, draw(logits, u, **filters), **filters)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("levels", [1, 2, 3, 17])
@pytest.mark.parametrize("vocab", [5, 2048, 20011])
def test_many_ties(levels, vocab, dtype):
    """Few different logits, weights that are exact (powers of two): ties go to the lower id, at every border."""
    m = 12
    rng = np.random.default_rng(levels + vocab)
    z = torch.tensor(rng.integers(0, levels, (m, vocab)) * 0.5).to(dtype).to(DEV)
    heat = np.full(m, 0.5 / np.log(2), np.float32)               # (each level is half of the next, to fp32's rounding of the temperature)
    u = rng.random(m).astype(np.float32)
    u[:4] = [0, 0.5, 0.25, 1 - 2.0 ** -24]
    for filters in (dict(), dict(top_k=rng.integers(1, vocab + 1, m)), dict(top_p=rng.random(m)), dict(top_k=rng.integers(1, vocab + 1, m), top_p=rng.random(m)),
                    dict(min_p=rng.choice([0.1, 0.5, 0.7, 1.0], m))):
        filters = dict(filters, temperature=heat)
        check(z, u, draw(z, u, **filters), **filters)


def test_borders_that_are_exact():
    """All weights alike: half of the mass is half of the tokens."""
    z = torch.zeros(8, 64, device=DEV)
    u = np.array([0, 0.5, 0.25, 0.75, 0.984375, 0.49999997, 0.015625, 0.9999999], np.float32)
    got = draw(z, u)
    assert got[0] == [0, 32, 16, 48, 63, 31, 1, 63] and got[2] == [64] * 8
    got = draw(z, u, top_p=np.full(8, 0.5))
    assert got[2] == [32] * 8 and got[0] == [0, 16, 8, 24, 31, 15, 0, 31]
    got = draw(z, u, top_k=np.full(8, 3))
    assert got[2] == [3] * 8 and got[0] == [0, 1, 0, 2, 2, 1, 0, 2]


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("vocab", [9, 3000])
def test_numbers_that_are_not_finite(vocab, dtype):
    z = bell(12, vocab, torch.float32, 4).cpu()
    lowest = torch.finfo(dtype).min
    z[0] = -INF                                                  # nothing to draw
    z[1] = float("nan")
    z[2, ::2] = float("nan")
    z[3, 5] = INF                                                # the only one with weight
    z[4, 3], z[4, 7] = INF, INF
    z[5] = lowest                                                # a mask of the type's lowest value throughout: all alike
    z[6, 1:] = lowest
    z[7, 1:] = -INF                                              # one token
    z[8] = -0.0
    z[8, 4] = 0.0                                                # both zeros are one number
    z[9, :4] = float("nan")
    z[10] = torch.finfo(dtype).max
    z = z.to(dtype).to(DEV)
    u = np.linspace(0, 0.999, 12).astype(np.float32)
    for filters in ({}, dict(top_k=np.full(12, 2)), dict(top_p=np.full(12, 0.6)), dict(min_p=np.full(12, 0.5)), dict(temperature=np.full(12, INF)),
                    dict(top_k=np.full(12, 4), top_p=np.full(12, 0.9), temperature=np.full(12, 1e-30))):
        got = draw(z, u, **filters)
        check(z, u, got, **filters)
        assert got[0][:2] == [0, 0] and got[1][:2] == [0, 0] and got[2][:2] == [0, 0]


@pytest.mark.parametrize("u,same_as", [(-1.0, 0.0), (float("nan"), 0.0), (1.0, 1 - 2.0 ** -24), (INF, 1 - 2.0 ** -24)])
def test_uniform_numbers_out_of_range(u, same_as):
    z = bell(3, 500, F, 1)
    assert draw(z, np.full(3, u)) == draw(z, np.full(3, same_as))


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("vocab,gap,offset", [(1000, 24, 0), (1000, 1, 0), (999, 2, 3), (64, 0, 1), (5000, 8, 8)])
def test_rows_that_lie_apart_and_are_not_aligned(vocab, gap, offset, dtype):
    m = 9
    store = bell(1, m * (vocab + gap) + offset, dtype, 2)[0]
    z = store[offset:].view(m, vocab + gap)[:, :vocab]
    u = np.random.default_rng(2).random(m).astype(np.float32)
    filters = dict(top_k=np.resize([0, 20, 3], m), top_p=np.resize([0.9, 1.0], m))
    check(z, u, draw(z, u, **filters), **filters)


def test_rows_by_a_map_and_past_the_count():
    z = bell(6, 700, BF, 5)
    u = np.random.default_rng(3).random(8).astype(np.float32)
    to = [5, 0, 0, 3, -1, 6, 2, 1]                               # one of them twice, two that are not there
    got = draw(z, u, m=7, row_map=to, top_k=np.full(8, 30))
    assert got[0][7] == -77 and got[2][7] == -77 and got[1][7] == -77.0
    for r in (4, 5):
        assert (got[0][r], got[1][r], got[2][r]) == (0, 0.0, 0)
    keep = [0, 1, 2, 3, 6]
    check(z, u[keep], [[g[r] for r in keep] for g in got], row_map=[to[r] for r in keep], top_k=np.full(5, 30))


@pytest.mark.parametrize("count", [0, -2, 100])
def test_row_count_from_the_device(count):
    z = bell(4, 300, F, 6)
    u = np.full(4, 0.3, np.float32)
    got = draw(z, u, m=count)
    if count <= 0:
        assert got[0] == [-77] * 4
    else:
        check(z, u, got)


def test_shares_of_draws():
    """Evenly spread numbers draw each token in proportion to its weight (a stratified draw misses by less than one)."""
    m = 4096
    z = torch.tensor([0.3, -1.0, 2.0, 0.0, 1.5, -INF, 1.5]).repeat(m, 1).to(DEV)
    u = ((np.arange(m) + 0.5) / m).astype(np.float32)
    token = np.array(draw(z, u)[0])
    p = torch.softmax(z[0].double(), 0).cpu().numpy()
    assert (np.abs(np.bincount(token, minlength=7) - m * p) <= 1).all()


@pytest.mark.parametrize("m,vocab", [(3, 5000), (70, 8192)])
def test_same_results_captured_and_on_another_stream(m, vocab):
    z = bell(m, vocab, BF, 7)
    rng = np.random.default_rng(4)
    u, m_dev = dev(rng.random(m), F), dev([m], torch.int32)
    p, k = dev(np.resize([0.9, 1.0], m), F), dev(np.resize([0, 50, 0], m), torch.int32)
    ws = [torch.empty(max(256, B.sl_sample_filtered_bytes(m, vocab)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [torch.zeros(m, dtype=torch.int32, device=DEV) for _ in range(3)]
    call = lambda i, w: B.sl_sample_filtered(z, m_dev, m, u, outs[i], ws[w], top_p=p, top_k=k)  # noqa: E731
    call(0, 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        call(1, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(2, 1)
    for _ in range(3):
        u.copy_(torch.rand(m))
        ws[1].fill_(0xFF)
        outs[2].zero_()
        call(0, 0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])


ALL_FILTERS = dict(top_k=[0, 40, 0, 300, 0], top_p=[0.9, 1.0, 0.5, 0.95, 1.0], min_p=[0.0, 0.0, 0.02, 0.001, 0.0], temperature=[1.0, 0.8, 1.3])


def all_filters(m):
    return {n: np.resize(np.array(v, np.float64), m) for n, v in ALL_FILTERS.items()}


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("m,vocab", [(256, 900), (257, 900), (300, 4104), (257, 1 << 18), (258, 126463), (321, 1 << 18), (330, 5001)])
def test_many_rows(m, vocab, dtype):
    """More rows than CUs: smaller workgroups.  Of four rows of logits, each drawn from again and again; the first twenty against the definition."""
    z = bell(4, vocab, dtype, m)
    u = np.resize(np.random.default_rng(m).random(20).astype(np.float32), m)
    filters, to = all_filters(m), np.resize([2, 0, 3, 1], m)
    got = draw(z, u, row_map=to, **filters)
    check(z, u[:20], [g[:20] for g in got], row_map=to, **{n: v[:20] for n, v in filters.items()})
    seen = {}
    for r in range(m):
        key = (u[r], to[r]) + tuple(v[r] for v in filters.values())
        assert seen.setdefault(key, [g[r] for g in got]) == [g[r] for g in got]


def spans(vocab, seed):
    """Rows of bf16 numbers in places of their own: by name, what they hold."""
    g = torch.Generator().manual_seed(seed)
    n = torch.randn(vocab, generator=g)
    some = torch.rand(vocab, generator=g) < 0.5
    return {
        "large": n * 500 + 3000, "large and small": torch.where(some, n, n * 300 + 900), "negative": n * 2 - 14, "far below": torch.where(some, n, torch.tensor(-3e5)),
        "far below too": torch.where(some, n, torch.tensor(torch.finfo(BF).min)), "tiny": n * 2.0 ** -13, "tiny and below": torch.where(some, n * 2.0 ** -13, -n.abs() - 1),
        "tiny and above": torch.where(some, n * 2.0 ** -13, n.abs() * 2), "subnormal": n * 1e-39, "zeros": torch.where(some, torch.tensor(0.0), torch.tensor(-0.0)), "at the tiny ones' end":
        torch.where(some, torch.tensor(2.0 ** -10), torch.tensor(2.0 ** -10 - 2.0 ** -18)) * torch.sign(n), "steps of 2^-7": torch.round(n * 128) / 128, "negative and tiny": torch.where(some, -n.abs() * 2.0 ** -13, -n.abs() - 0.01),
        "wide": n * 200, "one far above": torch.where(torch.arange(vocab) == vocab // 3, torch.tensor(1e30), n),
    }


SPANS = list(spans(2, 0))


@pytest.mark.parametrize("name", SPANS)
@pytest.mark.parametrize("vocab", [60, 5001, 20000])
def test_numbers_of_every_size(name, vocab):
    """Where numbers lie decides how a bf16 row is worked on: one by one or digit by digit.  (At 20000 there are more tiny numbers than are listed.)"""
    kinds = [{}, dict(top_k=3), dict(top_k=vocab // 3), dict(top_k=vocab - 1), dict(top_k=vocab * 3 // 4, top_p=0.7), dict(top_p=0.3), dict(top_p=0.9999), dict(min_p=0.3), dict(min_p=0.9995),
             dict(top_p=0.8, temperature=1e4), dict(min_p=0.5, temperature=1e5), dict(top_k=vocab // 2, top_p=0.9, min_p=0.05, temperature=30.0), dict(temperature=0.0),
             dict(top_p=0.9, min_p=0.9999, temperature=2.0 ** -12), dict(top_k=vocab // 2, min_p=1e-30), dict(top_k=1)]
    plain = dict(top_k=0, top_p=1.0, min_p=0.0, temperature=1.0)
    filters = {n: np.array([k.get(n, v) for k in kinds]) for n, v in plain.items()}
    z = spans(vocab, vocab)[name].to(BF).repeat(len(kinds), 1).to(DEV)
    u = np.random.default_rng(vocab + SPANS.index(name)).random(len(kinds)).astype(np.float32)
    check(z, u, draw(z, u, **filters), **filters)


@pytest.mark.parametrize("dtype", [F, BF])
def test_rows_far_apart(dtype):
    """Offsets beyond 2^31 numbers: rows 2^20 numbers apart, the last of them 2^31 and more from the first."""
    n = (1 << 11) + 3
    store = torch.empty((n - 1 << 20) + 1000, dtype=dtype, device=DEV)
    z = store.as_strided((n, 1000), (1 << 20, 1))
    rows = [0, 1, n - 3, n - 1]
    z[rows] = bell(4, 1000, dtype, 8)
    u = np.random.default_rng(9).random(4).astype(np.float32)
    filters = all_filters(4)
    got = draw(z, u, row_map=rows, **filters)
    check(z[rows], u, got, **filters)


def test_two_draws_at_once_and_twice():
    """Two streams with a workspace each, many times: the same tokens every time."""
    m, vocab = 40, 9000
    z = bell(m, vocab, BF, 11)
    u, m_dev, p = dev(np.random.default_rng(12).random(m), F), dev([m], torch.int32), dev(np.full(m, 0.9), F)
    ws = [torch.empty(max(256, B.sl_sample_filtered_bytes(m, vocab)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = torch.full((2, 20, m), -1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(20):
        for w, s in enumerate(streams):
            with torch.cuda.stream(s):
                B.sl_sample_filtered(z, m_dev, m, u, outs[w, i], ws[w], top_p=p)
    torch.cuda.synchronize()
    assert bool((outs == outs[0, 0]).all()) and int(outs.min()) >= 0
