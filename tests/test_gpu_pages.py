"""sl_kv8_pages_*: tables, stacks and rows against their definition, entry by entry (whole numbers: equality)."""
import random

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import serving_ref as ref
from tests.gpu_util import DEV, dev

pytestmark = pytest.mark.gpu
MARK = -77


def state(pages, table, lens, stack, n_free):
    for t, v in ((pages.page_table, table), (pages.seq_len, lens), (pages.free_pages, stack), (pages.n_free, [n_free])):
        t.copy_(torch.tensor(v, dtype=torch.int32).view_as(t))


def pool(rng, lens, page, max_pages, spare):
    """A pool in use: pages in no order."""
    held = [-(-n // page) for n in lens]
    order = list(range(sum(held) + spare))
    rng.shuffle(order)
    table, at = [], 0
    for n in held:
        table.append(order[at:at + n] + [-1] * (max_pages - n))
        at += n
    return table, order[at:] + [MARK] * at, spare


def resize(pages, want, m_upper, to=None):
    b = pages.batch
    out = dict(cu=torch.full((b + 1,), MARK, dtype=torch.int32, device=DEV), slot=torch.full((m_upper,), MARK, dtype=torch.int64, device=DEV))
    out.update({n: torch.full((m_upper,), MARK, dtype=torch.int32, device=DEV) for n in ("pos", "len", "seq")})
    B.sl_kv8_pages_resize(pages, dev(want, torch.int32), out["cu"], out["pos"], m_upper, to=to, row_len=out["len"], row_seq=out["seq"], row_slot=out["slot"])
    return {n: t.tolist() for n, t in out.items()}


def check(to, got, want):
    table, lens, stack, n_free, cu, rows = want
    assert to.n_free.tolist() == [n_free] and to.seq_len.tolist() == lens
    assert to.page_table.tolist() == table and to.free_pages.tolist() == stack
    pad = [MARK] * (len(got["pos"]) - len(rows))
    assert got["cu"] == cu
    assert got["pos"] == [r[0] for r in rows] + pad and got["len"] == [r[0] + 1 for r in rows] + pad
    assert got["seq"] == [r[1] for r in rows] + pad and got["slot"] == [r[2] for r in rows] + pad


# page slots, sequences, most pages of one, free pages, bound on rows, longest growth
CASES = [(16, 1, 1, 1, 1, 1), (16, 3, 8, 4, 3, 1), (16, 3, 8, 4, 40, 30), (32, 7, 5, 3, 64, 50), (64, 64, 9, 40, 900, 100), (64, 65, 9, 500, 5000, 70), (128, 20, 3, 9, 700, 300),
         (256, 255, 4, 100, 3000, 40), (16, 255, 33, 3000, 20000, 300), (32, 255, 64, 90, 255, 1), (256, 4, 100, 400, 1 << 17, 25600)]


@pytest.mark.parametrize("page,batch,max_pages,spare,m_upper,grow", CASES)
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("seed", [1, 2])
def test_resize(page, batch, max_pages, spare, m_upper, grow, apart, seed):
    """Three steps in a row: what one leaves is what the next finds."""
    rng = random.Random(seed * 1000 + batch + page)
    most = max_pages * page
    lens = [rng.choice([0, 1, page, rng.randint(0, most)]) for _ in range(batch)]
    table, stack, n_free = pool(rng, [min(n, most) for n in lens], page, max_pages, spare)
    lens = [min(n, most) for n in lens]
    pages = B.KV8Pages(len(stack), page, batch, max_pages)
    state(pages, table, lens, stack, n_free)
    for _ in range(3):
        want = [rng.choice([-1, 0, n, n + 1, n + 1, n + rng.randint(1, grow), n // 2, max(0, n - 1), most, most + 1]) for n in lens]
        before = [t.clone() for t in (pages.page_table, pages.seq_len, pages.free_pages, pages.n_free)]
        to = B.KV8Pages(len(stack), page, batch, max_pages) if apart else pages
        expected = ref.pages_resize(table, lens, stack, n_free, want, page, len(stack), m_upper)
        check(to, resize(pages, want, m_upper, to if apart else None), expected)
        if apart:
            assert all(torch.equal(t, u) for t, u in zip((pages.page_table, pages.seq_len, pages.free_pages, pages.n_free), before))
        pages, (table, lens, stack, n_free) = to, expected[:4]


def test_a_pool_starts_free_and_pages_come_in_order():
    pages = B.KV8Pages(5, 16, 2, 3)
    assert pages.page_table.tolist() == [[-1] * 3] * 2 and pages.seq_len.tolist() == [0, 0] and pages.n_free.tolist() == [5]
    got = resize(pages, [17, 40], 64)
    assert pages.page_table.tolist() == [[0, 1, -1], [2, 3, 4]] and pages.n_free.tolist() == [0] and got["cu"] == [0, 17, 57]
    resize(pages, [0, 0], 0)
    assert pages.page_table.tolist() == [[-1] * 3] * 2 and pages.n_free.tolist() == [5]


def test_one_that_does_not_fit_does_not_keep_others_out():
    pages = B.KV8Pages(4, 16, 3, 4)
    got = resize(pages, [16, 64, 30], 100)                      # 1, 4 and 2 pages, of 4
    assert pages.seq_len.tolist() == [16, 0, 30] and got["cu"] == [0, 16, 16, 46]
    got = resize(pages, [17, 0, 31], 1)                         # one page is left, and one row
    assert pages.seq_len.tolist() == [17, 0, 30] and got["cu"] == [0, 1, 1, 1]


@pytest.mark.parametrize("spare,m_upper", [(500, 1 << 20), (20000, 3000), (300, 2000), (0, 500), (37, 37)])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_little_room_for_growth_of_every_size(spare, m_upper, seed):
    """Who is served depends on all before: growth from one slot to far more than there is room for."""
    rng = random.Random(seed)
    page, batch, max_pages = 16, 255, 210
    lens = [rng.randint(0, 40) for _ in range(batch)]
    table, stack, n_free = pool(rng, lens, page, max_pages, spare)
    want = [rng.choice([n + int(2 ** rng.uniform(0, 11.7)), n // 2, n + 1]) for n in lens]
    pages = B.KV8Pages(len(stack), page, batch, max_pages)
    state(pages, table, lens, stack, n_free)
    expected = ref.pages_resize(table, lens, stack, n_free, want, page, len(stack), m_upper)
    assert any(n < w for n, w in zip(expected[1], want))
    check(pages, resize(pages, want, m_upper), expected)


def test_longer_than_a_sequence_can_be_and_lengths_out_of_range():
    pages = B.KV8Pages(20, 16, 4, 2)
    for want in ([33, 32, 2 ** 31 - 1, 1], [-2 ** 31, 32, -5, 40]):
        table, lens, stack, n_free = ([pages.page_table.tolist(), pages.seq_len.tolist(), pages.free_pages.tolist()] + pages.n_free.tolist())
        expected = ref.pages_resize(table, lens, stack, n_free, want, 16, 20, 100)
        check(pages, resize(pages, want, 100), expected)
    pages.seq_len.copy_(torch.tensor([-3, 1000, 5, 32]))        # a state that no call left
    pages.n_free.fill_(50)
    pages.page_table.copy_(torch.tensor([[-1, 99], [3, -7], [4, -1], [5, 6]]))
    args = (pages.page_table.tolist(), pages.seq_len.tolist(), pages.free_pages.tolist(), 50, [20, 1, 9, 0], 16, 20, 100)
    expected = ref.pages_resize(*args)
    check(pages, resize(pages, [20, 1, 9, 0], 100), expected)


def test_only_the_rows_are_asked_for():
    pages = B.KV8Pages(8, 16, 2, 4)
    cu, pos = torch.empty(3, dtype=torch.int32, device=DEV), torch.full((20,), MARK, dtype=torch.int32, device=DEV)
    B.sl_kv8_pages_resize(pages, dev([3, 5], torch.int32), cu, pos, 20)
    assert cu.tolist() == [0, 3, 8] and pos.tolist() == [0, 1, 2, 0, 1, 2, 3, 4] + [MARK] * 12


@pytest.mark.parametrize("m_upper", [40, 30000])
def test_captured_steps_of_one_state(m_upper):
    """A graph that grows every sequence to the lengths a caller leaves in want: replayed, with eager work between."""
    batch, page = 9, 32
    a, e = B.KV8Pages(200, page, batch, 20), B.KV8Pages(200, page, batch, 20)
    want, cu, pos = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (batch, batch + 1, m_upper))
    cu2, pos2 = torch.zeros_like(cu), torch.zeros_like(pos)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.sl_kv8_pages_resize(a, want, cu, pos, m_upper)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sl_kv8_pages_resize(a, want, cu, pos, m_upper)
    rng = np.random.default_rng(5)
    lens = np.zeros(batch, int)
    for i in range(5):
        lens = np.where(rng.random(batch) < 0.2, 0, np.minimum(lens + rng.integers(0, 5, batch), 640))
        want.copy_(torch.tensor(lens))
        graph.replay()
        B.sl_kv8_pages_resize(e, want, cu2, pos2, m_upper)
        torch.cuda.synchronize()
        for x, y in ((a.page_table, e.page_table), (a.seq_len, e.seq_len), (a.n_free, e.n_free), (a.free_pages, e.free_pages), (cu, cu2), (pos, pos2)):
            assert torch.equal(x, y), i


def test_many_pages_given_up_in_place_take_no_longer_than_beside():
    """A step that only releases: a million pages, no rows.  What is done in place is less than what states apart take, by however few rows the call is bounded."""
    page, batch, max_pages = 16, 255, 4112
    n = batch * max_pages
    full, a, other = (B.KV8Pages(n, page, batch, max_pages) for _ in range(3))
    full.page_table.copy_(torch.randperm(n, device=DEV).view(batch, max_pages))
    full.seq_len.fill_(max_pages * page)
    full.n_free.fill_(0)
    stay, none = (torch.full((batch,), v, dtype=torch.int32, device=DEV) for v in (-1, 0))
    cu, pos = torch.zeros(batch + 1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)

    def time_of(**to):
        ms = []
        for _ in range(5):
            B.sl_kv8_pages_resize(full, stay, cu, pos, 0, to=a)
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            B.sl_kv8_pages_resize(a, none, cu, pos, 0, **to)
            end.record()
            torch.cuda.synchronize()
            ms.append(start.elapsed_time(end))
        return min(ms)

    beside, in_place = time_of(to=other), time_of()
    for p in (a, other):
        assert p.n_free.tolist() == [n] and torch.equal(p.free_pages, full.page_table.view(-1)) and not p.seq_len.any() and (p.page_table == -1).all()
    assert in_place <= 5 * beside, (in_place, beside)


@pytest.mark.parametrize("batch,max_pages,m_upper", [(8, 250, 47), (64, 128, 128), (64, 128, 129), (32, 256, 32), (33, 249, 33), (255, 8, 8), (64, 64, 0), (20, 600, 20)])
@pytest.mark.parametrize("seed", [1, 2])
def test_in_place_with_few_rows_and_many_pages(batch, max_pages, m_upper, seed):
    """Around the size up to which one workgroup does it, and beyond, where lengths are copied first."""
    rng, page = random.Random(seed), 16
    lens = [rng.randint(0, max_pages * page) for _ in range(batch)]
    table, stack, n_free = pool(rng, lens, page, max_pages, batch * max_pages)
    pages = B.KV8Pages(len(stack), page, batch, max_pages)
    state(pages, table, lens, stack, n_free)
    for _ in range(3):
        want = [rng.choice([-1, 0, 0, n // 2, n + 1, n + rng.randint(0, 5)]) for n in lens]
        expected = ref.pages_resize(table, lens, stack, n_free, want, page, len(stack), m_upper)
        check(pages, resize(pages, want, m_upper), expected)
        table, lens, stack, n_free = expected[:4]
