"""sl_kv8_*: the paged 8-bit cache and the attention over it, against their definitions in 64 bits (tests/lowbit_ref.py).

What is written and read back is compared bit by bit: scale and codes are fixed by the definition.  The attention's bound counts fp32
roundings of sums and the bits of its probabilities (lowbit_ref.kv8_attention_bound), plus half a step of the result's type."""
import math

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as ref
from tests.gpu_util import DEV, dev

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def i32(a):
    return dev(np.asarray(a, dtype=np.int32).reshape(np.shape(a)))


class Case:
    """A cache of ragged sequences, filled through sl_kv8_write; K, V: what it holds, in float64."""

    def __init__(self, lens, heads, d, page, dtype, seed=0, spare_pages=2, garbage=0xFF):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare_pages
        order = rng.permutation(self.n_pages)
        width = max(max(need), 1)
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.lens, self.heads, self.d, self.page, self.dtype = lens, heads, d, page, dtype
        self.kv = B.KV8(self.n_pages, page, heads, d, i32(self.table))
        self.kv.pool.fill_(garbage)                                # 0xFF..: codes of -1 and scales that are NaN
        self.k = [torch.randn(n, heads, d, generator=g).to(dtype) for n in lens]
        self.v = [(torch.randn(n, heads, d, generator=g) * 2.0 ** torch.randint(-4, 5, (n, heads, 1), generator=g)).to(dtype) for n in lens]
        self.write([list(range(n)) for n in lens])
        self.K = [ref.kv8_values(ref.f64(k)) if len(k) else np.zeros((0, heads, d)) for k in self.k]
        self.V = [ref.kv8_values(ref.f64(v)) if len(v) else np.zeros((0, heads, d)) for v in self.v]

    def rows(self, pos):
        cu = np.concatenate([[0], np.cumsum([len(p) for p in pos])])
        return i32([p for ps in pos for p in ps] or [0]), i32(cu), int(cu[-1])

    def write(self, pos):
        row_pos, cu, m = self.rows(pos)
        if m:
            k = torch.cat([self.k[b][p] for b, p in enumerate(pos)]).to(DEV)
            v = torch.cat([self.v[b][p] for b, p in enumerate(pos)]).to(DEV)
            B.sl_kv8_write(self.kv, k, v, row_pos, cu, m)

    def attend(self, counts, share, row_len=None, m_upper=None, len_upper=None, seed=5, q=None, seq_len=None, ws_fill=0xFF, stride=0):
        """-> (q, out) with rows behind the last sequence in place (-77 before the call)."""
        H, m = self.heads * share, sum(counts)
        mu = m if m_upper is None else m_upper
        if q is None:
            q = torch.randn(mu, H, self.d, generator=torch.Generator().manual_seed(seed)).to(self.dtype)
        hold = torch.full((mu, H * self.d + stride), float("nan"), dtype=self.dtype, device=DEV)
        qd = hold[:, :H * self.d].view(mu, H, self.d) if stride == 0 else hold.as_strided((mu, H, self.d), (H * self.d + stride, self.d, 1))
        qd.copy_(q.to(DEV))
        out = torch.full((mu, H * self.d + stride), -77.0, dtype=self.dtype, device=DEV)
        od = out.as_strided((mu, H, self.d), (H * self.d + stride, self.d, 1))
        lens = self.lens if seq_len is None else seq_len
        up = max(max(lens), 0) if len_upper is None else len_upper
        ws = torch.full((B.sl_kv8_attention_bytes(self.kv, H, mu, up),), ws_fill, dtype=torch.uint8, device=DEV)
        B.sl_kv8_attention(self.kv, qd, i32(np.concatenate([[0], np.cumsum(counts)])), i32(lens), mu, up, 1.0 / math.sqrt(self.d), od, ws,
                           row_len=None if row_len is None else i32(row_len))
        if stride:
            assert (ref.f64(out[:, H * self.d:]) == -77.0).all()
        return q, ref.f64(od)

    def check(self, q, got, counts, row_len=None, absent=None, seq_len=None):
        at = 0
        for b, m in enumerate(counts):
            n = self.lens[b] if seq_len is None else min(seq_len[b], self.lens[b])
            for r in range(at, at + m):
                limit = n if row_len is None else min(n, row_len[r])
                want, mass, size = ref.kv8_attention(ref.f64(q[r]), self.K[b], self.V[b], limit, 1.0 / math.sqrt(self.d),
                                                     absent[b] if absent else ())
                bound = ref.kv8_attention_bound(mass, size, max(limit, 1), self.d, self.dtype) + ref.half_step(want, self.dtype) * 1.01
                err = np.abs(got[r] - want)
                assert (err <= bound).all(), (b, r, float((err / bound).max()))
            at += m


# ---- writing and reading back --------------------------------------------------------------------------
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 64), (5, 256), (32, 32)])
def test_what_is_read_back(d, dtype, heads, page):
    c = Case([37, 1, 0, 130, 16], heads, d, page, dtype, seed=d + heads)
    pos = [list(range(37)), [0], [], list(range(129, -1, -1)), [3, 2, 15, 0]]        # any order
    row_pos, cu, m = c.rows(pos)
    k, v = (torch.full((m + 3, heads, d), -77.0, dtype=dtype, device=DEV) for _ in range(2))
    B.sl_kv8_read(c.kv, k[:m], v[:m], row_pos, cu, m)
    at = 0
    for b, ps in enumerate(pos):
        for got, held in ((k, c.K), (v, c.V)):
            want = torch.as_tensor(held[b][ps]).to(F).to(dtype)
            assert torch.equal(got[at:at + len(ps)].cpu(), want), (b, d, heads, page)
        at += len(ps)
    assert (ref.f64(k[m:]) == -77.0).all() and (ref.f64(v[m:]) == -77.0).all()


def test_extreme_vectors():
    """Zero, tiny, huge, non-finite: scale 0, scales down to the smallest number, NaN throughout."""
    x = torch.randn(1, 10, 4, 64, generator=torch.Generator().manual_seed(1))[0]
    x[0] = 0
    x[1] *= 1e-38
    x[2] *= 1e-44
    x[3] *= 1e36
    x[4, :, 7] = float("inf")
    x[5, 1] = float("nan")
    x[6, 2, :63] = 0
    x[7, 0] = -0.0
    x[8] = 1.4e-45
    kv = B.KV8(1, 16, 4, 64, i32([[0]]))
    kv.pool.fill_(0xFF)
    pos, cu = i32(range(10)), i32([0, 10])
    B.sl_kv8_write(kv, x.to(DEV), x.flip(1).contiguous().to(DEV), pos, cu, 10)
    k, v = (torch.empty(10, 4, 64, device=DEV) for _ in range(2))
    B.sl_kv8_read(kv, k, v, pos, cu, 10)
    want = torch.as_tensor(ref.kv8_values(ref.f64(x))).float()
    assert np.array_equal(ref.f64(k), ref.f64(want), equal_nan=True)
    assert np.array_equal(ref.f64(v), ref.f64(want.flip(1)), equal_nan=True)


def test_strided_rows_of_a_fused_projection():
    heads, d, m = 4, 128, 9
    qkv = torch.randn(m, 3 * heads * d, generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    k, v = (qkv[:, i * heads * d:(i + 1) * heads * d].view(m, heads, d) for i in (1, 2))
    kv = B.KV8(3, 16, heads, d, i32([[2, 0]]))
    pos, cu = i32([0, 1, 2, 3, 5, 6, 15, 16, 31]), i32([0, m])
    B.sl_kv8_write(kv, k, v, pos, cu, m)
    out = torch.full((m, 2 * heads * d), -77.0, dtype=BF, device=DEV)
    B.sl_kv8_read(kv, out[:, :heads * d].view(m, heads, d), out[:, heads * d:].view(m, heads, d), pos, cu, m)
    for got, x in ((out[:, :heads * d], k), (out[:, heads * d:], v)):
        assert torch.equal(got.reshape(m, heads, d).cpu(), torch.as_tensor(ref.kv8_values(ref.f64(x))).float().bfloat16())


def test_rows_that_are_not_written():
    """Negative slots, slots past the table, slots on no page, rows behind the last sequence: the pool stays as it is; the first three
    read back as zeros, the last are left alone."""
    heads, d = 2, 64
    kv = B.KV8(4, 16, heads, d, i32([[1, -1, 9], [3, 2, 1 << 30]]))
    kv.pool.fill_(0x11)
    before = kv.pool.clone()
    pos = i32([-1, 16, 47, 48, 2 ** 31 - 1, -2 ** 31, 40, 33, 5, 6])
    cu, m = i32([0, 4, 8]), 10
    x = torch.randn(m, heads, d, device=DEV)
    B.sl_kv8_write(kv, x, x, pos, cu, m)
    assert torch.equal(kv.pool, before)
    k, v = (torch.full((m, heads, d), -77.0, device=DEV) for _ in range(2))
    B.sl_kv8_read(kv, k, v, pos, cu, m)
    for t in (k, v):
        assert (ref.f64(t)[:8] == 0).all() and (ref.f64(t)[8:] == -77.0).all()


def test_a_write_leaves_its_neighbours_alone():
    """Odd slots rewritten, in runs that start and end anywhere: the others read back as before."""
    c = Case([50, 23], 3, 128, 16, BF, seed=4)
    new = [torch.randn(n, 3, 128, generator=torch.Generator().manual_seed(9 + n)).bfloat16() for n in (50, 23)]
    pos = [[1, 2, 3, 7, 13, 14, 15, 16, 17, 18, 19, 20, 33, 47, 49], [0, 5, 22]]
    row_pos, cu, m = c.rows(pos)
    rows = torch.cat([new[b][p] for b, p in enumerate(pos)]).to(DEV)
    B.sl_kv8_write(c.kv, rows, rows, row_pos, cu, m)
    every = [list(range(50)), list(range(23))]
    row_pos, cu, m = c.rows(every)
    k, v = (torch.empty(m, 3, 128, dtype=BF, device=DEV) for _ in range(2))
    B.sl_kv8_read(c.kv, k, v, row_pos, cu, m)
    for got, old in ((k, c.K), (v, c.V)):
        want = [torch.as_tensor(o).float().bfloat16() for o in old]
        for b, ps in enumerate(pos):
            want[b][ps] = torch.as_tensor(ref.kv8_values(ref.f64(new[b][ps]))).float().bfloat16()
        assert torch.equal(got.cpu(), torch.cat(want))


def test_of_adjacent_rows_with_one_slot_the_last_is_kept():
    heads, d = 2, 32
    kv = B.KV8(2, 16, heads, d, i32([[1], [0]]))
    pos, cu = i32([3, 3, 3, 4, 5, 5, 5, 5, 5, 5, 3, 3]), i32([0, 10, 12])      # the second sequence has its own slot 3
    x = torch.randn(12, heads, d, generator=torch.Generator().manual_seed(3))
    B.sl_kv8_write(kv, x.to(DEV), (-x).to(DEV), pos, cu, 12)
    k, v = (torch.empty(12, heads, d, device=DEV) for _ in range(2))
    B.sl_kv8_read(kv, k, v, pos, cu, 12)
    kept = [2, 2, 2, 3, 9, 9, 9, 9, 9, 9, 11, 11]
    want = torch.as_tensor(ref.kv8_values(ref.f64(x)))[kept].float()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), -want)


@pytest.mark.parametrize("heads", [1, 3])
def test_many_rows_that_name_one_quad(heads):
    """Longer than a wave: 64, 65 and 200 adjacent rows on one slot, and on the slots of one quad in turn."""
    d, m = 64, 329
    kv = B.KV8(1, 16, heads, d, i32([[0], [0], [0]]))
    pos = [2] * 64 + [5] * 65 + [8 + i % 4 for i in range(200)]
    cu = i32([0, 64, 129, 329])
    x = torch.randn(m, heads, d, generator=torch.Generator().manual_seed(6))
    B.sl_kv8_write(kv, x.to(DEV), (-x).to(DEV), i32(pos), cu, m)
    k, v = (torch.empty(m, heads, d, device=DEV) for _ in range(2))
    B.sl_kv8_read(kv, k, v, i32(pos), cu, m)
    # rows on slots 8 .. 11 in turn name a slot again four rows on; they share the quad and stay in order
    last = {p: max(i for i in range(m) if pos[i] == p) for p in set(pos)}
    want = torch.as_tensor(ref.kv8_values(ref.f64(x)))[[last[p] for p in pos]].float()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), -want)


# ---- attention ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("share", [1, 4])
def test_attention_types_and_heads(d, dtype, share):
    c = Case([130, 1, 17, 64], 2, d, 16, dtype, seed=d)
    counts = [1, 1, 3, 0]
    q, got = c.attend(counts, share)
    c.check(q, got, counts)


@pytest.mark.parametrize("lens,counts", [([1], [1]), ([15, 16, 17], [1, 1, 1]), ([63, 64, 65, 129], [2, 1, 4, 1]), ([255, 257, 1000], [1, 17, 5]),
                                         ([2048], [64]), ([5000, 3, 0, 777], [1, 1, 2, 3]), ([300] * 40, [1] * 40), ([70], [33])])
@pytest.mark.parametrize("page", [16, 128])
def test_attention_lengths(lens, counts, page):
    c = Case(lens, 2, 64, page, BF, seed=len(lens))
    q, got = c.attend(counts, 1)
    c.check(q, got, counts)


@pytest.mark.parametrize("share,count", [(3, 7), (8, 2), (8, 1), (5, 1), (17, 1), (40, 2)])
def test_attention_shared_heads(share, count):
    """Queries of a tile come from several heads and rows; a row's heads lie in several tiles."""
    c = Case([333, 50], 2, 64, 32, BF, seed=share)
    q, got = c.attend([count, 1], share)
    c.check(q, got, [count, 1])


@pytest.mark.parametrize("dtype", [BF, F])
def test_row_lengths(dtype):
    """Each row its own length: none, one, inside a tile, longer than the sequence, negative."""
    c = Case([200, 700], 2, 64, 16, dtype, seed=7)
    counts, row_len = [7, 5], [0, 1, 16, 17, 200, 1 << 30, -5, 699, 700, 640, 0, 64]
    q, got = c.attend(counts, 2, row_len=row_len)
    c.check(q, got, counts, row_len=row_len)
    assert (got[[0, 6, 10]] == 0).all()


def test_lengths_that_do_not_fit():
    """A sequence length past the table, past the bound, negative or zero: what there is, or zeros."""
    c = Case([64, 64, 64, 64], 1, 64, 32, BF, seed=8)
    q, got = c.attend([1, 1, 1, 1], 1, seq_len=[1 << 30, -4, 0, 40], len_upper=4000)
    c.check(q, got, [1, 1, 1, 1], seq_len=[64, 0, 0, 40])
    assert (got[1:3] == 0).all()
    q, got = c.attend([1, 1, 1, 1], 1, seq_len=[64, 64, 64, 64], len_upper=33)
    c.check(q, got, [1, 1, 1, 1], seq_len=[33, 33, 33, 33])
    q, got = c.attend([1, 1, 1, 1], 1, len_upper=0)
    assert (got == 0).all()


def test_rows_behind_the_last_sequence_are_left():
    c = Case([100, 90], 2, 64, 16, BF, seed=9)
    q, got = c.attend([2, 1], 2, m_upper=9)
    c.check(q, got, [2, 1])
    assert (got[3:] == -77.0).all()


def test_more_rows_than_the_bound():
    """cu_rows beyond m_upper: the first m_upper rows are computed, nothing past them is touched."""
    c = Case([100, 90], 2, 64, 16, BF, seed=10)
    q, full = c.attend([4, 5], 1)
    H = 2
    out = torch.full((9, H, 64), -77.0, dtype=BF, device=DEV)
    ws = torch.empty(B.sl_kv8_attention_bytes(c.kv, H, 6, 100), dtype=torch.uint8, device=DEV)
    B.sl_kv8_attention(c.kv, q.to(DEV), i32([0, 4, 9]), i32([100, 90]), 6, 100, 1 / 8, out, ws)
    got = ref.f64(out)
    assert np.array_equal(got[:6], full[:6]) and (got[6:] == -77.0).all()


def test_pages_that_do_not_exist():
    """Entries outside the pool are absent slots, whatever the lengths say; a sequence with none at all gives zeros."""
    c = Case([100, 100, 50], 2, 64, 16, BF, seed=11)
    table = c.table.copy()
    table[0, 2], table[0, 6] = -1, 1 << 30
    table[2, :] = c.n_pages
    c.kv = B.KV8(c.n_pages, 16, 2, 64, i32(table), c.kv.pool)
    q, got = c.attend([2, 1, 1], 2)
    c.check(q, got, [2, 1, 1], absent=[set(range(32, 48)) | set(range(96, 112)), set(), set(range(50))])
    assert (got[3] == 0).all()


def test_broken_slots_only_reach_rows_that_see_them():
    """A slot of NaN and one of infinities: rows that see neither are exact, rows that see one are NaN."""
    c = Case([90], 2, 64, 16, BF, seed=12)
    k, v = c.k[0].clone(), c.v[0].clone()
    k[70], v[80, :, 3] = float("nan"), float("inf")
    B.sl_kv8_write(c.kv, k.to(DEV), v.to(DEV), i32(range(90)), i32([0, 90]), 90)
    row_len = [70, 71, 60, 5, 81, 90, 1, 70]
    q, got = c.attend([8], 2, row_len=row_len)
    keep = [0, 2, 3, 6, 7]
    assert np.isnan(got[[1, 4, 5]]).all()
    for r in keep:
        want, mass, size = ref.kv8_attention(ref.f64(q[r]), c.K[0], c.V[0], row_len[r], 1 / 8)
        assert (np.abs(got[r] - want) <= ref.kv8_attention_bound(mass, size, row_len[r], 64, BF) + ref.half_step(want, BF) * 1.01).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_one_slot_takes_all_the_weight(dtype):
    """A query along one key, far ahead of the others, whose value is a millionth of theirs: the sharp softmax and values of very
    different size."""
    c = Case([400], 1, 64, 16, dtype, seed=13)
    c.k[0][123] = 8.0 * torch.sign(c.k[0][123].float()).to(dtype)
    c.v[0][123] = (c.v[0][123].float() * 1e-6).to(dtype)
    c.write([list(range(400))])
    c.K, c.V = [ref.kv8_values(ref.f64(c.k[0]))], [ref.kv8_values(ref.f64(c.v[0]))]
    q = (4.0 * torch.sign(c.k[0][123].float()).to(dtype))[None].contiguous()
    q, got = c.attend([1], 1, q=q)
    c.check(q, got, [1])


def test_strided_queries_and_results():
    c = Case([150, 70], 2, 128, 64, BF, seed=14)
    q, got = c.attend([3, 2], 2, stride=64)
    c.check(q, got, [3, 2])


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB whose sequence lies in its last pages."""
    n_pages, page, heads, d = 4200, 256, 16, 128                   # 4.3 GiB
    table = np.arange(n_pages - 2, n_pages, dtype=np.int32)[None]
    kv = B.KV8(n_pages, page, heads, d, i32(table))
    assert kv.pool.numel() > 1 << 32
    c = Case([300], heads, d, page, BF, seed=15)
    c.kv = kv
    c.write([list(range(300))])
    q, got = c.attend([2], 1)
    c.check(q, got, [2])


def test_long_sequence_fp32():
    c = Case([40000], 1, 64, 256, F, seed=16)
    q, got = c.attend([2], 2, row_len=[40000, 31111])
    c.check(q, got, [2], row_len=[40000, 31111])


def test_the_largest_batch():
    lens = [(b * 7) % 50 for b in range(255)]
    c = Case(lens, 1, 32, 16, BF, seed=17)
    counts = [b % 3 for b in range(255)]
    q, got = c.attend(counts, 1)
    c.check(q, got, counts)


def test_same_bits_whatever_the_workspace_holds_and_on_another_stream():
    c = Case([3000, 100], 2, 64, 64, BF, seed=18)
    q, a = c.attend([2, 3], 2, ws_fill=0xFF)
    _, b = c.attend([2, 3], 2, ws_fill=0x7F)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        _, s = c.attend([2, 3], 2)
        torch.cuda.synchronize()
    assert np.array_equal(a, b) and np.array_equal(a, s)


def test_what_the_binding_refuses_and_what_is_nothing_to_do():
    """Types, layouts and devices that the library would misread raise; no rows at all are fine."""
    c = Case([20], 2, 64, 16, BF, seed=19)
    q = torch.zeros(1, 2, 64, dtype=BF, device=DEV)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    good = dict(kv=c.kv, q=q, cu_rows=i32([0, 1]), seq_len=i32([20]), m_upper=1, len_upper=20, scale=0.1, out=torch.zeros_like(q), workspace=ws)
    B.sl_kv8_attention(**good)
    for change in (dict(q=q.cpu()), dict(q=q.half()), dict(q=q.float()), dict(out=q[0]), dict(seq_len=torch.tensor([20], device=DEV)),
                   dict(cu_rows=torch.tensor([0, 1], dtype=torch.int32)), dict(q=torch.zeros(1, 64, 2, dtype=BF, device=DEV).transpose(1, 2)),
                   dict(workspace=ws.float()), dict(row_len=torch.zeros(1, device=DEV))):
        with pytest.raises((ValueError, KeyError)):
            B.sl_kv8_attention(**dict(good, **change))
    with pytest.raises(B.SureLockError) as e:
        B.sl_kv8_attention(**dict(good, len_upper=100000, workspace=ws[:0]))
    assert e.value.status in (B.SL_EINVAL, B.SL_ENOSPC)
    none = torch.zeros(0, 2, 64, dtype=BF, device=DEV)
    B.sl_kv8_attention(**dict(good, q=none, out=none, m_upper=0))
    B.sl_kv8_write(c.kv, none, none, i32([0]), i32([0, 0]), 0)
    x = torch.zeros(2, 64, dtype=BF, device=DEV)
    packed = torch.empty(B.sl_linear_q4_bytes(8, 64, 32), dtype=torch.uint8, device=DEV)
    for change in (dict(x=x.float()), dict(x=x.cpu()), dict(x=torch.zeros(64, 2, dtype=BF, device=DEV).T), dict(y_f32=torch.zeros(2, 8, dtype=BF, device=DEV)),
                   dict(m_dev=torch.tensor([2], device=DEV)), dict(packed=packed.float())):
        args = dict(dict(x=x, packed=packed, m_dev=i32([2]), m_upper=2, n=8, k=64, group=32, y_f32=torch.zeros(2, 8, device=DEV)), **change)
        with pytest.raises(ValueError):
            B.sl_linear_q4_forward(**args)
    B.sl_linear_q4_forward(x[:0], packed, i32([0]), 0, 8, 64, 32, y_f32=torch.zeros(0, 8, device=DEV))


def test_a_cache_on_another_device_is_refused():
    """The kernels would follow its pool and page table: no call starts unless both are on the current device."""
    c = Case([20], 2, 64, 16, BF, seed=23)
    with pytest.raises(ValueError):
        B.KV8(c.n_pages, 16, 2, 64, i32(c.table), c.kv.pool.cpu())
    with pytest.raises(ValueError):
        B.KV8(c.n_pages, 16, 2, 64, i32(c.table).cpu())
    x = torch.zeros(1, 2, 64, dtype=BF, device=DEV)
    away = c.kv.sequence(0)
    away.device += 1                                        # as a cache of another device says
    for call in (lambda: B.sl_kv8_write(away, x, x, i32([0]), i32([0, 1]), 1), lambda: B.sl_kv8_read(away, x, x, i32([0]), i32([0, 1]), 1),
                 lambda: B.sl_kv8_attention(away, x, i32([0, 1]), i32([20]), 1, 20, 0.1, torch.zeros_like(x),
                                            torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            call()


# ---- a decoding block's few-row work, all together ----------------------------------------------------------
def _block(st):
    """Q|K|V with 4-bit weights, the rows' K and V into the cache, attention, Out with 4-bit weights."""
    m, H, d, width = st["m"], st["H"], st["d"], st["H"] * st["d"]
    B.sl_linear_q4_forward(st["x"], st["wqkv"], st["count"], m, 3 * width, width, 128, y_bf16=st["qkv"])
    q, k, v = (st["qkv"][:, i * width:(i + 1) * width].view(m, H, d) for i in range(3))
    B.sl_kv8_write(st["kv"], k, v, st["pos"], st["cu"], m)
    B.sl_kv8_attention(st["kv"], q, st["cu"], st["len"], m, st["upper"], 1 / math.sqrt(d), st["o"], st["ws"], row_len=st["row_len"])
    B.sl_linear_q4_forward(st["o"].view(m, width), st["wo"], st["count"], m, width, width, 128, y_bf16=st["y"])


def test_a_block_of_few_rows_eager_and_captured():
    """The operators in a row, as a decoding step has them, against the definitions; then the same launches captured once and
    replayed with other rows, other slots and longer sequences, the program's own eager calls in between."""
    H, d, page = 4, 128, 16
    width, lens, counts = H * d, [700, 45, 300], [3, 1, 4]
    m, n_cap = sum(counts), 720
    c = Case([n_cap] * 3, H, d, page, BF, seed=20)
    rng = np.random.default_rng(21)
    wq = {}
    for name, n in (("wqkv", 3 * width), ("wo", width)):
        w = torch.as_tensor(0.04 * rng.standard_normal((n, width))).float()
        codes, scales, zeros = ref.q4_quantize(ref.f64(w), 128, True)
        packed = torch.empty(B.sl_linear_q4_bytes(n, width, 128), dtype=torch.uint8, device=DEV)
        cd, sc, zp = (torch.empty(s, dtype=t, device=DEV) for s, t in (((n, width // 2), torch.uint8), ((n, width // 128), BF),
                                                                       ((n, width // 128), torch.uint8)))
        B.sl_linear_q4_quantize(w.to(DEV), 128, cd, sc, zp)
        B.sl_linear_q4_pack(cd, sc, zp, n, width, 128, packed)
        wq[name] = (packed, ref.q4_weights(codes, scales, zeros, 128), ref.q4_bound, (codes, scales, zeros, 128))
    st = {"m": m, "H": H, "d": d, "wqkv": wq["wqkv"][0], "wo": wq["wo"][0], "kv": c.kv, "upper": n_cap, "count": i32([m]),
          "cu": i32([0, 3, 4, 8]), "x": torch.zeros(m, width, dtype=BF, device=DEV), "qkv": torch.zeros(m, 3 * width, dtype=BF, device=DEV),
          "o": torch.zeros(m, H, d, dtype=BF, device=DEV), "y": torch.zeros(m, width, dtype=BF, device=DEV), "pos": i32([0] * m),
          "len": i32(lens), "row_len": i32([0] * m), "ws": torch.empty(B.sl_kv8_attention_bytes(c.kv, H, m, n_cap), dtype=torch.uint8, device=DEV)}

    def load(step):
        r = np.random.default_rng(100 + step)
        now = [n + step for n in lens]
        pos = [sorted(r.choice(n, k, replace=False)) for n, k in zip(now, counts)]
        st["x"].copy_(torch.as_tensor(r.standard_normal((m, width))).bfloat16())
        flat = [int(p) for ps in pos for p in ps]
        st["pos"].copy_(i32(flat))
        st["len"].copy_(i32(now))
        seen = [n if i % 2 else min(n, p + 1) for i, (n, p) in enumerate(zip(np.repeat(now, counts), flat))]
        st["row_len"].copy_(i32(seen))
        return now, pos, seen

    def check(now, pos, seen):
        torch.cuda.synchronize()
        x, qkv, o, y = (ref.f64(st[n]) for n in ("x", "qkv", "o", "y"))
        want = x @ wq["wqkv"][1].T
        assert (np.abs(qkv - want) <= ref.q4_bound(x, *wq["wqkv"][3]) + ref.half_step(want, BF) * 1.01).all()
        at = 0
        for b, ps in enumerate(pos):
            rows = qkv[at:at + len(ps)]
            c.K[b][ps] = ref.kv8_values(rows[:, width:2 * width].reshape(-1, H, d))
            c.V[b][ps] = ref.kv8_values(rows[:, 2 * width:].reshape(-1, H, d))
            at += len(ps)
        at = 0
        for b, ps in enumerate(pos):
            for r in range(at, at + len(ps)):
                wo, mass, size = ref.kv8_attention(qkv[r, :width].reshape(H, d), c.K[b], c.V[b], min(now[b], seen[r]), 1 / math.sqrt(d))
                bound = ref.kv8_attention_bound(mass, size, now[b], d, BF) + ref.half_step(wo, BF) * 1.01
                assert (np.abs(o[r] - wo) <= bound).all()
            at += len(ps)
        flat = o.reshape(m, width)
        want = flat @ wq["wo"][1].T
        assert (np.abs(y - want) <= ref.q4_bound(flat, *wq["wo"][3]) + ref.half_step(want, BF) * 1.01).all()

    state = load(0)
    _block(st)
    check(*state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _block(st)
    for step in range(1, 5):
        state = load(step)
        graph.replay()
        check(*state)
        if step == 2:                                              # an eager step between two replays
            state = load(9)
            _block(st)
            check(*state)
