"""sl_kv8_*: the kernel forms that sizes choose -- many rows at once, results in pieces, long tables -- for every head size and type,
against the definitions in 64 bits (bounds: tests/test_gpu_kv8_values.py)."""
import math

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as ref
from tests.gpu_util import DEV
from tests.test_gpu_kv8 import Case, i32
from tests.test_gpu_kv8_values import attention

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


# ---- writing and reading more rows than the small kernels take (2048) ---------------------------------------
@pytest.mark.parametrize("order", ["ascending", "shuffled"])
@pytest.mark.parametrize("heads,page", [(1, 256), (3, 16), (5, 64)])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_many_rows_written_and_read(d, dtype, heads, page, order):
    """Ragged sequences, written and read back in order and out of order: then the slots of a quad belong to different waves, which
    write bytes of the same words."""
    lens = [1021, 1, 0, 700, 64, 470]
    rng = np.random.default_rng(d + heads)
    pos = [list(range(n)) if order == "ascending" else [int(p) for p in rng.permutation(n)] for n in lens]
    m = sum(lens)
    assert m > 2048
    need = [-(-n // page) for n in lens]
    table, pages = np.full((len(lens), max(need)), -1), rng.permutation(sum(need))
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pages[at:at + n]
        at += n
    kv = B.KV8(sum(need), page, heads, d, i32(table))
    kv.pool.fill_(0xFF)
    g = torch.Generator().manual_seed(d)
    qkv = torch.randn(m, 2 * heads * d, generator=g).to(dtype).to(DEV)
    k, v = (qkv[:, i * heads * d:(i + 1) * heads * d].view(m, heads, d) for i in (0, 1))
    row_pos, cu = i32([p for ps in pos for p in ps]), i32(np.concatenate([[0], np.cumsum(lens)]))
    B.sl_kv8_write(kv, k, v, row_pos, cu, m)
    # read back in yet another order, with rows behind the last sequence
    again = [[int(p) for p in rng.permutation(n)] for n in lens]
    out = torch.full((2, m + 9, heads, d), -77.0, dtype=dtype, device=DEV)
    more = i32([p for ps in again for p in ps] + [0] * 9)
    B.sl_kv8_read(kv, out[0], out[1], more, cu, m + 9)
    source = np.concatenate([np.cumsum([0] + lens)[b] + np.argsort(pos[b])[again[b]] for b in range(len(lens)) if lens[b]])
    for got, x in zip(out, (k, v)):
        want = torch.as_tensor(ref.kv8_values(ref.f64(x))).float().to(dtype)[source]
        assert torch.equal(got[:m].cpu(), want)
        assert (ref.f64(got[m:]) == -77.0).all()


def test_few_rows_of_a_quad_in_any_order():
    """The small kernels: single slots of the same quads from rows far apart."""
    heads, d, n = 3, 128, 256
    rng = np.random.default_rng(1)
    kv = B.KV8(16, 16, heads, d, i32(rng.permutation(16)[None]))
    kv.pool.fill_(0xFF)
    x = torch.randn(2, n, heads, d, generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    pos = rng.permutation(n)
    B.sl_kv8_write(kv, x[0], x[1], i32(pos), i32([0, n]), n)
    out = torch.empty(2, n, heads, d, dtype=BF, device=DEV)
    B.sl_kv8_read(kv, out[0], out[1], i32(range(n)), i32([0, n]), n)
    for got, y in zip(out, x):
        assert torch.equal(got.cpu(), torch.as_tensor(ref.kv8_values(ref.f64(y))).float().bfloat16()[np.argsort(pos)])


# ---- attention ----------------------------------------------------------------------------------------------
def check(c, q, got, counts, limits):
    share, r = q.shape[1] // c.heads, 0
    for b, m in enumerate(counts):
        for _ in range(m):
            n = min(c.lens[b], limits[r])
            for h in range(q.shape[1]):
                if n <= 0:
                    assert (got[r, h] == 0).all()
                    continue
                want, bound = attention(ref.f64(q[r, h]), c.K[b][:n, h // share], c.V[b][:n, h // share], 1.0 / math.sqrt(c.d), c.dtype)
                err = np.abs(got[r, h] - want)
                assert (err <= bound).all(), (b, r, h, float(np.nanmax(err / bound)))
            r += 1


@pytest.mark.parametrize("share", [1, 4])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_results_in_pieces(d, dtype, share):
    """Long and short sequences together: some segments are cut and joined, some not, some rows see none of the later pieces."""
    c = Case([1300, 5000, 513, 40, 512], 2, d, 64, dtype, seed=d)
    counts, limits = [2, 3, 1, 1, 2], [1300, 17, 5000, 600, -1, 1 << 30, 40, 512, 0]
    q, got = c.attend(counts, share, row_len=limits)
    check(c, q, got, counts, limits)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_more_rows_than_a_tile_of_queries(d, dtype):
    """Codes that several workgroups ask for: the loads through the caches."""
    c = Case([700, 90], 2, d, 16, dtype, seed=d + 1)
    counts = [23, 17]
    q, got = c.attend(counts, 1)
    check(c, q, got, counts, [1 << 30] * 40)


@pytest.mark.parametrize("dtype", [BF, F])
def test_cut_segments_of_more_than_64_sequences(dtype):
    """Sequences are looked at 64 at a time: pieces and partial results are counted over all of them."""
    lens = [(b * 131) % 1500 for b in range(150)]
    c = Case(lens, 1, 32, 64, dtype, seed=3)
    counts = [(b % 4) // 2 for b in range(150)]
    q, got = c.attend(counts, 2)
    check(c, q, got, counts, [1 << 30] * sum(counts))


def test_more_than_256_partial_results():
    """One row of one sequence so long that the join takes its partial results in several rounds."""
    c = Case([150000], 1, 32, 256, F, seed=4)
    q, got = c.attend([1], 1)
    check(c, q, got, [1], [1 << 30])


@pytest.mark.parametrize("dtype", [BF, F])
def test_every_row_of_a_sequence(dtype):
    """All rows active, as in a run's first step, each seeing the slots up to its own or up to the end of its block of 32."""
    lens = [300, 77]
    c = Case(lens, 2, 64, 64, dtype, seed=5)
    limits = [p + 1 for p in range(300)] + [min(77, (p // 32 + 1) * 32) for p in range(77)]
    q, got = c.attend(lens, 2, row_len=limits)
    check(c, q, got, lens, limits)


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_batch_of_eight_with_scattered_rows(dtype):
    """The counts of a late step of eight sequences."""
    lens, counts = [1024] * 8, [3, 8, 12, 16, 19, 22, 26, 31]
    c = Case(lens, 2, 128, 64, dtype, seed=6)
    q, got = c.attend(counts, 1)
    check(c, q, got, counts, [1 << 30] * sum(counts))
