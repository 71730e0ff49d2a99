"""The low-bit entry points refuse what they cannot do before anything is launched (no GPU needed), and their plain definitions."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as ref

OK, BAD, SMALL = B.SL_OK, B.SL_EINVAL, B.SL_ENOSPC


def call(name, good, **change):
    args = dict(good, **change)
    return getattr(B.lib(), name)(*args.values())


FORWARD = dict(stream=None, x=256, packed=256, m=256, m_upper=0, n=64, k=256, group=64, y_f32=256, y_bf16=None, row_map=None)
PACK = dict(stream=None, codes=256, scales=256, zeros=None, n=64, k=256, group=64, packed=256, size=0)
QUANT = dict(stream=None, w=256, dtype=1, n=64, k=256, group=64, codes=256, scales=256, zeros=None)


@pytest.mark.parametrize("change", [dict(x=None), dict(packed=None), dict(m=None), dict(m_upper=-1), dict(m_upper=(1 << 20) + 1), dict(n=0),
                                    dict(n=(1 << 24) + 1), dict(k=0), dict(k=260), dict(k=1 << 25), dict(n=1 << 20, k=1 << 20), dict(group=16), dict(group=256),
                                    dict(y_f32=None), dict(y_bf16=256), dict(row_map=256), dict(x=264), dict(packed=264), dict(y_f32=258)])
def test_q4_forward_refuses(change):
    assert call("sl_linear_q4_forward", FORWARD) == OK                     # no rows: nothing to launch
    assert call("sl_linear_q4_forward", FORWARD, **change) == BAD


@pytest.mark.parametrize("change", [dict(codes=None), dict(scales=None), dict(packed=None), dict(packed=264), dict(scales=257), dict(k=12),
                                    dict(group=0)])
def test_q4_pack_refuses(change):
    assert call("sl_linear_q4_pack", PACK) == SMALL
    assert call("sl_linear_q4_pack", PACK, size=B.sl_linear_q4_bytes(64, 256, 64) - 1) == SMALL
    assert call("sl_linear_q4_pack", PACK, **change) == BAD


@pytest.mark.parametrize("change", [dict(w=None), dict(codes=None), dict(scales=None), dict(dtype=2), dict(dtype=-1), dict(w=264), dict(codes=258), dict(scales=257), dict(k=20),
                                    dict(n=-1), dict(group=48)])
def test_q4_quantize_refuses(change):
    assert call("sl_linear_q4_quantize", QUANT, **change) == BAD


def test_q4_bytes():
    assert B.sl_linear_q4_bytes(64, 256, 128) == 4 * 2 * (1024 + 64)       # 4 bits a weight, 4 bytes a group
    assert B.sl_linear_q4_bytes(65, 264, 32) == 5 * 3 * (1024 + 256)       # columns and depth up to a whole block
    out = C.c_size_t()
    assert B.lib().sl_linear_q4_bytes(64, 256, 128, None) == BAD
    assert B.lib().sl_linear_q4_bytes(64, 250, 128, C.byref(out)) == BAD


def cache(**change):
    f = dict(pool=256, pool_bytes=1 << 40, page_table=256, n_pages=10, page_slots=64, n_kv_heads=4, d_head=128, batch=2, max_pages=5)
    return C.byref(B.sl_kv8(*dict(f, **change).values()))


ROWS = dict(stream=None, kv=None, k=256, v=256, dtype=1, ks=512, vs=512, pos=256, cu=256, m=0)
ATTN = dict(stream=None, kv=None, q=256, dtype=1, qs=1024, heads=8, cu=256, len=256, row_len=None, m=0, upper=100, scale=C.c_float(0.1), out=256,
            outs=1024, ws=256, size=1 << 40)
BAD_CACHE = [dict(pool=None), dict(pool=128), dict(page_table=None), dict(page_table=258), dict(n_pages=0), dict(page_slots=8),
             dict(page_slots=48), dict(page_slots=512), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(d_head=96), dict(d_head=512), dict(batch=0),
             dict(batch=256), dict(max_pages=0), dict(max_pages=1 << 25)]


@pytest.mark.parametrize("name", ["sl_kv8_write", "sl_kv8_read"])
def test_kv8_rows_refuse(name):
    good = dict(ROWS, kv=cache())
    assert call(name, good) == OK                                          # no rows
    for c in BAD_CACHE:
        assert call(name, good, kv=cache(**c)) == BAD, c
    assert call(name, good, kv=cache(pool_bytes=100)) == SMALL
    for c in (dict(kv=None), dict(k=None), dict(v=None), dict(k=264), dict(v=264), dict(dtype=2), dict(ks=511), dict(ks=516), dict(vs=508),
              dict(pos=None), dict(cu=None), dict(m=-1), dict(m=(1 << 20) + 1), dict(vs=1 << 41)):
        assert call(name, good, **c) == BAD, c


def test_kv8_attention_refuses():
    good = dict(ATTN, kv=cache())
    assert call("sl_kv8_attention", good) == OK
    for c in BAD_CACHE:
        assert call("sl_kv8_attention", good, kv=cache(**c)) == BAD, c
    for c in (dict(kv=None), dict(q=None), dict(out=None), dict(q=264), dict(out=264), dict(dtype=7), dict(qs=1023), dict(qs=1028), dict(outs=1016),
              dict(heads=0), dict(heads=6), dict(heads=1 << 15), dict(m=1 << 20, heads=256, qs=1 << 15, outs=1 << 15), dict(cu=None), dict(len=None), dict(m=-1), dict(m=(1 << 20) + 1), dict(upper=-1),
              dict(scale=C.c_float(0.0)), dict(scale=C.c_float(float("inf"))), dict(scale=C.c_float(float("nan"))), dict(ws=None), dict(ws=128)):
        assert call("sl_kv8_attention", good, **c) == BAD, c
    assert call("sl_kv8_attention", good, m=1, size=0) == SMALL            # refused before anything is launched
    assert call("sl_kv8_attention", good, kv=cache(pool_bytes=100)) == SMALL


def test_kv8_sizes():
    assert B.sl_kv8_bytes(10, 64, 4, 128) == 10 * 64 * 4 * 2 * (128 + 4)   # a byte a number and 4 bytes a vector
    out = C.c_size_t()
    assert B.lib().sl_kv8_bytes(10, 64, 4, 128, None) == BAD
    assert B.lib().sl_kv8_bytes(0, 64, 4, 128, C.byref(out)) == BAD
    assert B.lib().sl_kv8_attention_bytes(cache(), 8, 1, 100, None) == BAD
    assert B.lib().sl_kv8_attention_bytes(cache(), 7, 1, 100, C.byref(out)) == BAD


# ---- the definitions the GPU tests compare against ------------------------------------------------------
def test_kv8_definition():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64)).astype(np.float32).astype(np.float64)
    x[3] = 0
    x[4, 5] = np.inf
    x[5, 6] = np.nan
    code, scale = ref.kv8_codes(x)
    got = ref.kv8_values(x)
    assert (got[3] == 0).all() and np.isnan(got[4]).all() and np.isnan(got[5]).all()
    rest = [r for r in range(50) if r not in (4, 5)]
    assert (np.abs(got - x)[rest] <= (0.5 + 1e-5) * scale[rest]).all() and np.abs(code).max() == 127


def test_attention_definition_against_torch():
    g = torch.Generator().manual_seed(1)
    q, K, V = torch.randn(4, 32, generator=g).double(), torch.randn(9, 2, 32, generator=g).double(), torch.randn(9, 2, 32, generator=g).double()
    o, mass, _ = ref.kv8_attention(q.numpy(), K.numpy(), V.numpy(), 7, 0.3)
    for h in range(4):
        want = torch.softmax(0.3 * K[:7, h // 2] @ q[h], 0) @ V[:7, h // 2]
        assert np.allclose(o[h], want.numpy(), atol=1e-14)
    assert (ref.kv8_attention(q.numpy(), K.numpy(), V.numpy(), 0, 0.3)[0] == 0).all()
    without = ref.kv8_attention(q.numpy(), K.numpy(), V.numpy(), 7, 0.3, absent={2, 6})[0]
    kept = [0, 1, 3, 4, 5]
    assert np.allclose(without, ref.kv8_attention(q.numpy(), K.numpy()[kept], V.numpy()[kept], 5, 0.3)[0], atol=1e-14)


def test_q4_definition():
    w = np.array([[0.0, 1.5, -0.5, 1.0, 0.25, 0.5, 0.75, -0.25]])
    codes, scales, zeros = ref.q4_quantize(w, 32, True)                    # range 2, step bf16(2 / 15)
    assert zeros[0, 0] == 4 and abs(scales[0, 0] - 2 / 15) < 2 / 15 * 2 ** -8
    assert np.abs(ref.q4_weights(codes, scales, zeros, 32) - w).max() <= scales[0, 0] / 2 + 15 * scales[0, 0] * 2 ** -8
    codes, scales, zeros = ref.q4_quantize(w, 32, False)
    assert zeros[0, 0] == 8 and codes.min() >= 1 and codes.max() == 15
