"""The serving-step calls refuse what they cannot do before anything is launched (no GPU needed), the binding compares every buffer with the sizes
that the library will touch, and the definitions that the GPU tests go by hold where they can be worked out by hand."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import serving_ref as ref
from tests.test_lowbit_binding_cpu import Library

OK, BAD, SMALL = B.SL_OK, B.SL_EINVAL, B.SL_ENOSPC
BF, F, I32, I64, U8 = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.uint8


def call(name, good, **change):
    return getattr(B.lib(), name)(*dict(good, **change).values())


# ---- the library's refusals -------------------------------------------------------------------------
def pages(**change):
    f = dict(page_table=256, seq_len=512, free_pages=768, n_free=1024, n_pages=10, page_slots=64, batch=2, max_pages=5)
    return C.byref(B.sl_kv8_pages(*dict(f, **change).values()))


OTHER = dict(page_table=2256, seq_len=2512, free_pages=2768, n_free=3024)
BAD_PAGES = [dict(page_table=None), dict(seq_len=None), dict(free_pages=None), dict(n_free=None), dict(page_table=258), dict(n_free=1025), dict(n_pages=0),
             dict(n_pages=(1 << 30) + 1), dict(page_slots=48), dict(page_slots=512), dict(batch=0), dict(batch=256), dict(max_pages=0),
             dict(page_slots=256, max_pages=(1 << 22) + 1), dict(batch=255, page_slots=16, max_pages=1 << 23)]
RESIZE = dict(stream=None, source=None, to=None, want=256, cu=256, pos=256, len=None, seq=None, slot=None, m=4, ws=256, ws_bytes=0)


@pytest.mark.parametrize("change", BAD_PAGES)
def test_pages_refuse_a_state(change):
    assert B.lib().sl_kv8_pages_init(None, pages(**change)) == BAD
    both = dict(source=pages(**change), to=pages(**change))
    assert call("sl_kv8_pages_resize", RESIZE, **both) == BAD


@pytest.mark.parametrize("change", [dict(want=None), dict(cu=None), dict(pos=None), dict(want=257), dict(cu=258), dict(pos=258), dict(len=258), dict(seq=257), dict(slot=260),
                                    dict(m=-1), dict(m=(1 << 20) + 1), dict(ws=None), dict(ws=258), dict(want=512), dict(source=None), dict(to=None)])
def test_pages_resize_refuses(change):
    good = dict(RESIZE, source=pages(), to=pages())
    assert call("sl_kv8_pages_resize", good) == SMALL and call("sl_kv8_pages_resize", good, ws_bytes=11) == SMALL
    assert call("sl_kv8_pages_resize", good, **change) == BAD


@pytest.mark.parametrize("change", [dict(n_pages=11), dict(page_slots=32), dict(batch=1), dict(max_pages=4), dict(page_table=256), dict(seq_len=512), dict(free_pages=768),
                                    dict(n_free=1024)])
def test_pages_resize_refuses_states_that_do_not_go_together(change):
    assert call("sl_kv8_pages_resize", RESIZE, source=pages(), to=pages(**OTHER)) == SMALL
    assert call("sl_kv8_pages_resize", RESIZE, source=pages(), to=pages(**dict(OTHER, **change))) == BAD


def test_pages_bytes():
    assert B.sl_kv8_pages_bytes(2) == 12 and B.sl_kv8_pages_bytes(255) == 1024
    out = C.c_size_t()
    assert [B.lib().sl_kv8_pages_bytes(b, C.byref(out)) for b in (0, 256)] == [BAD, BAD] and B.lib().sl_kv8_pages_bytes(1, None) == BAD


FREQS = dict(stream=None, freqs=256, rot=64, theta=1e4, scaling=0, factor=1.0, original=0.0, low=0.0, high=0.0)


@pytest.mark.parametrize("change", [dict(freqs=None), dict(freqs=260), dict(rot=0), dict(rot=63), dict(rot=1026), dict(theta=0.0), dict(theta=float("nan")), dict(theta=float("inf")),
                                    dict(scaling=-1), dict(scaling=4), dict(factor=0.0), dict(factor=float("inf")), dict(scaling=2, rot=2), dict(scaling=3),
                                    dict(scaling=3, original=8e3, low=4.0, high=1.0), dict(scaling=3, original=0.0, low=1.0, high=4.0),
                                    dict(scaling=3, original=float("inf"), low=1.0, high=4.0), dict(scaling=3, original=8e3, low=1.0, high=float("inf"))])
def test_rope_freqs_refuses(change):
    assert call("sl_rope_freqs", FREQS, **change) == BAD


ROPE = dict(stream=None, q=256, qs=512, qo=1 << 20, qos=512, heads=8, k=4096, ks=128, ko=1 << 21, kos=128, kv=2, ti=1, to=1, d=64, rot=32, inter=0, freqs=256, amp=C.c_float(1), pos=256,
            m_dev=256, m=0)


@pytest.mark.parametrize("change", [dict(q=None), dict(qo=None), dict(ko=None), dict(freqs=None), dict(pos=None), dict(m_dev=None), dict(q=257), dict(q=258, ti=0), dict(qo=(1 << 20) + 2, to=0),
                                    dict(freqs=260), dict(pos=258), dict(m_dev=257), dict(qs=511), dict(kos=127), dict(qs=(1 << 40) + 1), dict(heads=0), dict(kv=0),
                                    dict(heads=1 << 15, qs=1 << 30, qos=1 << 30), dict(ti=2), dict(to=-1), dict(d=1), dict(d=1025, qs=1 << 20, qos=1 << 20), dict(rot=0), dict(rot=33),
                                    dict(rot=66), dict(m=-1), dict(m=(1 << 20) + 1), dict(qo=256, qos=520), dict(qo=256, to=0), dict(ko=1 << 20)])
def test_rope_rows_refuses(change):
    assert call("sl_rope_rows", ROPE) == OK                               # no rows: nothing to launch
    assert call("sl_rope_rows", ROPE, qo=256, ko=4096) == OK              # in place
    assert call("sl_rope_rows", ROPE, k=None, ko=None, kv=0, ks=0) == OK  # queries alone
    assert call("sl_rope_rows", ROPE, **change) == BAD


def adapters(**change):
    f = dict(bank=256, bank_bytes=1 << 40, n_slots=4, max_rank=16, n=64, k=128)
    return C.byref(B.sl_adapters(*dict(f, **change).values()))


BAD_ADAPTERS = [dict(bank=None), dict(bank=264), dict(n_slots=0), dict(n_slots=(1 << 16) + 1), dict(max_rank=0), dict(max_rank=257), dict(n=0), dict(n=(1 << 20) + 1), dict(k=4),
                dict(k=132), dict(k=(1 << 20) + 8)]
PACK = dict(stream=None, ad=None, slot=0, rank=3, scale=C.c_float(1), a=256, b=256)
FORWARD = dict(stream=None, ad=None, x=256, which=256, m_dev=256, m=0, base=256, splits=1, y_f32=512, y_bf16=None, ws=256, ws_bytes=0)


@pytest.mark.parametrize("change", BAD_ADAPTERS)
def test_adapters_refuse_a_bank(change):
    ad = adapters(**change)
    assert B.lib().sl_adapters_init(None, ad) == BAD
    assert call("sl_adapters_pack", PACK, ad=ad) == BAD
    assert call("sl_adapters_forward", FORWARD, ad=ad) == BAD


@pytest.mark.parametrize("change", [dict(slot=-1), dict(slot=4), dict(rank=-1), dict(rank=17), dict(a=None), dict(b=None), dict(a=264), dict(b=257), dict(ad=None)])
def test_adapters_pack_refuses(change):
    need = B.sl_adapters_bytes(4, 16, 64, 128)
    for rank in (0, 3):
        assert call("sl_adapters_pack", PACK, ad=adapters(bank_bytes=need - 1), rank=rank) == SMALL
    assert call("sl_adapters_pack", dict(PACK, ad=adapters()), **change) == BAD


@pytest.mark.parametrize("change", [dict(x=None), dict(which=None), dict(m_dev=None), dict(x=264), dict(which=258), dict(m_dev=258), dict(m=-1), dict(m=(1 << 16) + 1), dict(splits=0),
                                    dict(splits=65), dict(y_f32=None), dict(y_bf16=512), dict(base=258), dict(y_f32=514), dict(y_f32=None, y_bf16=513), dict(y_f32=256, splits=2),
                                    dict(y_f32=None, y_bf16=256), dict(ws=None), dict(ws=128)])
def test_adapters_forward_refuses(change):
    good = dict(FORWARD, ad=adapters())
    assert call("sl_adapters_forward", good) == OK                        # no rows: nothing to launch
    assert call("sl_adapters_forward", good, y_f32=256) == OK             # in place
    assert call("sl_adapters_forward", good, base=None) == OK
    assert call("sl_adapters_forward", good, m=1) == SMALL
    assert call("sl_adapters_forward", good, **change) == BAD


def test_adapters_sizes():
    out = C.c_size_t()
    assert B.sl_adapters_bytes(4, 16, 64, 128) == 256 + 4 * (4 * 1024 + 4 * 512)       # two bytes a number
    assert B.sl_adapters_bytes(40, 17, 65, 136) == 512 + 40 * 2 * (5 * 1024 + 5 * 512) # ranks, inputs and outputs up to a tile
    assert B.lib().sl_adapters_bytes(4, 16, 64, 128, None) == BAD and B.lib().sl_adapters_bytes(4, 16, 64, 12, C.byref(out)) == BAD
    assert B.lib().sl_adapters_workspace_bytes(adapters(), -1, C.byref(out)) == BAD and B.lib().sl_adapters_workspace_bytes(adapters(), 1, None) == BAD
    assert B.lib().sl_adapters_workspace_bytes(adapters(), 3, C.byref(out)) == OK and out.value >= 3 * 16 * 4


DRAW = dict(stream=None, logits=256, dtype=1, stride=1000, rows=5, vocab=1000, row_map=None, m_dev=256, m=0, heat=None, k=None, p=None, least=None, u=256, token=256, prob=None, kept=None,
            ws=256, ws_bytes=0)


@pytest.mark.parametrize("change", [dict(logits=None), dict(m_dev=None), dict(u=None), dict(token=None), dict(dtype=2), dict(logits=257), dict(logits=258, dtype=0), dict(stride=999),
                                    dict(stride=(1 << 40) + 1), dict(rows=0), dict(vocab=0), dict(vocab=(1 << 18) + 1, stride=1 << 30), dict(m=-1), dict(m=(1 << 20) + 1), dict(row_map=257),
                                    dict(m_dev=258), dict(heat=258), dict(k=258), dict(p=258), dict(least=258), dict(u=258), dict(token=258), dict(prob=258), dict(kept=258),
                                    dict(ws=None), dict(ws=264)])
def test_sample_filtered_refuses(change):
    assert call("sl_sample_filtered", DRAW) == OK                         # no rows: nothing to launch
    assert call("sl_sample_filtered", DRAW, m=1) == SMALL
    assert call("sl_sample_filtered", DRAW, **change) == BAD


def test_sample_filtered_bytes():
    out = C.c_size_t()
    assert B.sl_sample_filtered_bytes(1, 1) > 0
    for m, v in ((-1, 10), ((1 << 20) + 1, 10), (1, 0), (1, (1 << 18) + 1)):
        assert B.lib().sl_sample_filtered_bytes(m, v, C.byref(out)) == BAD
    assert B.lib().sl_sample_filtered_bytes(1, 1, None) == BAD


# ---- the binding's refusals -------------------------------------------------------------------------
@pytest.fixture
def library(monkeypatch):
    lib = Library(B.lib())
    monkeypatch.setattr(B, "lib", lambda: lib)
    monkeypatch.setattr(B, "_require_gpu", lambda t: None)
    monkeypatch.setattr(B, "_here", lambda: (-1, 0))              # (get_device() of a CPU tensor is -1)
    return lib


class State:
    """A KV8Pages or Adapters without a GPU."""

    def __init__(self, **fields):
        self.device, self.desc_ref = -1, None
        self.__dict__.update(fields)


def ints(*shape):
    return torch.zeros(*shape, dtype=I32)


def resize():
    return dict(pages=State(batch=3, workspace=torch.zeros(16, dtype=U8)), want_len=ints(3), cu_rows=ints(4), row_pos=ints(9), m_upper=9, row_len=ints(9), row_seq=ints(9),
                row_slot=torch.zeros(9, dtype=I64))


def rope():
    return dict(q=torch.zeros(5, 4, 64), q_out=torch.zeros(5, 4, 64, dtype=BF), k=torch.zeros(5, 2, 64), k_out=torch.zeros(5, 2, 64, dtype=BF),
                freqs=torch.zeros(16, dtype=torch.float64), row_pos=ints(5), m_dev=ints(1), m_upper=5)


def forward():
    ad = B.sl_adapters(256, 1 << 40, 2, 16, 40, 64)
    return dict(ad=State(n=40, k=64, desc_ref=C.byref(ad)), x=torch.zeros(3, 64, dtype=BF), row_adapter=ints(3), m_dev=ints(1), m_upper=3, workspace=torch.zeros(4096, dtype=U8),
                base=torch.zeros(2, 3, 40), splits=2, y_bf16=torch.zeros(3, 40, dtype=BF))


def pack():
    return dict(ad=State(n=40, k=64), slot=0, a=torch.zeros(5, 64, dtype=BF), b=torch.zeros(40, 5, dtype=BF))


def draw():
    return dict(logits=torch.zeros(6, 100), m_dev=ints(1), m_upper=6, uniform=torch.zeros(6), token=ints(6), workspace=torch.zeros(256, dtype=U8), temperature=torch.zeros(6), top_k=ints(6),
                top_p=torch.zeros(6), min_p=torch.zeros(6), row_map=ints(6), prob=torch.zeros(6), kept=ints(6))


SHORT = ([("sl_kv8_pages_resize", resize, c) for c in (dict(want_len=ints(2)), dict(cu_rows=ints(3)), dict(row_pos=ints(8)), dict(row_len=ints(8)), dict(row_seq=ints(8)),
                                                       dict(row_slot=torch.zeros(8, dtype=I64)), dict(row_slot=ints(9)), dict(want_len=torch.zeros(3, dtype=I64)),
                                                       dict(to=State(batch=3, workspace=torch.zeros(16, dtype=U8), device=1)))]
         + [("sl_rope_rows", rope, c) for c in (dict(q=torch.zeros(4, 4, 64)), dict(q_out=torch.zeros(4, 4, 64)), dict(q_out=torch.zeros(5, 4, 32)), dict(k=torch.zeros(5, 2, 64, dtype=BF)),
                                                dict(k_out=torch.zeros(5, 2, 64)), dict(k_out=torch.zeros(4, 2, 64, dtype=BF)), dict(freqs=torch.zeros(16)), dict(row_pos=ints(4)),
                                                dict(m_dev=ints(0)), dict(q=torch.zeros(5, 4, 128)[..., ::2]), dict(q=torch.zeros(5, 4, 64, dtype=torch.float16)))]
         + [("sl_adapters_forward", forward, c) for c in (dict(x=torch.zeros(2, 64, dtype=BF)), dict(x=torch.zeros(3, 64)), dict(row_adapter=ints(2)), dict(m_dev=ints(0)),
                                                          dict(base=torch.zeros(1, 3, 40)), dict(y_bf16=torch.zeros(2, 40, dtype=BF)), dict(y_bf16=None, y_f32=torch.zeros(2, 40)),
                                                          dict(base=torch.zeros(2, 3, 40, dtype=BF)))]
         + [("sl_adapters_pack", pack, c) for c in (dict(a=torch.zeros(5, 72, dtype=BF)), dict(b=torch.zeros(40, 4, dtype=BF)), dict(a=torch.zeros(5, 64)), dict(b=torch.zeros(40, 5)),
                                                    dict(b=torch.zeros(5, 40, dtype=BF).T))]
         + [("sl_sample_filtered", draw, c) for c in (dict(uniform=torch.zeros(5)), dict(token=ints(5)), dict(temperature=torch.zeros(5)), dict(top_k=ints(5)), dict(top_k=torch.zeros(6)),
                                                      dict(top_p=torch.zeros(5)), dict(min_p=torch.zeros(5)), dict(row_map=ints(5)), dict(prob=torch.zeros(5)), dict(kept=ints(5)),
                                                      dict(logits=torch.zeros(5, 100), row_map=None), dict(logits=torch.zeros(6, 200)[:, ::2]),
                                                      dict(logits=torch.zeros(6, 100, dtype=torch.float16)))])


@pytest.mark.parametrize("name,good,change", SHORT, ids=[f"{n}-{'-'.join(c)}-{i}" for i, (n, _, c) in enumerate(SHORT)])
def test_a_buffer_that_does_not_fit_is_refused(library, name, good, change):
    getattr(B, name)(**good())
    assert library.calls == [name]
    with pytest.raises(ValueError):
        getattr(B, name)(**dict(good(), **change))
    assert library.calls == [name]                                # nothing was launched


def test_a_scaling_that_is_none_is_refused(library):
    f = torch.zeros(8, dtype=torch.float64)
    B.sl_rope_freqs(f, 1e4)
    with pytest.raises(ValueError):
        B.sl_rope_freqs(f, 1e4, scaling="cubic")
    assert library.calls == ["sl_rope_freqs"]


def test_no_rows_is_nothing_to_do(library):
    B.sl_rope_rows(**dict(rope(), m_upper=0))
    B.sl_adapters_forward(**dict(forward(), m_upper=0))
    B.sl_sample_filtered(**dict(draw(), m_upper=0))
    assert library.calls == []
    B.sl_kv8_pages_resize(**dict(resize(), m_upper=0))            # (sequences may still give up pages)
    assert library.calls == ["sl_kv8_pages_resize"]


# ---- the definitions ---------------------------------------------------------------------------------
def test_pages_by_hand():
    table, lens, stack, n_free, cu, rows = ref.pages_resize([[4, 2, -1], [7, -1, -1], [0, 1, 5]], [20, 3, 40], [3, 6, 9, 8], 2, [0, 30, 41], 16, 10, 100)
    # the first gives up 4 and 2; the second takes 4; 2 goes on top of the stack; the third has room on its page
    assert table == [[-1, -1, -1], [7, 4, -1], [0, 1, 5]] and lens == [0, 30, 41]
    assert n_free == 3 and stack == [3, 6, 2, 8]
    assert cu == [0, 0, 27, 28] and rows[0] == (3, 1, 7 * 16 + 3) and rows[13] == (16, 1, 4 * 16) and rows[27] == (40, 2, 5 * 16 + 8)


def test_draws_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [ref.sample(z, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.99)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert ref.sample(z, 0.5, top_k=2)[::2] == (1, 2) and ref.sample(z, 0.6, top_k=2)[::2] == (3, 2)
    assert ref.sample(z, 0.99, top_p=0.65)[::2] == (3, 2) and ref.sample(z, 0.99, top_p=0.75)[2] == 3
    assert ref.sample(z, 0.5, min_p=0.6)[2] == 2 and ref.sample(z, 0.5, temperature=0.0) == (1, 1.0, 1)
    assert abs(ref.sample(z, 0.6, top_k=2)[1] - 3 / 7) < 1e-12 and ref.sample(np.full(4, -np.inf), 0.5) == (0, 0.0, 0)


def test_turns_by_hand():
    x = np.array([[[1.0, 0.0, 5.0]]])
    y, mass = ref.rope_rows(x, [1], [0.25], True, 2.0)
    assert np.allclose(y, [[[0.0, 2.0, 5.0]]]) and mass.tolist() == [[[2.0, 2.0, 0.0]]]
    f = ref.rope_freqs(4, 100.0)
    assert np.allclose(f * 2 * np.pi, [1.0, 0.1])
    assert np.allclose(ref.rope_freqs(4, 100.0, "linear", 4.0), f / 4) and np.allclose(ref.rope_freqs(4, 100.0, "base", 4.0) * 2 * np.pi, [1.0, 1600 ** -0.5])
    assert np.allclose(ref.rope_freqs(4, 100.0, "turns", 4.0, 2 * np.pi * 10, 1.0, 10.0), [f[0], f[1] / 4])


@pytest.mark.parametrize("change", [dict(a=None), dict(b=None)])
def test_half_an_adapter_is_refused(library, change):
    with pytest.raises(ValueError):
        B.sl_adapters_pack(**dict(pack(), **change))
    assert library.calls == []
    B.sl_adapters_pack(**dict(pack(), a=None, b=None))            # (empties the slot)
    assert library.calls == ["sl_adapters_pack"]


def test_keys_without_a_place_for_them_are_refused(library):
    with pytest.raises(ValueError):
        B.sl_rope_rows(**dict(rope(), k_out=None))
    assert library.calls == []
    B.sl_rope_rows(**dict(rope(), k=None, k_out=None))
    B.sl_rope_rows(**dict(rope(), k=None))                        # (k_out is not looked at)
    assert library.calls == ["sl_rope_rows"] * 2
