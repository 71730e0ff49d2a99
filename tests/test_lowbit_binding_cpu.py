"""The binding of the low-bit calls compares every buffer with the sizes that the library will read and write (no GPU: the library is
replaced by one that takes note of its calls, tensors stand on the CPU)."""
import pytest
import torch

from paper_2602_06412_amd import binding as B

BF, F, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Library:
    """Size queries go to the real one, launches are noted."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)

        def noted(*args):
            self.calls.append(name)
            return B.SL_OK
        return noted


@pytest.fixture
def library(monkeypatch):
    lib = Library(B.lib())
    monkeypatch.setattr(B, "lib", lambda: lib)
    monkeypatch.setattr(B, "_require_gpu", lambda t: None)
    monkeypatch.setattr(B, "_here", lambda: (-1, 0))              # (get_device() of a CPU tensor is -1)
    return lib


def ints(*shape):
    return torch.zeros(*shape, dtype=I32)


def linear():
    return dict(x=torch.zeros(3, 256, dtype=BF), packed=torch.zeros(B.sl_linear_q4_bytes(40, 256, 32), dtype=U8), m_dev=ints(1), m_upper=3, n=40, k=256,
                group=32, y_bf16=torch.zeros(3, 40, dtype=BF), row_map=ints(3))


def quantize():
    return dict(w=torch.zeros(40, 264), group=64, codes=torch.zeros(40, 132, dtype=U8), scales=torch.zeros(40, 5, dtype=BF),
                zeros=torch.zeros(40, 5, dtype=U8))


def pack():
    return dict(codes=torch.zeros(40, 132, dtype=U8), scales=torch.zeros(40, 5, dtype=BF), zeros=torch.zeros(40, 5, dtype=U8), n=40, k=264, group=64,
                packed=torch.zeros(B.sl_linear_q4_bytes(40, 264, 64), dtype=U8))


def cache():
    return B.KV8(6, 16, 2, 64, ints(2, 3))


def rows():
    return dict(kv=cache(), k=torch.zeros(5, 2, 64), v=torch.zeros(5, 2, 64), row_pos=ints(5), cu_rows=ints(3), m_upper=5)


def read():
    a = rows()
    return dict(a, k_out=a.pop("k"), v_out=a.pop("v"))


def attention():
    return dict(kv=cache(), q=torch.zeros(5, 4, 64), cu_rows=ints(3), seq_len=ints(2), m_upper=5, len_upper=48, scale=0.1, out=torch.zeros(5, 4, 64),
                workspace=torch.zeros(256, dtype=U8), row_len=ints(5))


SHORT = [
    ("sl_linear_q4_forward", linear, dict(x=torch.zeros(2, 256, dtype=BF))),
    ("sl_linear_q4_forward", linear, dict(x=torch.zeros(3, 248, dtype=BF))),
    ("sl_linear_q4_forward", linear, dict(packed=torch.zeros(B.sl_linear_q4_bytes(40, 256, 128), dtype=U8))),       # of another group
    ("sl_linear_q4_forward", linear, dict(packed=torch.zeros(B.sl_linear_q4_bytes(24, 256, 32), dtype=U8))),        # of another shape
    ("sl_linear_q4_forward", linear, dict(m_dev=ints(0))),
    ("sl_linear_q4_forward", linear, dict(row_map=ints(2))),
    ("sl_linear_q4_forward", linear, dict(y_bf16=torch.zeros(2, 40, dtype=BF), row_map=None)),
    ("sl_linear_q4_forward", linear, dict(y_bf16=None, row_map=None, y_f32=torch.zeros(2, 40))),
    ("sl_linear_q4_quantize", quantize, dict(codes=torch.zeros(40, 131, dtype=U8))),
    ("sl_linear_q4_quantize", quantize, dict(scales=torch.zeros(40, 4, dtype=BF))),
    ("sl_linear_q4_quantize", quantize, dict(zeros=torch.zeros(39, 5, dtype=U8))),
    ("sl_linear_q4_quantize", quantize, dict(w=torch.zeros(40, 264, dtype=torch.float16))),
    ("sl_linear_q4_pack", pack, dict(codes=torch.zeros(39, 132, dtype=U8))),
    ("sl_linear_q4_pack", pack, dict(scales=torch.zeros(40, 4, dtype=BF))),
    ("sl_linear_q4_pack", pack, dict(zeros=torch.zeros(40, 4, dtype=U8))),
    ("sl_kv8_write", rows, dict(k=torch.zeros(4, 2, 64))),
    ("sl_kv8_write", rows, dict(v=torch.zeros(4, 2, 64))),
    ("sl_kv8_write", rows, dict(row_pos=ints(4))),
    ("sl_kv8_write", rows, dict(cu_rows=ints(2))),
    ("sl_kv8_write", rows, dict(k=torch.zeros(5, 2, 64, dtype=torch.float16), v=torch.zeros(5, 2, 64, dtype=torch.float16))),
    ("sl_kv8_read", read, dict(k_out=torch.zeros(4, 2, 64))),
    ("sl_kv8_read", read, dict(v_out=torch.zeros(4, 2, 64))),
    ("sl_kv8_read", read, dict(row_pos=ints(4))),
    ("sl_kv8_read", read, dict(cu_rows=ints(2))),
    ("sl_kv8_attention", attention, dict(q=torch.zeros(4, 4, 64))),
    ("sl_kv8_attention", attention, dict(out=torch.zeros(4, 4, 64))),
    ("sl_kv8_attention", attention, dict(cu_rows=ints(2))),
    ("sl_kv8_attention", attention, dict(seq_len=ints(1))),
    ("sl_kv8_attention", attention, dict(row_len=ints(4))),
    ("sl_kv8_attention", attention, dict(q=torch.zeros(5, 4, 64, dtype=torch.float16), out=torch.zeros(5, 4, 64, dtype=torch.float16))),
]


@pytest.mark.parametrize("name,good,change", SHORT, ids=[f"{n}-{'-'.join(c)}-{i}" for i, (n, _, c) in enumerate(SHORT)])
def test_a_buffer_that_is_too_small_is_refused(library, name, good, change):
    getattr(B, name)(**good())
    assert library.calls == [name]
    with pytest.raises(ValueError):
        getattr(B, name)(**dict(good(), **change))
    assert library.calls == [name]                            # nothing was launched


def test_a_scattered_result_may_have_any_number_of_rows(library):
    B.sl_linear_q4_forward(**dict(linear(), y_bf16=torch.zeros(1, 40, dtype=BF)))
    assert library.calls == ["sl_linear_q4_forward"]


def test_larger_buffers_than_needed_are_fine(library):
    a = linear()
    B.sl_linear_q4_forward(**dict(a, x=torch.zeros(9, 256, dtype=BF), packed=torch.zeros(a["packed"].numel() + 5, dtype=U8), row_map=ints(7)))
    a = attention()
    B.sl_kv8_attention(**dict(a, q=torch.zeros(9, 4, 64), out=torch.zeros(8, 4, 64), cu_rows=ints(9), seq_len=ints(9), row_len=ints(9)))
    assert len(library.calls) == 2


def test_shapes_that_the_library_refuses_reach_it(library):
    """A group, size or count out of range is the library's to report, with its own status."""
    for change in (dict(group=48), dict(k=260), dict(n=0), dict(m_upper=-1)):
        B.sl_linear_q4_forward(**dict(linear(), **change))
    assert len(library.calls) == 4


def test_a_pool_that_is_not_dense_is_refused(library):
    need = B.sl_kv8_bytes(6, 16, 2, 64)
    B.KV8(6, 16, 2, 64, ints(2, 3), torch.zeros(need, dtype=U8))
    for pool in (torch.zeros(2 * need, dtype=U8)[::2], torch.zeros(need - 1, dtype=U8)):
        with pytest.raises(ValueError):
            B.KV8(6, 16, 2, 64, ints(2, 3), pool)


def test_one_sequence_of_a_cache(library):
    kv = B.KV8(6, 16, 2, 64, torch.arange(6, dtype=I32).view(2, 3))
    assert kv.sequence(1).page_table.tolist() == [[3, 4, 5]] and kv.sequence(-1).page_table.tolist() == [[3, 4, 5]]
    for b in (2, -3):
        with pytest.raises(IndexError):
            kv.sequence(b)


# ---- the library's own refusal ----------------------------------------------------------------------
def test_a_scale_that_overflows_in_powers_of_two_is_refused():
    """Scores are taken in powers of two, so scale log2(e) has to be finite (2.35e38 is, 2.37e38 is not)."""
    kv = B.C.byref(B.sl_kv8(256, 1 << 40, 256, 10, 64, 4, 128, 2, 5))
    call = lambda scale: B.lib().sl_kv8_attention(None, kv, 256, 1, 1024, 8, 256, 256, None, 0, 100, scale, 256, 1024, 256, 1 << 40)  # noqa: E731
    assert call(2.35e38) == B.SL_OK                           # (no rows: nothing to launch)
    assert call(2.37e38) == B.SL_EINVAL and call(3.4e38) == B.SL_EINVAL
