"""The calls of one serving step in a row, as a program uses them: room for the new rows, the fused projection with 4-bit weights and each request's
adapter, rotary positions, the write into the cache, attention in causal order, and a draw from logits; eager and as a graph.

Every stage is checked against its definition on what the stage before left, so bounds are those of the single calls."""
import math

import numpy as np
import pytest
import torch

from paper_2602_06412_amd import binding as B
from tests import lowbit_ref as low
from tests import serving_ref as ref
from tests.gpu_util import DEV, dev

pytestmark = pytest.mark.gpu
BF, F, I32 = torch.bfloat16, torch.float32, torch.int32
H, HKV, D, K, GROUP, VOCAB, PAGE, BATCH = 8, 2, 64, 256, 64, 1024, 16, 3
N = (H + 2 * HKV) * D
M = 128                                                           # bound on the rows of a step


class Program:
    """What a serving program holds for one layer."""

    def __init__(self):
        g = torch.Generator().manual_seed(1)
        w = 0.06 * torch.randn(N, K, generator=g)
        self.codes, self.scales, self.zeros = low.q4_quantize(low.f64(w), GROUP, False)
        self.packed = torch.empty(B.sl_linear_q4_bytes(N, K, GROUP), dtype=torch.uint8, device=DEV)
        B.sl_linear_q4_pack(dev(low.q4_pack_nibbles(self.codes)), dev(self.scales, BF), None, N, K, GROUP, self.packed)
        self.ad, self.weights = B.Adapters(2, 16, N, K), {}
        for slot, rank in ((0, 16), (1, 5)):
            a, b = (torch.randn(rank, K, generator=g) / 16).to(BF), (torch.randn(N, rank, generator=g) / 8).to(BF)
            B.sl_adapters_pack(self.ad, slot, a.to(DEV), b.to(DEV), 0.7)
            self.weights[slot] = (low.f64(a), low.f64(b), 0.7)
        self.pages = B.KV8Pages(24, PAGE, BATCH, 8)
        self.kv = B.KV8(24, PAGE, HKV, D, self.pages.page_table)
        self.freqs = torch.empty(D // 2, dtype=torch.float64, device=DEV)
        B.sl_rope_freqs(self.freqs, 10000.0)
        new = lambda *shape, dtype=F: torch.zeros(*shape, dtype=dtype, device=DEV)  # noqa: E731
        self.want, self.cu, self.pos, self.len, self.seq = new(BATCH, dtype=I32), new(BATCH + 1, dtype=I32), *(new(M, dtype=I32) for _ in range(3))
        self.request_adapter = dev([1, -1, 0], I32)
        self.x, self.which = new(M, K, dtype=BF), new(M, dtype=I32)
        self.y, self.qkv = new(1, M, N), new(M, N)
        self.q, self.k, self.out = new(M, H, D, dtype=BF), new(M, HKV, D, dtype=BF), new(M, H, D, dtype=BF)
        self.head = (torch.randn(VOCAB, H * D, generator=g) / 4).to(BF).to(DEV)
        self.logits, self.uniform, self.token = new(M, VOCAB, dtype=BF), new(M), new(M, dtype=I32)
        self.top_k, self.top_p = dev([20] * M, I32), dev([0.9] * M, F)
        u8 = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)  # noqa: E731
        self.ws_ad, self.ws_attn = u8(B.sl_adapters_workspace_bytes(self.ad, M)), u8(B.sl_kv8_attention_bytes(self.kv, H, M, 8 * PAGE))
        self.ws_draw = u8(B.sl_sample_filtered_bytes(M, VOCAB))

    def step(self):
        m = self.cu[BATCH:]
        B.sl_kv8_pages_resize(self.pages, self.want, self.cu, self.pos, M, row_len=self.len, row_seq=self.seq)
        torch.index_select(self.request_adapter, 0, self.seq, out=self.which)
        B.sl_linear_q4_forward(self.x, self.packed, m, M, N, K, GROUP, y_f32=self.y[0])
        B.sl_adapters_forward(self.ad, self.x, self.which, m, M, self.ws_ad, base=self.y, y_f32=self.qkv)
        q, k, v = self.qkv[:, :H * D].view(M, H, D), self.qkv[:, H * D:(H + HKV) * D].view(M, HKV, D), self.qkv[:, (H + HKV) * D:].view(M, HKV, D)
        B.sl_rope_rows(q, self.q, k, self.k, self.freqs, self.pos, m, M)
        B.sl_kv8_write(self.kv, self.k, v.to(BF), self.pos, self.cu, M)
        B.sl_kv8_attention(self.kv, self.q, self.cu, self.pages.seq_len, M, 8 * PAGE, 1 / math.sqrt(D), self.out, self.ws_attn, row_len=self.len)
        torch.mm(self.out.view(M, H * D), self.head.T, out=self.logits)
        B.sl_sample_filtered(self.logits, m, M, self.uniform, self.token, self.ws_draw, top_k=self.top_k, top_p=self.top_p)


STEPS = [[20, 33, 0], [21, 34, 17], [22, 0, 18], [22, 50, 19]]    # prompts; one more each, and a new request; one ends; another takes its place


def check_step(p, want, lens, cached):
    """cached: {sequence: (K, V) float64} of what the cache holds, grown here."""
    f64 = low.f64
    rows = [(b, s) for b, (o, w) in enumerate(zip(lens, want)) for s in range(o, w)]
    m = len(rows)
    assert p.pages.seq_len.tolist() == want and p.cu.tolist() == np.cumsum([0] + [max(0, w - o) for o, w in zip(lens, want)]).tolist()
    assert list(zip(p.seq[:m].tolist(), p.pos[:m].tolist())) == rows
    x, which = f64(p.x)[:m], [[1, -1, 0][b] for b, _ in rows]
    w = low.q4_weights(p.codes, p.scales, p.zeros, GROUP)
    assert (np.abs(f64(p.y[0])[:m] - x @ w.T) <= low.q4_bound(x, p.codes, p.scales, p.zeros, GROUP) + 1e-30).all()
    want_qkv, bound = ref.adapters(x, f64(p.y)[:, :m], which, p.weights)
    qkv = f64(p.qkv)[:m]
    assert (np.abs(qkv - want_qkv) <= bound + low.half_step(want_qkv, F)).all()
    q, k, v = qkv[:, :H * D].reshape(m, H, D), qkv[:, H * D:(H + HKV) * D].reshape(m, HKV, D), qkv[:, (H + HKV) * D:].reshape(m, HKV, D)
    pos = np.array([s for _, s in rows])
    for got, raw in ((p.q, q), (p.k, k)):
        turned, mass = ref.rope_rows(raw, pos, f64(p.freqs), False, 1.0)
        assert (np.abs(f64(got)[:m] - turned) <= ref.rope_bound(turned, mass, torch.finfo(BF).eps)).all()
    for b, (o, n) in enumerate(zip(lens, want)):
        if n < o:
            cached[b] = tuple(c[:n] for c in cached[b])
    for r, (b, s) in enumerate(rows):
        for i, new in enumerate((f64(p.k)[r], low.bf16(v[r]))):
            cached[b][i].append(low.kv8_values(new))
    for r, (b, s) in enumerate(rows):
        kk, vv = np.array(cached[b][0]), np.array(cached[b][1])
        o, mass, size = low.kv8_attention(f64(p.q)[r], kk, vv, s + 1, 1 / math.sqrt(D))
        bound = low.kv8_attention_bound(mass, size, s + 1, D, BF) + low.half_step(o, BF) * 1.01
        assert (np.abs(f64(p.out)[r] - o) <= bound).all()
        token = ref.sample(f64(p.logits)[r], f64(p.uniform)[r], top_k=20, top_p=float(np.float32(0.9)))[0]
        assert p.token[r].item() == token
    return m


@pytest.mark.parametrize("captured", [False, True])
def test_steps_of_several_requests(captured):
    p, graph = Program(), None
    lens, cached = [0] * BATCH, {b: ([], []) for b in range(BATCH)}
    if captured:
        with torch.cuda.stream(torch.cuda.Stream()):
            p.step()                                              # (wants nothing: first calls, libraries and all)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.step()
    g = torch.Generator().manual_seed(5)
    for i, want in enumerate(STEPS):
        p.want.copy_(torch.tensor(want))
        p.x.copy_(torch.randn(M, K, generator=g).to(BF))
        p.uniform.copy_(torch.rand(M, generator=g))
        before = p.token.clone()
        torch.cuda.synchronize()
        graph.replay() if captured else p.step()
        torch.cuda.synchronize()
        cached = {b: (list(c[0]), list(c[1])) for b, c in cached.items()}
        m = check_step(p, want, lens, cached)
        assert torch.equal(p.token[m:], before[m:])
        lens = want
