"""Plain definitions of the low-bit operators in 64 bits (not collected by pytest): what sl_linear_q4_* and sl_kv8_* compute,
written from their definitions with NumPy.  Roundings that belong to a definition (scales, quotients) are taken in fp32."""
import numpy as np
import torch


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def bf16(x):
    """Rounded to bf16, as float64."""
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


# ---- 4-bit weights -----------------------------------------------------------------------------
def q4_quantize(w, group, with_zeros):
    """w: float64 array holding fp32 or bf16 values -> codes [n, k], scales (float64 of bf16), zeros."""
    n, k = w.shape
    groups = -(-k // group)
    codes, scales, zeros = np.zeros((n, k), np.uint8), np.zeros((n, groups)), np.full((n, groups), 8, np.uint8)
    f = np.float32
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group].astype(f)
        finite = np.isfinite(part).all(1)
        safe = np.where(finite[:, None], part, f(0))
        lo, hi = np.minimum(safe.min(1), f(0)), np.maximum(safe.max(1), f(0))
        s = bf16((hi - lo) / f(15) if with_zeros else np.maximum(hi, -lo) / f(7)).astype(f)
        some = s > 0
        one = np.where(some, s, f(1))
        z = np.clip(np.rint(-lo / one), 0, 15) if with_zeros else np.full(n, f(8))
        z = np.where(some & finite, z, 0.0 if with_zeros else 8.0).astype(f)
        c = np.clip(np.rint(safe / one[:, None]) + z[:, None], 0, 15)
        c = np.where((some & finite)[:, None], c, z[:, None])
        codes[:, g * group:(g + 1) * group], scales[:, g], zeros[:, g] = c, np.where(finite, s, np.nan), z
    return codes, scales, zeros


def q4_pack_nibbles(codes):
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def q4_weights(codes, scales, zeros, group):
    k = codes.shape[1]
    spread = lambda a: np.repeat(a.astype(np.float64), group, 1)[:, :k]  # noqa: E731
    return spread(scales) * (codes.astype(np.float64) - spread(zeros))


def q4_bound(x, codes, scales, zeros, group):
    """|error| of the product in fp32, any order of summation: the kernel sums x q and x apart, k terms each."""
    k = codes.shape[1]
    spread = lambda a: np.repeat(a.astype(np.float64), group, 1)[:, :k]  # noqa: E731
    most = np.abs(spread(scales)) * (codes + spread(zeros))
    return (k + 16) * 2.0 ** -24 * (np.abs(x) @ most.T)


# ---- the 8-bit cache -----------------------------------------------------------------------------
def kv8_codes(x):
    """x [.., d] float64 (fp32 or bf16 values) -> codes, scale; all quotients in fp32."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        peak = np.abs(x).max(-1, keepdims=True)
        scale = np.where(np.isfinite(peak), peak / np.float32(127), np.float32(np.nan)).astype(np.float32)
        code = np.where(scale > 0, np.clip(np.rint(x / np.where(scale > 0, scale, np.float32(1))), -127, 127), 0)
    return np.nan_to_num(code), scale


def kv8_values(x):
    """What the cache holds of x, as float64."""
    code, scale = kv8_codes(x)
    return code * scale.astype(np.float64)


def kv8_attention(q, K, V, limit, scale, absent=()):
    """q [H, d], K, V [slots, Hkv, d] (float64) -> (o [H, d], sum P|V|, largest |score| mass) over slots < limit not in absent."""
    H, d = q.shape
    share = H // K.shape[1]
    seen = [p for p in range(max(0, min(limit, K.shape[0]))) if p not in absent]
    out, mass, size = np.zeros((H, d)), np.zeros((H, d)), np.zeros(H)
    if not seen:
        return out, mass, size
    for h in range(H):
        k, v = K[seen, h // share], V[seen, h // share]
        s = scale * (k @ q[h])
        with np.errstate(all="ignore"):
            p = np.exp(s - s.max())
            p /= p.sum()
        out[h], mass[h] = p @ v, p @ np.abs(v)
        size[h] = scale * np.max(np.abs(k) @ np.abs(q[h]))
    return out, mass, size


def kv8_attention_bound(mass, size, slots, d, dtype):
    """|error| of one output element: a score's error (fp32 sums of d terms, four more roundings) moves a probability by as much
    relative to itself, and the normaliser again; a probability times V's scale goes in with 16 bits (bf16 results) or 23 (fp32: three
    parts of 8 bits, the last rounded); exponential and its argument, the sums over the slots and the join of partial
    results: slots + 64 roundings of fp32.  Then the result's own rounding, half a step."""
    e = 2.0 ** -24
    rel = 2 * (d + 8) * e * size[..., None] + (2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -23) + (slots + 64) * e
    return rel * mass


def half_step(x, dtype):
    return np.abs(x) * torch.finfo(dtype).eps / 2 + 1e-37
