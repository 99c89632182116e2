"""The 8-bit cache's definitions in 64 bits (NumPy), for the tests of the operators around it."""
import numpy as np
import torch

PAGE = 16
TOP = {"e4m3": 448.0, "int8": 127.0}
DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TINY = 2.0 ** -110


def code_values(codes: torch.Tensor) -> np.ndarray:
    return codes.cpu().float().numpy().astype(np.float64)


def quantise(x32: np.ndarray, fmt: str):
    """Codes (torch, CPU) and fp32 scales of fp32 rows [..., D], product by product as the format says."""
    x32 = np.asarray(x32, dtype=np.float32)
    a = np.abs(x32).max(-1)
    bad = ~np.isfinite(x32).all(-1)
    live = ~bad & (a >= TINY)
    one = np.float32(1)
    inv = np.float32(TOP[fmt]) * (one / np.where(live, a, one))
    scale = np.where(live, a * (one / np.float32(TOP[fmt])), np.float32(0)).astype(np.float32)
    scale[bad] = np.nan
    y = np.where(live[..., None], np.where(live[..., None], x32, 0) * inv[..., None].astype(np.float32), np.float32(0)).astype(np.float32)
    y = torch.from_numpy(np.ascontiguousarray(y))
    codes = torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
    return codes, scale


def rotated(x: np.ndarray, pos, freq, magnitude: float, layout: str) -> np.ndarray:
    """x [N, H, D] turned at positions [N], as complex numbers."""
    freq = np.asarray(freq, dtype=np.float64)
    half = len(freq)
    z = magnitude * np.exp(1j * (np.asarray(pos, dtype=np.float64)[:, None] * freq))[:, None]
    out = np.array(x, dtype=np.float64)
    i, j = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    w = (out[..., i] + 1j * out[..., j]) * z
    out[..., i], out[..., j] = w.real, w.imag
    return out


def turn_slack(x: np.ndarray, freq, magnitude: float, layout: str) -> np.ndarray:
    """How far fp32 rotation may be from rotated(): per element, for the pair's |x| + |y|: the angle's fraction of a turn rounded to
    fp32 (2^-25 of a turn, 1.9e-7), sine and cosine (2 ulp, 1.2e-7), magnitude, two products and their sum (2^-24 each)."""
    out = np.zeros(x.shape)
    half = len(freq)
    i, j = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    s = np.abs(x[..., i]) + np.abs(x[..., j])
    out[..., i] = out[..., j] = s
    return out * abs(magnitude) * (1.9e-7 + 1.2e-7 + 4 * 2.0 ** -24)


def attention(q, k, v, n: int, G: int, scale: float, want_pages: bool = False, rows=None):
    """One sequence.  q [G, Hq, D], k and v [n, Hkv, D] float64 values.  Row t sees keys 0 .. n - G + t.  Returns (out [G, Hq, D], the mean
    |v| under the weights [G, Hq, D], the largest sum_d |q_d k_d| * scale, page scores or None)."""
    Gq, Hq, D = q.shape
    Hkv = k.shape[1]
    g = Hq // Hkv
    out, spread = np.zeros((G, Hq, D)), np.zeros((G, Hq, D))
    per_token = np.zeros(max(n, 1))
    l1 = 0.0
    if n > 0:
        seen = np.arange(n)[None] <= n - G + np.arange(G)[:, None]                      # [G, n]
        for h in range(Hkv):
            qh = q[:, h * g:(h + 1) * g].reshape(G * g, D)
            logits = (qh @ k[:, h].T * scale).reshape(G, g, n)
            l1 = max(l1, float((np.abs(qh) @ np.abs(np.nan_to_num(k[:, h])).T).max()) * scale)
            logits = np.where(seen[:, None], logits, -np.inf)
            top = logits.max(-1, keepdims=True)
            w = np.where(seen[:, None], np.exp(logits - np.where(np.isfinite(top), top, 0.0)), 0.0)
            total = w.sum(-1, keepdims=True)
            w = w / np.where(total > 0, total, 1.0)
            out[:, h * g:(h + 1) * g] = (w.reshape(G * g, n) @ v[:, h]).reshape(G, g, D)
            spread[:, h * g:(h + 1) * g] = (w.reshape(G * g, n) @ np.abs(v[:, h])).reshape(G, g, D)
            if want_pages:
                per_token += w[rows].sum((0, 1))
    scores = None
    if want_pages:
        pages = -(-n // PAGE)
        scores = np.pad(per_token[:n], (0, pages * PAGE - n)).reshape(pages, PAGE).sum(-1) / (len(rows) * Hq)
    return out, spread, l1, scores


def weight_slack(l1: float, D: int) -> float:
    """How far a weight may be off, relative: its logit's fp32 accumulation of D exact products ((D + 8) 2^-24 of the sum of magnitudes,
    every rounding aligned), exponential and reference (2^-20)."""
    return (D + 8) * 2.0 ** -24 * l1 + 2.0 ** -20


def out_tolerance(out, spread, l1: float, D: int):
    """bf16 output (half a step, 2^-8 of the value) of weights rounded to bf16 (2^-8 of each, all aligned; the sum has them
    unrounded) that are off by weight_slack twice (numerator and sum)."""
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * weight_slack(l1, D)) * spread + 1e-30
