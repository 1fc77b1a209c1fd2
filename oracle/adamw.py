"""AdamW of one tensor on the host: the step in fp64, the moments by their definition (fp32 operations, each rounded), in 32 or 8 bits."""
from __future__ import annotations

import numpy as np

f32 = np.float32
BLOCK = 256


class State:
    """m, v as fp32 values; in 8 bits also the codes cm, cu and the scales of their blocks."""

    def __init__(self, n: int, bits: int):
        self.bits = bits
        self.m, self.v = np.zeros(n, f32), np.zeros(n, f32)
        self.cm, self.cu = np.zeros(n, np.int8), np.zeros(n, np.uint8)


def chances(n: int, t: int, tensor: int, seed: int):
    """Two numbers in (0, 1) per element, from SplitMix64's finaliser."""
    M = (1 << 64) - 1
    out = np.empty((2, n), f32)
    for e in range(0, n, 2):
        z = (seed ^ (t * 0x9E3779B97F4A7C15)) & M
        z ^= (((tensor << 40) + e // 2) * 0xC2B2AE3D27D4EB4F) & M
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M
        z ^= z >> 31
        for k in range(min(2, n - e)):
            w = z >> (32 * k)
            out[0, e + k] = ((w & 0xFFFF) + 0.5) / 65536
            out[1, e + k] = ((w >> 16 & 0xFFFF) + 0.5) / 65536
    return out


def hold(x: np.ndarray, L: int, a: np.ndarray):
    """Codes (magnitudes) and values of x: block by block."""
    codes, values = np.zeros(len(x), np.int32), np.zeros(len(x), f32)
    for b in range(0, len(x), BLOCK):
        y = np.abs(x[b:b + BLOCK])
        top = y.max()
        if top < f32(2.0 ** -60):
            continue
        scale = f32(top * f32(1.0 / (L * L)))
        y = (y * f32(f32(1) / scale)).astype(f32)
        c = np.minimum(np.floor(np.sqrt(y.astype(np.float64))), L)
        rest = y.astype(np.float64) - c * c                          # exact, in fp32 as well
        c = c + ((rest > (a[b:b + BLOCK] * (2 * c + 1).astype(f32)).astype(f32)) & (c < L))
        if L == 255:
            c = np.where((c == 0) & (x[b:b + BLOCK] > 0), 1, c)
        codes[b:b + BLOCK] = c
        values[b:b + BLOCK] = (c * c).astype(f32) * scale
    return codes, values


def step(s: State, p: np.ndarray, grad: np.ndarray, t: int, tensor: int, lr, b1, b2, eps, decay, grad_scale, seed):
    """The new parameters in fp64 from p (fp64), and the largest step that the parts of m and the decay could add up to; s is advanced."""
    g = grad.astype(f32) * f32(grad_scale)
    b1, b2 = float(f32(b1)), float(f32(b2))                          # one number throughout: 1 - b belongs to the powers of b
    n1, n2 = f32(1) - f32(b1), f32(1) - f32(b2)
    m = s.m * f32(b1) + g * n1
    v = s.v * f32(b2) + (g * n2) * g
    md = s.m.astype(np.float64) * float(f32(b1)) + g.astype(np.float64) * float(n1)
    vd = s.v.astype(np.float64) * float(f32(b2)) + g.astype(np.float64) ** 2 * float(n2)
    root = np.sqrt(vd / (1 - b2 ** t)) + eps
    new = p - lr * (decay * p + (md / (1 - b1 ** t)) / root)
    parts = np.abs(s.m.astype(np.float64)) * b1 + np.abs(g.astype(np.float64)) * (1 - b1)
    most = lr * (decay * np.abs(p) + parts / (1 - b1 ** t) / root)
    if s.bits == 8:
        a = chances(len(p), t, tensor, seed)
        cm, held = hold(m, 127, a[0])
        s.cm, s.m = (np.sign(m) * cm).astype(np.int8), np.copysign(held, m).astype(f32)
        s.cu, u = hold(np.sqrt(v), 255, a[1])
        s.cu, s.v = s.cu.astype(np.uint8), u * u
    else:
        s.m, s.v = m, v
    return new, most
