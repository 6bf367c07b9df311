"""Oracle of the paged cache in 8 bits and of rotary positions, in plain Python and float64.

TEST INFRASTRUCTURE, like the rest of ``oracle/``: only the test suite may use it, and it
shares no code with the GPU library.
"""
from __future__ import annotations

import math

import torch

#: (largest code, exponent of the largest magnitude's unit, ...) by code and 16-bit type
TOP = {"e4m3": 448.0, "int8": 127.0}
MOST = {("e4m3", "fp16"): 240 * 2.0 ** 8, ("int8", "fp16"): 127 * 2.0 ** 9, ("e4m3", "bf16"): 240 * 2.0 ** 120, ("int8", "bf16"): 127 * 2.0 ** 121}
LEAST = {("e4m3", "fp16"): -15, ("int8", "fp16"): -24, ("e4m3", "bf16"): -110, ("int8", "bf16"): -110}


def held(x, code: str, kind: str):
    """x (float64) as far as it can be held."""
    return x.clamp(-MOST[code, kind], MOST[code, kind])


def exponent(x, code: str, kind: str) -> int:
    """The least exponent that takes the magnitudes of x (NaN aside) to codes."""
    top = float(torch.nan_to_num(held(x, code, kind), 0.0).abs().max()) if x.numel() else 0.0
    if top == 0:
        return LEAST[code, kind]
    part, e = math.frexp(top / TOP[code])       # (rounded, but never to a power of two that it is not)
    return max(e - (part == 0.5), LEAST[code, kind])


def rounded(x, e: int, code: str):
    """x (float64, within the codes' range at exponent e) as the nearest code * 2^e, ties to even; NaN stays in
    e4m3 and becomes 0 in int8."""
    y = x * 2.0 ** -e
    if code == "int8":
        return torch.nan_to_num(torch.round(y), 0.0) * 2.0 ** e
    # 3 bits behind the leading one, none below 2^-9
    e3 = torch.frexp(torch.nan_to_num(y).abs().clamp(min=2.0 ** -6)).exponent - 4
    unit = torch.tensor([2.0 ** i for i in range(-9, 64)], dtype=torch.float64)[e3.long() + 9]
    return torch.round(y / unit) * unit * 2.0 ** e


class Stored:
    """One request's keys (or values) [H][tokens][d] in blocks of `block` tokens."""

    def __init__(self, H: int, d: int, code: str, kind: str, block: int):
        self.code, self.kind, self.block = code, kind, block
        self.values = torch.zeros(H, 0, d, dtype=torch.float64)
        self.exponents = [[] for _ in range(H)]

    def step(self, x, keep: int | None = None):
        """Keeps the first `keep` tokens (all) and adds x [H][n][d]."""
        T = self.block
        first = self.values.shape[1] if keep is None else min(keep, self.values.shape[1])
        values = torch.cat([self.values[:, :first], x.double()], 1)
        L = values.shape[1]
        if x.shape[1] == 0:
            self.values = values
            return
        for h, exponents in enumerate(self.exponents):
            for j in range(first // T * T, L, T):
                older = max(0, first - j)
                e = exponent(values[h, j + older:j + T], self.code, self.kind)
                if older:
                    e = max(e, exponents[j // T])
                del exponents[j // T:]
                exponents.append(e)
                block = values[h, j:j + T].clone()
                block[older:] = held(block[older:], self.code, self.kind)
                values[h, j:j + T] = rounded(block, e, self.code)
        self.values = values


def to_fp16(x):
    """float64 to fp16, magnitudes over 65504 to 65504."""
    return x.clamp(-65504, 65504).to(torch.float16)


def rates(rot: int, base: float, scaling: str = "plain", factor: float = 1.0, original_len: float = 0.0, low: float = 1.0,
          high: float = 32.0):
    """Radians per position of every pair, from the formulas."""
    out = []
    for i in range(rot // 2):
        if scaling == "base":
            r = (base * factor ** (rot / (rot - 2))) ** (-2 * i / rot)
        else:
            r = base ** (-2 * i / rot)
        if scaling == "linear":
            r /= factor
        if scaling == "turns":
            g = min(max((original_len * r / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            r = g * r + (1 - g) * r / factor
        out.append(r)
    return out


def rotate(x, positions, rates, rot: int, layout: str, magnitude: float = 1.0, inverse: bool = False):
    """x [n][heads][d] turned by positions [n], float64, and what an element's rounding errors are multiplied by
    (|x_a| + |x_b| of its pair, times the magnitude; 0 where it is copied)."""
    x = x.double()
    y, mag = x.clone(), torch.zeros_like(x)
    for i, r in enumerate(rates):
        a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        # (the angle as a whole number of turns and the rest, so that its size costs nothing)
        angle = torch.tensor([math.fmod(int(p) * r, 2 * math.pi) for p in positions.tolist()], dtype=torch.float64, device=x.device)
        c, s = torch.cos(angle)[:, None] * magnitude, torch.sin(angle)[:, None] * magnitude * (-1 if inverse else 1)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        mag[..., a] = mag[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(magnitude)
    return y, mag
