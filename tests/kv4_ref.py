"""Plain forms of the 4-bit cache's rows in 64 bits, written from their definitions (include/pasta_kv4.h).  Its attention is kv8_ref.attend over the values."""
from __future__ import annotations

import math

import numpy as np

from kv8_ref import attend  # noqa: F401

BLOCK, GROUP, NONE = 16, 32, 255
E_MIN, E_MAX = -100, 119
LEVEL = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])  # by code


def scale_byte(amax):
    if not math.isfinite(amax):
        return NONE
    e = E_MIN
    while e < E_MAX and amax > 7.0 * 2.0 ** e:
        e += 1
    return e + 127


def code(x):
    """nearest code to x in units of the scale (float64), ties to the even code"""
    a = np.abs(x)
    c = np.zeros(a.shape, np.uint8)
    for k in range(7):
        mid = (LEVEL[k] + LEVEL[k + 1]) / 2
        c += (a > mid) | ((a == mid) & (k % 2 == 1))
    return c | (np.signbit(x).astype(np.uint8) << 3)


def code_group(x):
    """(codes, scale's byte) of the values under one scale"""
    b = scale_byte(float(np.abs(x).max()) if np.isfinite(x).all() else math.inf)
    return (np.zeros(x.shape, np.uint8), b) if b == NONE else (code(x * 2.0 ** (127 - b)), b)


def values(codes, byte):
    return np.full(codes.shape, math.nan) if byte == NONE else LEVEL[codes] * 2.0 ** (int(byte) - 127)


class Cache:
    """Codes and scales of one layer: kc, vc [pages, H, P, D] a code to an element, ks [pages, H, P, D / 32], vs [pages, H, P]."""

    def __init__(self, pages, H, P, D, kc, vc, ks, vs):
        self.pages, self.H, self.P, self.D, self.kc, self.vc, self.ks, self.vs = pages, H, P, D, kc, vc, ks, vs

    @classmethod
    def unpack(cls, pages, H, P, D, k_codes, v_codes, k_scale, v_scale):
        """From the bytes as they lie in memory (of one layer)."""
        B = P // BLOCK
        k = np.asarray(k_codes).reshape(pages, H, B, D // 32, BLOCK, 16)
        k = np.stack([k & 15, k >> 4], -1).reshape(pages, H, B, D // 32, BLOCK, 32).transpose(0, 1, 2, 4, 3, 5).reshape(pages, H, P, D)
        v = np.asarray(v_codes).reshape(pages, H, B, D, 8)
        v = np.stack([v & 15, v >> 4], -1).reshape(pages, H, B, D, BLOCK).transpose(0, 1, 2, 4, 3).reshape(pages, H, P, D)
        return cls(pages, H, P, D, k.copy(), v.copy(), np.asarray(k_scale).reshape(pages, H, P, D // 32).copy(), np.asarray(v_scale).reshape(pages, H, P).copy())

    def pack(self):
        B, D = self.P // BLOCK, self.D
        k = self.kc.reshape(self.pages, self.H, B, BLOCK, D // 32, 16, 2).transpose(0, 1, 2, 4, 3, 5, 6)
        v = self.vc.reshape(self.pages, self.H, B, BLOCK, D).transpose(0, 1, 2, 4, 3).reshape(self.pages, self.H, B, D, 8, 2)
        return k[..., 0] | k[..., 1] << 4, v[..., 0] | v[..., 1] << 4, self.ks, self.vs

    def append(self, slot, k, v):
        for i, s in enumerate(slot):
            if not 0 <= s < self.pages * self.P:
                continue
            p, t = s // self.P, s % self.P
            for h in range(self.H):
                for g in range(self.D // GROUP):
                    d = slice(g * GROUP, g * GROUP + GROUP)
                    self.kc[p, h, t, d], self.ks[p, h, t, g] = code_group(k[i, h, d])
                self.vc[p, h, t], self.vs[p, h, t] = code_group(v[i, h])

    def natural(self):
        """K, V [slots, H, D] float64"""
        with np.errstate(invalid="ignore"):
            ks, vs = (np.where(s == NONE, math.nan, 2.0 ** (s.astype(np.float64) - 127)) for s in (self.ks, self.vs))
            k, v = LEVEL[self.kc] * np.repeat(ks, GROUP, -1), LEVEL[self.vc] * vs[..., None]
        flat = lambda x: x.transpose(0, 2, 1, 3).reshape(self.pages * self.P, self.H, self.D)  # noqa: E731
        return flat(k), flat(v)
