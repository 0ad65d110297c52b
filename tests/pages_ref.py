"""The operators around the paged K/V store of eight bits, from their definitions, in float64 on the CPU.  A store is a list of
values: code numbers and scale exponents, page by page."""
from __future__ import annotations

import math

import numpy as np
import torch

from helpers import e4m3_round

E4M3, INT8 = 0, 1
LARGEST = {E4M3: 448.0, INT8: 127.0}
HIGHEST = {E4M3: 119, INT8: 121}
LOWEST = -110
TORCH = {E4M3: torch.float8_e4m3fn, INT8: torch.int8}


def nearest_code(x: np.ndarray, fmt: int) -> np.ndarray:
    x = np.asarray(x, np.float64)
    if fmt == INT8:
        return np.where(np.isnan(x), 0.0, np.clip(np.rint(np.where(np.isnan(x), 0.0, x)), -127, 127))
    with np.errstate(invalid="ignore"):
        big = np.clip(np.where(np.isnan(x), 0.0, x), -1e30, 1e30)
    return np.where(np.isnan(x), np.nan, e4m3_round(big))


def exponent_for(x: np.ndarray, fmt: int) -> int:
    """The smallest e in range with max|finite x| <= largest code * 2^e."""
    a = np.abs(np.asarray(x, np.float64))
    a = a[np.isfinite(a)]
    top = float(a.max()) if a.size else 0.0
    if top == 0.0:
        return LOWEST
    e = math.frexp(top)[1] - math.frexp(LARGEST[fmt])[1] - 1
    while top > math.ldexp(LARGEST[fmt], e):
        e += 1
    return min(max(e, LOWEST), HIGHEST[fmt])


class Store:
    """codes [pages, heads, 2, T, d] as numbers, exponents [pages, heads, 2]."""

    def __init__(self, n_pages, heads, T, d, fmt):
        self.fmt, self.T = fmt, T
        self.codes = np.zeros((n_pages, heads, 2, T, d))
        self.exps = np.zeros((n_pages, heads, 2), np.int64)

    def write(self, table, lengths, rows, k, v):
        """k, v: per sequence [rows, heads, d] float64."""
        for s, n in enumerate(lengths):
            for first in range(n // self.T * self.T, n + rows[s], self.T):
                page = table[s][first // self.T]
                t0, t1 = max(first, n) - first, min(first + self.T, n + rows[s]) - first
                for w, x in ((0, k[s]), (1, v[s])):
                    new = x[first + t0 - n:first + t1 - n]
                    for h in range(x.shape[1]):
                        e = exponent_for(new[:, h], self.fmt)
                        block = self.codes[page, h, w]
                        if t0:
                            old = int(self.exps[page, h, w])
                            e = max(e, old)
                            block[:t0] = nearest_code(np.ldexp(block[:t0], old - e), self.fmt)
                        block[t0:t1] = nearest_code(np.ldexp(new[:, h], -e), self.fmt)
                        self.exps[page, h, w] = e

    def values(self, table_row, n):
        """[2][n, heads, d]: what the first n tokens of a sequence stand for."""
        pages = list(table_row[:(n + self.T - 1) // self.T])
        x = np.ldexp(self.codes[pages], self.exps[pages][..., None, None])
        x = np.moveaxis(x, 2, 0)                                        # [2][pages][heads][T][d]
        return x.transpose(0, 1, 3, 2, 4).reshape(2, -1, x.shape[2], x.shape[4])[:, :n]

    def to(self, device, page_slack=0):
        """(codes, scales) as tensors; page_slack: unused bytes between the pages."""
        n, rest = self.codes.shape[0], self.codes.shape[1:]
        size = int(np.prod(rest))
        codes = torch.tensor(self.codes).to(TORCH[self.fmt])
        if self.fmt == E4M3:
            codes = codes.view(torch.uint8).view(n, size)
        else:
            codes = codes.view(torch.uint8).view(n, size)
        wide = torch.full((n, size + page_slack), 0x7f, dtype=torch.uint8)
        wide[:, :size] = codes
        wide = wide.to(device)[:, :size].view(TORCH[self.fmt])
        strides = [int(np.prod(rest[i + 1:])) for i in range(len(rest))]
        codes = wide.as_strided((n, *rest), (size + page_slack, *strides))
        return codes, torch.tensor(np.ldexp(1.0, self.exps), dtype=torch.float32).to(device)


def attention(q, K, V, end, scale, T):
    """One sequence: q [rows, Hq, d], K, V [n, H, d] from pages of T tokens, end [rows] tokens seen; float64.  Returns out, lse and
    what an output's error is made of: sum p |v| (and what fp16 weights lose below 2^-14: half a step of 2^-24 of the largest p 2^e
    each, times a largest code, in a block whose largest value is above half of that), and sum |q k| of the worst seen key."""
    rows, Hq, d = q.shape
    block = np.array([np.nanmax(np.abs(V[t // T * T:t // T * T + T]), axis=(0, 2), initial=0.0) for t in range(0, V.shape[0])]).reshape(-1, K.shape[1])
    H = K.shape[1]
    out, lse = np.zeros((rows, Hq, d)), np.full((rows, Hq), -np.inf)
    spread, reach = np.zeros((rows, Hq, d)), np.zeros((rows, Hq))
    for i in range(rows):
        n = max(0, min(int(end[i]), K.shape[0]))
        if n == 0:
            continue
        for h in range(Hq):
            kh, vh = K[:n, h // (Hq // H)], V[:n, h // (Hq // H)]
            s = kh @ q[i, h] * scale
            if np.isnan(s).any():
                out[i, h], lse[i, h] = np.nan, np.nan
                continue
            p = np.exp(s - s.max())
            lse[i, h] = s.max() + np.log(p.sum())
            p /= p.sum()
            out[i, h] = p @ vh
            spread[i, h] = p @ np.abs(vh) + n * 2.0 ** -25 / 2.0 ** -11 * 2 * (p * block[:n, h // (Hq // H)]).max()
            reach[i, h] = (np.abs(kh) @ np.abs(q[i, h])).max() * scale
    return out, lse, spread, reach


def attention_bounds(out, lse, spread, reach, dtype, d):
    """How far the kernel's outputs may be off.  Scores: d products summed in fp32, each sum off by 2^-24 of the partial sums, and as
    many roundings again for the scales: (d + 8) 2^-24 of sum |q k|.  Weights: that, exp2's own 2^-21, and a half step of fp16 (2^-11,
    absolute 2^-25 of the top weight for subnormal ones: in `spread`), in the product and the denominator.  The output: half a step."""
    ds = (d + 8) * 2.0 ** -24 * reach
    dp = 2.0 ** -11 + 2 * (np.expm1(ds) + 2.0 ** -20)
    step = torch.finfo(dtype).eps / 2
    tiny = float(torch.finfo(dtype).smallest_normal) * step
    return step * np.abs(out) * (1 + 2.0 ** -8) + dp[..., None] * spread * (1 + step) + tiny, ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))
