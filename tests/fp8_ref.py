"""Operators on 8-bit rows in 64 bits, from their definitions (include/gacer.h), on the CPU."""
import math

import numpy as np
import torch

BLOCK = 128
# every magnitude of e4m3 by its code: subnormal steps of 2^-9, then eight a power of two up to 448 (code 127 is NaN)
GRID = np.array([c / 512.0 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])


def nearest(q):
    """Codes' values nearest to q (float64), ties to the even code, beyond the largest the largest."""
    a = np.abs(q)
    hi = np.clip(np.searchsorted(GRID, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    down, up = a - GRID[lo], GRID[hi] - a
    pick = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return np.copysign(GRID[pick], q)


def blocks(n):
    return -(-n // BLOCK)


def weight(gen, out, cin, spread=1.0):
    """Random codes (subnormal, largest and zero ones among them) and scales: (float8 codes, scales, float64 values)."""
    w = torch.randn(out, cin, generator=gen) * spread
    w[torch.rand(out, cin, generator=gen) < 0.02] = 0.0
    codes = torch.from_numpy(nearest((w * 100).double().numpy())).to(torch.float8_e4m3fn)
    scales = (0.5 + torch.rand(blocks(out), blocks(cin), generator=gen)) * cin ** -0.5 / 100
    return codes, scales, codes.double() * scales.double().repeat_interleave(BLOCK, 0)[:out].repeat_interleave(BLOCK, 1)[:, :cin]


def rows(gen, n, features):
    """(float8 codes [n, features], scales [blocks, n], float64 values)"""
    x = torch.randn(n, features, generator=gen) * (1 + 5 * (torch.rand(features, generator=gen) < 0.03))
    codes = torch.from_numpy(nearest((x * 60).double().numpy())).to(torch.float8_e4m3fn)
    scales = (0.2 + torch.rand(blocks(features), n, generator=gen)) / 60
    return codes, scales, codes.double() * scales.double().t().repeat_interleave(BLOCK, 1)[:, :features]


def act(x, name):
    if name == "relu":
        return x.clamp_min(0)
    if name == "relu6":
        return x.clamp(0, 6)
    if name == "gelu":
        return x * torch.special.ndtr(x)
    if name == "hard_sigmoid":
        return (x + 3).clamp(0, 6) / 6
    if name == "hard_swish":
        return x * (x + 3).clamp(0, 6) / 6
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu_tanh":
        return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    assert name == "none"
    return x


def product(x, w):
    """(sum_k x w, its error bound): products are exact, each of the additions (within a block of 128, of blocks, of slices and waves) loses at most a unit
    in the last place (2^-23) of a partial sum, which the sum of magnitudes bounds."""
    n = BLOCK + blocks(x.shape[1]) + 32
    return x @ w.t(), n * 2.0 ** -23 * (x.abs() @ w.abs().t())


def check_rows(codes, scales, y, err):
    """8-bit rows against y (float64 [n, features], every element uncertain by err): scales, then every code between those of the ends of its interval."""
    n, features = y.shape
    for b in range(blocks(features)):
        part, e = y[:, b * BLOCK:(b + 1) * BLOCK].numpy(), err[:, b * BLOCK:(b + 1) * BLOCK].numpy()
        got, s = codes[:, b * BLOCK:(b + 1) * BLOCK].double().numpy(), scales[b].double().numpy()
        bad = ~np.isfinite(part).all(1)
        assert np.isnan(s[bad]).all() and (got[bad] == 0).all()
        assert np.isfinite(s[~bad]).all()
        part, e, got, s = part[~bad], e[~bad], got[~bad], s[~bad]
        if not len(s):
            continue
        want = np.maximum(np.abs(part).max(1), 2.0 ** -60) / 448
        assert (np.abs(s - want) <= e.max(1) / 448 + 2.0 ** -23 * want).all(), b
        # the factor 448 / m and the product with it: two roundings
        q, d = part / s[:, None], e / s[:, None] + 2.0 ** -22 * np.abs(part / s[:, None])
        assert (got >= nearest(q - d)).all() and (got <= nearest(q + d)).all(), b
