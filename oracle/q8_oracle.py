"""fp64 oracle of the 8-bit cache and of the token log probabilities, from the definitions (numpy; shares no code with the
library).  e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits, no infinities, S.1111.111 is NaN.  e8m0: 2^(code - 127), 255
is NaN."""
from __future__ import annotations

import numpy as np


def e4m3_values() -> np.ndarray:
    """The 256 values of e4m3 by code."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = np.ldexp(m / 8.0, -6) if e == 0 else np.ldexp(1 + m / 8.0, e - 7)
        out[c] = np.nan if e == 15 and m == 7 else (-v if c & 128 else v)
    return out


def e4m3_round(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value of x, |x| <= 448; ties to the even mantissa."""
    grid = e4m3_values()[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(grid[pick], x)


def scale_exponent(x: np.ndarray) -> int:
    """Exponent of the smallest power of two s >= 2^-100 with |x| <= 448 s."""
    m, e = np.max(np.abs(x)), -100
    while m > 448 * 2.0 ** e:
        e += 1
    return e


def append(values: np.ndarray, exps: np.ndarray, x: np.ndarray, start: int, block: int) -> None:
    """Appends x [n][H][D] (fp64) in place at `start` of a cache given as codes' values [capacity][H][D] and scale exponents
    [blocks][H]; NaN exponents are blocks that received something non-finite."""
    n = x.shape[0]
    for b in range(start // block, -(-(start + n) // block)):
        lo, hi = max(b * block, start), min((b + 1) * block, start + n)
        for h in range(x.shape[1]):
            new = x[lo - start:hi - start, h]
            old = exps[b, h] if lo > b * block else -100.0
            if not np.all(np.isfinite(new)) or np.isnan(old):
                exps[b, h] = np.nan
                continue
            e = max(scale_exponent(new), old)
            if lo > b * block and e > old:
                values[b * block:lo, h] = e4m3_round(values[b * block:lo, h] * 2.0 ** (old - e))
            values[lo:hi, h] = e4m3_round(new / 2.0 ** e)
            exps[b, h] = e


def cached(values: np.ndarray, exps: np.ndarray, length: int, block: int) -> np.ndarray:
    """What the first `length` tokens stand for."""
    return values[:length] * 2.0 ** exps[np.arange(length) // block][:, :, None]


def token_logprobs(logits: np.ndarray, tokens: np.ndarray, k: int, temperature: float):
    """(logprob, entropy, lse, top_ids, top_logprob) of rows of logits (fp64); token -1 is none."""
    R = logits.shape[0]
    lp, top = np.full(tokens.shape, -np.inf), np.full((R, k), -np.inf)
    entropy, lse, ids = np.zeros(R), np.full(R, -np.inf), np.full((R, k), -1, dtype=np.int64)
    for r in range(R):
        raw = logits[r]
        if np.isnan(raw).any() or (raw == np.inf).any():
            lp[r], top[r], entropy[r], lse[r] = np.nan, np.nan, np.nan, np.nan
            lp[r, tokens[r] == -1] = -np.inf
            continue
        ids[r] = np.lexsort((np.arange(raw.size), -raw))[:k]
        if np.all(raw == -np.inf):
            continue
        x = raw / temperature
        m = x.max()
        with np.errstate(under="ignore", over="ignore"):
            p = np.exp(x - m)
        lse[r] = m + np.log(p.sum())
        logp = (x - m) - np.log(p.sum())        # (and not x - lse, which loses log Z where |m| is huge)
        q = p / p.sum()
        seen = q > 0
        entropy[r] = -np.sum(q[seen] * logp[seen])
        given = tokens[r] >= 0
        lp[r, given] = logp[tokens[r, given]]
        top[r] = logp[ids[r]]
    return lp, entropy, lse, ids, top
