"""Helpers of the tests of the 8-bit cache: a guarded cache, its contents for the oracle, and the bounds of a comparison."""
import numpy as np
import torch

from oracle import q8_oracle
from oracle import specext_oracle as orc
from paper_2505_20776_b200.cache8 import KvCache8
from tests.guards import GuardedHotPath
from tests.util import f64


class GuardedCache8(KvCache8):
    """KvCache8 with guard bands around its buffers."""

    _alloc = GuardedHotPath._alloc
    check = GuardedHotPath.check


def garbage(cache, seed=0):
    """Every byte of codes and scales random: what lies behind the tokens must not matter."""
    g = torch.Generator().manual_seed(seed)
    for t in (cache.K, cache.V, cache.K_scale, cache.V_scale):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8))


def exponents(scale):
    """e8m0 as exponents (fp64, NaN for 255)."""
    c = scale.view(torch.uint8).cpu().numpy().astype(np.float64)
    return np.where(c == 255, np.nan, c - 127)


def values(cache, length=None):
    """K and V of the cached tokens as fp64, from the codes and scales as they stand."""
    n = cache.length if length is None else length
    table = q8_oracle.e4m3_values()
    return tuple(q8_oracle.cached(table[c[:n].view(torch.uint8).cpu().numpy()], exponents(s), n, cache.block_tokens)
                 for c, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)))


def check_attention(Q, K, V, Kt, Vt, parent, C, O, lse, score, scale=None):
    """O, lse and score (or None) of a call against the oracle on fp64 K, V [L][Hkv][D] (Q, Kt, Vt: bf16 tensors).

    Bounds.  A logit is a sum of D products of exact values in fp32: off by D + 2 roundings of 2^-24 of sum |q k|, the sum's own
    and the scalings'; ex2 and the row sums add 2^-19 relative.  Both sides of a probability's quotient have that.  A probability
    is rounded to f16 (2^-11 relative; 2^-30 of the row's largest may be lost per key), O once to bf16 (2^-8 relative).
    """
    q, kt, vt = f64(Q), f64(Kt), f64(Vt)
    D, G = q.shape[2], q.shape[1] // kt.shape[1]
    s = D ** -0.5 if not scale else scale
    ref_O, ref_lse, ref_score = orc.verify_attn(q, K, V, kt, vt, parent, C, scale)
    mag, _, _ = orc.verify_attn(q, K, np.abs(V), kt, np.abs(vt), parent, C, scale)       # sum p |v|
    keys = np.concatenate([np.abs(K), np.abs(kt)])
    reach = max(np.max(np.abs(q[:, h]) @ keys[:, h // G].T) for h in range(q.shape[1])) * s
    logit = (D + 2) * 2.0 ** -24 * reach + 2.0 ** -19
    lost = keys.shape[0] * 2.0 ** -30 * max(np.max(np.abs(V), initial=0.0), np.max(np.abs(vt)))
    bound = 2.0 ** -8 * np.abs(ref_O) + (2.0 ** -11 + 2 * logit) * 1.01 * mag + lost
    err = np.abs(f64(O) - ref_O)
    assert np.all(err <= bound), f"O off by {np.max(err - bound):.3e} over its bound, error {err.max():.3e}"
    np.testing.assert_allclose(f64(lse), ref_lse, rtol=0, atol=logit + 2.0 ** -23 * np.max(np.abs(ref_lse)))
    if score is not None:
        np.testing.assert_allclose(f64(score), ref_score, rtol=2 * logit + 2.0 ** -18, atol=1e-30)
    return ref_O, ref_lse, ref_score
