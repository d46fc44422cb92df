"""specext_token_logprobs on rows that one word dominates: what is left to the others, 1e-2 to nothing, decides the entropy and the best
word's log probability, which are held relative to themselves, and their signs to what they can be.

Bounds.  With x_b the best logit, t = (x - x_b) log2(e) / T and r the sum of 2^t over the other words, the results are sums of terms of
one sign: -log p_b = log1p(r), entropy = log1p(r) + sum |t| 2^t ln 2 / (1 + r), -log p_w = |t_w| ln 2 + log1p(r).  A term's t is off by
5 roundings (the factor's, two of the product and the difference, two of the shifts between partial sums, whose lengths add up to at
most |t| + 8): 3.5 (|t| + 8) 2^-24 of the term.  ex2 is off by 2^-22 here and in up to three shifts, and a sum by 60 additions;
where r is 1/2 and more these two count three times, since r may then be the sum of all words less the best one's 1, and for the entropy's
sum, of terms t 2^t with t as large as 4 that cancel by a sixteenth, 8 times.  With the words' |t| weighed as the sums weigh them:
(256 + 3.5 mean |t|) 2^-24 for r, (608 + 3.5 mean |t|) 2^-24 for the entropy, 4 roundings of the result's own, and 2^-126 a word of what
underflows.
"""
import numpy as np
import pytest
import torch

from tests.guards import GuardedHotPath
from tests.util import f64

pytestmark = pytest.mark.gpu


def _check(logits, temperature, k=3):
    """`logits`: rows whose best word is one alone; returns the largest relative errors of the best log probability and the entropy."""
    dev, (R, V) = logits.device, logits.shape
    T = float(np.float32(temperature))
    x = f64(logits)
    best = x.argmax(axis=1)
    tokens = np.stack([best, (best + 1) % V, np.full(R, V // 2)], axis=1)
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=dev)
    lp, ent, lse, ids, top = hp.token_logprobs(logits, torch.as_tensor(tokens, dtype=torch.int32, device=dev), min(k, V), T)
    assert hp.read_status() == 0
    hp.check()
    lp, ent, lse, ids, top = f64(lp), f64(ent), f64(lse), ids.cpu().numpy(), f64(top)
    assert (lp <= 0).all() and (top <= 0).all() and (ent >= 0).all()
    u = 2.0 ** -24
    worst = [0.0, 0.0]
    for row in range(R):
        m = x[row, best[row]]
        t = (x[row] - m) / T                                          # nats
        t[best[row]] = -np.inf
        some = t[np.isfinite(t)]
        w = np.exp(some)
        r, a, b = w.sum(), -(w * some).sum(), (w * some * some).sum()
        size = lambda p, q: p / q / np.log(2) if q > 0 else 0.0
        log_z, under = np.log1p(r), V * 2.0 ** -126
        tol, tol_e = (256 + 3.5 * size(a, r)) * u, (608 + 3.5 * size(b, a)) * u
        t[best[row]] = 0.0
        for got, ref in [(lp[row], t[tokens[row]] - log_z), (top[row], t[ids[row]] - log_z)]:
            np.testing.assert_allclose(got, ref, rtol=tol + 4 * u, atol=under)
        entropy = log_z + a / (1 + r)
        np.testing.assert_allclose(ent[row], entropy, rtol=tol_e + 4 * u, atol=200 * under)
        np.testing.assert_allclose(lse[row], m / T + log_z, rtol=1e-6, atol=2e-6)
        assert ids[row, 0] == best[row]
        if r > 1e-30:
            worst = [max(worst[0], abs(lp[row, 0] / -log_z - 1)), max(worst[1], abs(ent[row] / entropy - 1))]
    return worst


def _rows(R, V, dtype, dev, seed, stride=None, offset=0):
    """As a model's: a few words of every row stand out."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((R, V), generator=g) * 2
    n = min(40, V)
    x.scatter_add_(1, torch.randint(0, V, (R, n), generator=g), 6 * torch.rand((R, n), generator=g) + 4)
    x = x.to(dtype)
    x[torch.arange(R), x.argmax(1)] *= 1.0625                         # (one best word, ties apart)
    stride = stride or V
    room = torch.full((offset + R * stride + 16,), float("nan"), dtype=dtype, device=dev)
    view = room[offset:offset + R * stride].view(R, stride)[:, :V]
    view.copy_(x)
    return view


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("temperature", [0.5, 0.3, 0.1, 0.05])
@pytest.mark.parametrize("R,V", [(40, 33), (60, 1500), (33, 5003), (40, 32000), (16, 128256), (640, 9001)])
def test_what_is_left_to_the_others(cuda_device, dtype, temperature, R, V):
    print(_check(_rows(R, V, dtype, cuda_device, V, V + 1, V % 5), temperature))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [2, 300, 20011, 128256])
def test_the_best_word_in_any_place(cuda_device, dtype, V):
    """First, last, anywhere; with company of its size nearby, far away, everywhere, or none (all other words masked: certain)."""
    dev = cuda_device
    places = sorted({p for p in (0, 1, 7, 8, 255, 2047, 2048, V // 3, V - 9, V - 1) if 0 <= p < V})
    rows = []
    for p in places:
        for kind in range(4):
            x = torch.full((V,), -20.0) - torch.arange(V) % 5
            if kind == 0:
                x[(p + 3) % V] = -8
            if kind == 1:
                x[(p + V // 2) % V] = -12.5
            if kind == 2:
                x = torch.full((V,), float("-inf"))
            if kind == 3:
                x = torch.full((V,), torch.finfo(dtype).min)
                x[(p + 2048) % V] = -18
            x[p] = 3.0
            rows.append(x)
    _check(torch.stack(rows).to(dtype).to(dev), 1.0)


def test_logits_far_from_zero(cuda_device):
    """Around 2^20 and -2^20 times the temperature, on both sides of where the sums change their form."""
    dev, V = cuda_device, 30000
    g = torch.Generator().manual_seed(5)
    wide = torch.rand((4, V), generator=g, dtype=torch.float64) * 4
    wide[:, 12345] += 12
    wide[1, 29999] += 17
    for at in (2.0 ** 20 * np.log(2), 3e5, 1e6):
        _check(torch.stack([wide[0] - at, wide[1] + at, wide[2] - at - 9, wide[3] + at + 9]).float().to(dev), 1.0)


def test_rows_that_more_than_one_word_rules(cuda_device):
    """Around the change of form at r = 1/2: a second word of every weight down from the best one's."""
    dev, V = cuda_device, 4000
    x = torch.full((48, V), -30.0)
    x[:, 17] = 10.0
    x[torch.arange(48), 300 + 70 * torch.arange(48)] = 10.0 - 0.0625 * torch.arange(1, 49)
    _check(x.to(dev), 1.0)
    _check(x.to(torch.bfloat16).to(dev), 1.0, 2)


def test_temperatures_at_the_ends(cuda_device):
    """As cold as a float allows (the best word is certain) and as hot (all words that are not masked are alike)."""
    dev, V = cuda_device, 9001
    x = _rows(4, V, torch.float32, dev, 9)
    x[3, ::2] = float("-inf")
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=dev)
    best = x.argmax(1, keepdim=True).to(torch.int32)
    for T in (4.3e-39, 1e-38, 1e-30, 1e-10):
        lp, ent, lse, ids, top = hp.token_logprobs(x, best, 2, T)
        assert hp.read_status() == 0
        assert (lp == 0).all() and (ent == 0).all() and (ids[:, :1] == best).all() and (top[:, 0] == 0).all() and (top[:, 1] < 0).all()
        assert not lse.isnan().any()
    n = torch.tensor([V, V, V, V // 2], dtype=torch.float64)
    for T in (1e20, 1e30, 3e38):
        lp, ent, lse, ids, top = hp.token_logprobs(x, best, 2, T)
        assert hp.read_status() == 0
        for got in (ent, lse, -lp[:, 0], -top[:, 1]):
            np.testing.assert_allclose(f64(got), n.log().numpy(), rtol=1e-6)
    hp.check()
