"""Attention over the 8-bit cache at the ends of the range of its scales, in both kernels."""
import numpy as np
import pytest
import torch

from tests.guards import GuardedHotPath
from tests.q8_util import GuardedCache8, garbage
from tests.test_gpu_verify_q8 import _check, _tensors
from tests.util import random_forest

pytestmark = pytest.mark.gpu

# (Hq, Hkv, D, T, scored): few rows; one CTA of 128 rows, head_dim 64 and 128; a pair of CTAs
CALLS = [(8, 4, 64, 1, False), (16, 2, 128, 10, False), (8, 4, 64, 30, True), (8, 4, 128, 17, True), (32, 8, 128, 60, True)]


def _cache(dev, Hkv, D, K, V):
    c = GuardedCache8(Hkv, D, K.shape[0] + 40, 32, dev)
    garbage(c)
    c.append(K.to(torch.bfloat16).to(dev), V.to(torch.bfloat16).to(dev))
    return c


@pytest.mark.parametrize("Hq,Hkv,D,T,scored", CALLS)
@pytest.mark.parametrize("L", [1, 300, 511, 700])
def test_masked_keys_of_a_block_of_zeros(cuda_device, Hq, Hkv, D, T, scored, L):
    """The prefix ends inside a tile, in a block of zeros (scale 2^-100), and query rows are so small that their factor times that
    scale is no longer a number above zero: what lies behind the prefix is left out all the same."""
    dev = cuda_device
    g = torch.Generator().manual_seed(L)
    K, V = (torch.randn((L, Hkv, D), generator=g) for _ in range(2))
    K[(L - 1) // 32 * 32:] = 0
    c = _cache(dev, Hkv, D, K, V)
    t = _tensors(Hq, Hkv, D, T, dev, L)
    for h in range(Hq):
        t["Q"][:, h] *= 2.0 ** -(20 * (h % 6))
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    _check(hp, t, c, random_forest(np.random.default_rng(L), T), scored)


@pytest.mark.parametrize("Hq,Hkv,D,T,scored", CALLS)
@pytest.mark.parametrize("down", [60, 70, 100])
def test_a_tree_of_tiny_queries_and_keys(cuda_device, Hq, Hkv, D, T, scored, down):
    dev, L = cuda_device, 256
    g = torch.Generator().manual_seed(down)
    c = _cache(dev, Hkv, D, *(torch.randn((L, Hkv, D), generator=g) for _ in range(2)))
    t = _tensors(Hq, Hkv, D, T, dev, down)
    t["Q"] *= 2.0 ** -down
    t["K_tree"] *= 2.0 ** -down
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    _check(hp, t, c, random_forest(np.random.default_rng(down), T), scored)


@pytest.mark.parametrize("Hq,Hkv,D,T,scored", [(8, 4, 128, 17, True), (32, 8, 128, 60, True), (32, 8, 128, 40, False), (64, 8, 128, 128, False)])
def test_every_row_has_a_size_of_its_own(cuda_device, Hq, Hkv, D, T, scored):
    """Query rows each at another power of two, in another order every time: a row's factor is the one its own warp found, in both
    CTAs of a pair, whatever the call before left in its place."""
    dev, L = cuda_device, 3000
    g = torch.Generator().manual_seed(T)
    c = _cache(dev, Hkv, D, *(torch.randn((L, Hkv, D), generator=g) for _ in range(2)))
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    parent = random_forest(np.random.default_rng(T), T)
    t = _tensors(Hq, Hkv, D, T, dev, T)
    plain = t["Q"]
    for turn in range(3):
        size = torch.exp2(torch.randint(-12, 3, (T, Hq, 1), generator=g).float()).to(dev)
        t["Q"] = (plain.float() * size).to(torch.bfloat16)
        _check(hp, t, c, parent, scored)
