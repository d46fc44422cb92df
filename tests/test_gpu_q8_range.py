"""Attention over the 8-bit cache at the ends of the range of its scales, in both kernels."""
import numpy as np
import pytest
import torch

from oracle import specext_oracle as orc
from paper_2505_20776_b200 import api
from tests.guards import GuardedHotPath
from tests.q8_util import GuardedCache8, garbage, values
from tests.test_gpu_verify_q8 import _check, _tensors
from tests.util import f64, random_forest

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


@pytest.mark.parametrize("Hq,Hkv,D,T,scored", CALLS)
@pytest.mark.parametrize("what,up", [("query", 6), ("query", 10), ("query", 13), ("nodes", 5), ("nodes", 8), ("nodes", 10)])
def test_one_value_far_above_the_others(cuda_device, Hq, Hkv, D, T, scored, what, up):
    """Query rows with one element, or the tree with one node's keys and another's values, 2^up above the rest.

    The kernel for many rows takes the largest of a row, or of 32 nodes' keys, to [2^7, 2^8) and holds each value as two e4m3 numbers:
    exactly, or to the half of their smallest step, 2^-10, that is to 2^-17 of that largest.  So beside the bounds of the other tests a
    logit is off by 2^-17 of the row's largest times sum |k|, and for tree keys of the 32 nodes' largest times sum |q| as well.
    (The kernel for few rows holds them to 2^-39 and gets the same room.)"""
    dev, L = cuda_device, 389
    g = torch.Generator().manual_seed(up)
    K, V = (torch.randn((L, Hkv, D), generator=g) for _ in range(2))
    t = _tensors(Hq, Hkv, D, T, dev, up)
    if what == "query":
        K[:, :, 5] *= 2.0 ** -up                                     # (as keys are where queries have a large channel)
        t["K_tree"][:, :, 5] *= 2.0 ** -up
        t["Q"][:, ::2, 5] *= 2.0 ** up
    else:
        t["K_tree"][T // 2] *= 2.0 ** up
        t["V_tree"][T - 1] *= 2.0 ** up
    c = _cache(dev, Hkv, D, K, V)
    parent = random_forest(np.random.default_rng(up), T)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    hp.verify_attn_q8(t, c, torch.from_numpy(parent).to(dev), scored)
    assert hp.read_status() == 0
    hp.check()
    K, V = values(c)
    q, kt, vt = f64(t["Q"]), f64(t["K_tree"]), f64(t["V_tree"])
    O, lse, score = orc.verify_attn(q, K, V, kt, vt, parent, 32)
    mag, _, _ = orc.verify_attn(q, K, np.abs(V), kt, np.abs(vt), parent, 32)
    G, s = Hq // Hkv, D ** -0.5
    off = np.zeros((T, Hq))
    for h in range(Hq):
        a, head = np.abs(q[:, h]), h // G
        for j0 in range(0, T, 32):                                    # groups of nodes
            group = np.abs(kt[j0:j0 + 32, head])
            off[:, h] = np.maximum(off[:, h], a.max(1) * group.sum(1).max() + group.max() * a.sum(1))
        off[:, h] = np.maximum(off[:, h], a.max(1) * np.abs(K[:, head]).sum(1).max())
    seen = np.concatenate([np.abs(K), np.abs(kt)])
    reach = np.stack([(np.abs(q[:, h]) @ seen[:, h // G].T).max(1) for h in range(Hq)], axis=1) * s
    logit = (D + 2) * 2.0 ** -24 * reach + 2.0 ** -19 + 1.01 * 2.0 ** -17 * s * off
    lost = seen.shape[0] * 2.0 ** -30 * max(np.max(np.abs(V)), np.max(np.abs(vt)))
    bound = 2.0 ** -8 * np.abs(O) + (2.0 ** -11 + np.expm1(2 * logit))[:, :, None] * 1.01 * mag + lost
    err = np.abs(f64(hp.O) - O)
    assert np.all(err <= bound), f"O off by {np.max(err - bound):.3e} over its bound"
    assert np.all(np.abs(f64(hp.lse) - lse) <= logit.T + 2.0 ** -23 * np.max(np.abs(lse)))
    if scored:
        # a chunk's score is the mean over the heads, each off by its own relative error
        np.testing.assert_allclose(f64(hp.chunk_score(L)), score, rtol=float(np.expm1(2 * logit.max())) + 2.0 ** -18, atol=1e-30)


@pytest.mark.parametrize("Hq,Hkv,D,T,scored", [(4, 2, 64, 2, False), (4, 2, 64, 40, True), (8, 2, 128, 60, True)])
def test_offsets_past_32_bits(cuda_device, Hq, Hkv, D, T, scored):
    """Tokens a MB apart: those from 4096 on lie 2^32 bytes and more behind the first one, and one of them has most of every row."""
    dev, L, row = cuda_device, 4133, 1 << 20
    g = torch.Generator().manual_seed(T)
    K, V = (torch.randn((L, Hkv, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2))
    t = _tensors(Hq, Hkv, D, T, dev, T)
    t["Q"] = (t["Q"].float() * 0.25 + 1).to(torch.bfloat16)
    K[[4097, 4131]] = 2.0
    room = torch.zeros((2, L * row), dtype=torch.uint8, device=dev)
    codes = [room[i].view(torch.float8_e4m3fn).as_strided((L, Hkv, D), (row, row // 2, 1)) for i in range(2)]
    scales = [torch.zeros((-(-L // 32), Hkv), dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu) for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    for lo, hi in ((0, 4000), (4000, 4100), (4100, L)):               # (the later ones begin inside blocks)
        api.specext_quantize_kv(K[lo:hi], V[lo:hi], lo, *codes, *scales, 32, status)
    c = GuardedCache8(Hkv, D, L, 32, dev)
    for lo, hi in ((0, 4000), (4000, 4100), (4100, L)):
        c.append(K[lo:hi], V[lo:hi])
    for far, near in zip(codes, (c.K, c.V)):
        assert torch.equal(far.view(torch.uint8), near.view(torch.uint8))
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    parent = random_forest(np.random.default_rng(T), T)
    ref_O, _, _ = _check(hp, t, c, parent, scored)
    near = f64(V[[4097, 4131]].cpu())
    assert np.abs(ref_O - np.repeat(near.mean(0), Hq // Hkv, axis=0)).max() < 0.5       # (those two tokens are what counts)
    O, lse = torch.empty_like(hp.O), torch.empty_like(hp.lse)
    score = torch.empty((T, -(-L // 32)), dtype=torch.float32, device=dev) if scored else None
    d = api.make_attn_desc(t["Q"], codes[0], t["K_tree"], O, L, 32, 0.0, scored)
    ws = torch.empty(api.specext_verify_attn_q8_workspace(d, 32), dtype=torch.uint8, device=dev)
    api.specext_verify_attn_q8(d, t["Q"], *codes, *scales, 32, t["K_tree"], t["V_tree"], torch.from_numpy(parent).to(dev), O, lse,
                               score, ws, status)
    assert torch.equal(O, hp.O) and torch.equal(lse, hp.lse) and int(status) == 0
    assert not scored or torch.equal(score, hp.chunk_score(L))
