"""specext_verify_attn_q8 against the fp64 oracle on the values that the cache stands for."""
import numpy as np
import pytest
import torch

from oracle import specext_oracle as orc
from paper_2505_20776_b200 import api
from tests.guards import GuardedHotPath
from tests.q8_util import GuardedCache8, check_attention, garbage, values
from tests.util import random_forest

pytestmark = pytest.mark.gpu


def _tensors(Hq, Hkv, D, T, dev, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: (torch.randn(s, generator=g) * size).to(torch.bfloat16).to(dev)
    return {"Q": r(T, Hq, D), "K_tree": r(T, Hkv, D), "V_tree": r(T, Hkv, D)}


def _filled(Hkv, D, L, block, dev, seed, spare=9, channel=0.5):
    """A cache of L tokens, random bytes behind them."""
    c = GuardedCache8(Hkv, D, L + spare, block, dev)
    garbage(c, seed)
    if L:
        g = torch.Generator().manual_seed(seed)
        ch = torch.exp(channel * torch.randn((1, Hkv, D), generator=g))
        r = lambda: (torch.randn((L, Hkv, D), generator=g) * ch).to(torch.bfloat16).to(dev)
        c.append(r(), r())
    return c


def _check(hp, t, c, parent, score, scale=None):
    par = torch.from_numpy(parent).to(hp.device)
    hp.verify_attn_q8(t, c, par, score)
    assert hp.read_status() == 0 and c.read_status() == 0
    hp.check()
    c.check()
    K, V = values(c)
    return check_attention(t["Q"], K, V, t["K_tree"], t["V_tree"], parent, hp.C, hp.O, hp.lse,
                           hp.chunk_score(c.length) if score and c.length else None, scale)


SHAPES = [(32, 8, 128), (8, 8, 128), (64, 8, 128), (16, 1, 128), (12, 12, 64), (8, 2, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("T", [1, 2, 3, 9, 33, 60, 128])
def test_rows_and_heads(cuda_device, Hq, Hkv, D, T):
    """From one stacked row to a tree of 128 nodes, on a ragged prefix of a few tiles."""
    rng = np.random.default_rng(T)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, 700, device=cuda_device)
    c = _filled(Hkv, D, 389, 32, cuda_device, T + Hq)
    for score in (False, True):
        _check(hp, _tensors(Hq, Hkv, D, T, cuda_device, T), c, random_forest(rng, T), score)


@pytest.mark.parametrize("L", [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 257, 1000, 2048, 4097])
@pytest.mark.parametrize("Hq,Hkv,D,T", [(4, 4, 128, 1), (16, 2, 128, 3), (16, 2, 128, 40), (4, 4, 64, 1), (12, 12, 64, 20)])
def test_lengths(cuda_device, L, Hq, Hkv, D, T):
    rng = np.random.default_rng(L)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, max(L, 1), device=cuda_device)
    c = _filled(Hkv, D, L, 64, cuda_device, L + T, spare=1 if L % 2 else 131)
    _check(hp, _tensors(Hq, Hkv, D, T, cuda_device, L), c, random_forest(rng, T), False)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("C", [1, 4, 16, 32, 64, 128])
def test_chunk_sums_of_every_size(cuda_device, block, C):
    for Hq, Hkv, D, T, L in ((16, 4, 128, 20, 777), (4, 4, 64, 3, 500), (32, 8, 128, 1, 1111)):
        hp = GuardedHotPath(Hq, Hkv, D, T, C, 4, L, device=cuda_device)
        c = _filled(Hkv, D, L, block, cuda_device, C)
        _check(hp, _tensors(Hq, Hkv, D, T, cuda_device, block), c, random_forest(np.random.default_rng(C), T), True)


@pytest.mark.parametrize("T", [1, 7, 60])
def test_a_long_prefix_with_needles(cuda_device, T):
    """A few keys far back take nearly all of a row, the rest of 30000 very little each: both count."""
    dev, Hq, Hkv, D, L = cuda_device, 8, 2, 128, 30011
    g = torch.Generator().manual_seed(T)
    K = torch.randn((L, Hkv, D), generator=g)
    K[[17, 20000, 29999]] *= 6
    V = torch.randn((L, Hkv, D), generator=g)
    c = GuardedCache8(Hkv, D, L, 32, dev)
    c.append(K.to(torch.bfloat16).to(dev), V.to(torch.bfloat16).to(dev))
    t = _tensors(Hq, Hkv, D, T, dev, T)
    t["Q"][:, ::2] = (K[[17, 20000, 29999, 5]].repeat_interleave(1, 0)[np.arange(T) % 4][:, [0, 0, 1, 1]] / 6).to(torch.bfloat16).to(dev)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    _check(hp, t, c, random_forest(np.random.default_rng(T), T), True)


@pytest.mark.parametrize("T", [1, 30])
def test_scales_far_apart(cuda_device, T):
    """Blocks whose keys or values differ by many powers of two, zeros among them, and queries of any size."""
    dev, Hq, Hkv, D, L = cuda_device, 8, 4, 64, 640
    g = torch.Generator().manual_seed(T)
    K, V = torch.randn((L, Hkv, D), generator=g), torch.randn((L, Hkv, D), generator=g)
    for b in range(L // 32):
        V[b * 32:b * 32 + 32] *= 2.0 ** ((b * 7) % 41 - 20)
        K[b * 32:b * 32 + 32] *= 2.0 ** -((b * 5) % 23)
    V[64:96] = 0
    K[300:340] = 0
    c = GuardedCache8(Hkv, D, L, 32, dev)
    c.append(K.to(torch.bfloat16).to(dev), V.to(torch.bfloat16).to(dev))
    t = _tensors(Hq, Hkv, D, T, dev, T)
    t["Q"][:, 1] *= 2.0 ** -30
    t["Q"][:, 2] *= 2.0 ** 4
    t["Q"][:, 3] = 0
    t["V_tree"] *= 2.0 ** 12
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    _check(hp, t, c, random_forest(np.random.default_rng(T), T), True)


def test_strides_and_scale(cuda_device):
    """Q, O, the tree and the cache as parts of larger tensors, codes head by head, scales transposed, a softmax scale."""
    dev, Hq, Hkv, D, T, L = cuda_device, 16, 4, 128, 11, 333
    c = _filled(Hkv, D, L, 64, dev, 5)
    t = _tensors(Hq, Hkv, D, T, dev, 6)
    K, V = values(c)
    codes = [torch.empty((Hkv, L + 40, D + 32), dtype=torch.uint8, device=dev).random_(0, 256).view(torch.float8_e4m3fn)[:, :, :D].transpose(0, 1)
             for _ in range(2)]
    scales = [torch.empty((Hkv, 9), dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu).t() for _ in range(2)]
    for dst, src in zip(codes, (c.K, c.V)):
        dst.view(torch.uint8)[:L].copy_(src[:L].view(torch.uint8))
    for dst, src in zip(scales, (c.K_scale, c.V_scale)):
        dst.view(torch.uint8)[:6].copy_(src.view(torch.uint8)[:6])
    wide = {k: torch.zeros((v.shape[0], v.shape[1] + 1, D + 8), dtype=torch.bfloat16, device=dev) for k, v in t.items()}
    for k in wide:
        wide[k][:, 1:, 8:] = t[k]
        wide[k] = wide[k][:, 1:, 8:]
    O = torch.full((T, Hq + 2, D + 16), 7.0, dtype=torch.bfloat16, device=dev)
    lse = torch.empty((Hq, T), dtype=torch.float32, device=dev)
    parent = random_forest(np.random.default_rng(1), T)
    d = api.make_attn_desc(wide["Q"], codes[0], wide["K_tree"], O[:, 1:Hq + 1, 8:8 + D], L, 32, 0.05, False)
    ws = torch.empty(api.specext_verify_attn_q8_workspace(d, 64), dtype=torch.uint8, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    api.specext_verify_attn_q8(d, wide["Q"], *codes, *scales, 64, wide["K_tree"], wide["V_tree"], torch.from_numpy(parent).to(dev),
                               O[:, 1:Hq + 1, 8:8 + D], lse, None, ws, status)
    check_attention(t["Q"], K, V, t["K_tree"], t["V_tree"], parent, 32, O[:, 1:Hq + 1, 8:8 + D], lse, None, 0.05)
    assert int(status) == 0
    assert (O[:, 0] == 7).all() and (O[:, Hq + 1] == 7).all() and (O[:, :, :8] == 7).all() and (O[:, :, 8 + D:] == 7).all()


@pytest.mark.parametrize("T", [1, 40])
def test_a_nan_scale_reaches_its_head_only(cuda_device, T):
    dev, Hq, Hkv, D, L = cuda_device, 8, 4, 128, 500
    for which in ("K", "V"):
        c = GuardedCache8(Hkv, D, L, 32, dev)
        g = torch.Generator().manual_seed(3)
        K, V = (torch.randn((L, Hkv, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2))
        (K if which == "K" else V)[200, 1, 3] = float("inf")
        c.append(K, V)
        hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
        t = _tensors(Hq, Hkv, D, T, dev, 4)
        hp.verify_attn_q8(t, c, torch.from_numpy(random_forest(np.random.default_rng(T), T)).to(dev), False)
        assert hp.read_status() == 0
        O = hp.O.float().isnan()
        assert O[:, 2:4].all() and not O[:, :2].any() and not O[:, 4:].any()


def test_a_node_that_is_not_seen_may_hold_anything(cuda_device):
    """Keys of nodes that a row does not see: infinities and NaN there leave its result alone."""
    dev, Hq, Hkv, D, T, L = cuda_device, 8, 2, 128, 12, 200
    parent = np.array([-1, 0, 1, -1, 3, 3, 0, -1, 7, 8, 2, 2], dtype=np.int32)
    c = _filled(Hkv, D, L, 32, dev, 8)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, 9)
    par = torch.from_numpy(parent).to(dev)
    hp.verify_attn_q8(t, c, par, False)
    O, lse = hp.O.clone(), hp.lse.clone()
    t["K_tree"][8, 0, 5], t["K_tree"][8, 1, 0], t["K_tree"][9, 0, 1] = float("nan"), float("inf"), float("-inf")
    hp.verify_attn_q8(t, c, par, False)
    alone = [i for i in range(T) if i not in (8, 9)]
    assert torch.equal(hp.O[alone], O[alone]) and torch.equal(hp.lse[:, alone], lse[:, alone])


def test_a_bad_tree_is_reported(cuda_device):
    dev = cuda_device
    c = _filled(2, 64, 100, 32, dev, 1)
    hp = GuardedHotPath(4, 2, 64, 3, 32, 4, 100, device=dev)
    hp.verify_attn_q8(_tensors(4, 2, 64, 3, dev, 1), c, torch.tensor([-1, 1, 0], dtype=torch.int32, device=dev), False)
    assert "BAD_TREE" in api.status_bits(hp.read_status())


@pytest.mark.parametrize("T,L", [(1, 5000), (1, 40000), (8, 9000), (60, 3000), (60, 20000)])
def test_the_same_call_gives_the_same_bits(cuda_device, T, L):
    dev, Hq, Hkv, D = cuda_device, 32, 8, 128
    c = _filled(Hkv, D, L, 32, dev, T)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, T)
    par = torch.from_numpy(random_forest(np.random.default_rng(T), T)).to(dev)
    hp.verify_attn_q8(t, c, par, True)
    O, lse, cs = hp.O.clone(), hp.lse.clone(), hp.chunk_score(L).clone()
    for _ in range(20):
        hp.verify_attn_q8(t, c, par, True)
        assert torch.equal(hp.O, O) and torch.equal(hp.lse, lse) and torch.equal(hp.chunk_score(L), cs)
    hp.verify_attn_q8(t, c, par, False)
    O = hp.O.clone()
    for _ in range(20):
        hp.verify_attn_q8(t, c, par, False)
        assert torch.equal(hp.O, O)


def test_a_cache_past_32_bits_of_offset(cuda_device):
    """16 KV heads spread over rows of 512 KB: token 8191 lies more than 2^32 bytes behind token 0."""
    dev, Hkv, D, L, T = cuda_device, 2, 64, 8192, 2
    row = 1 << 19
    room = torch.empty((2, L * row), dtype=torch.uint8, device=dev)
    codes = [room[i].view(torch.float8_e4m3fn).as_strided((L, Hkv, D), (row, row // 4, 1)) for i in range(2)]
    scales = [torch.zeros((L // 32, Hkv), dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu) for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    g = torch.Generator().manual_seed(1)
    K, V = (torch.randn((L, Hkv, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2))
    api.specext_quantize_kv(K, V, 0, *codes, *scales, 32, status)
    c = GuardedCache8(Hkv, D, L, 32, dev)
    c.append(K, V)
    t = _tensors(4, Hkv, D, T, dev, 1)
    hp = GuardedHotPath(4, Hkv, D, T, 32, 4, L, device=dev)
    parent = np.array([-1, 0], dtype=np.int32)
    par = torch.from_numpy(parent).to(dev)
    ref, _, _ = _check(hp, t, c, parent, False)
    O, lse = torch.empty_like(hp.O), torch.empty_like(hp.lse)
    d = api.make_attn_desc(t["Q"], codes[0], t["K_tree"], O, L, 32)
    ws = torch.empty(api.specext_verify_attn_q8_workspace(d, 32), dtype=torch.uint8, device=dev)
    api.specext_verify_attn_q8(d, t["Q"], *codes, *scales, 32, t["K_tree"], t["V_tree"], par, O, lse, None, ws, status)
    assert torch.equal(O, hp.O) and torch.equal(lse, hp.lse) and int(status) == 0
