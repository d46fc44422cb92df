"""The forms that a call on the 8-bit cache takes, told apart by their launches, each against the oracle; behind a kernel that runs
for longer than the library's bounded waits last; and with queries and tree keys that are not finite."""
import numpy as np
import pytest
import torch

from paper_2505_20776_b200 import api
from tests.guards import GuardedHotPath
from tests.q8_util import check_attention, values
from tests.test_gpu_after_slow_kernel import slow_then
from tests.test_gpu_verify_q8 import _filled, _tensors
from tests.util import random_forest

pytestmark = pytest.mark.gpu

FORMS = [
    # (Hq, Hkv, D, T, L, scored, launches)
    (32, 8, 128, 1, 1012, False, 1),          # few rows: clusters, 8 rows,
    (32, 8, 128, 4, 2100, False, 1),          # 16 rows,
    (16, 2, 128, 10, 4003, False, 1),         # several blocks of 16, one of them ragged,
    (32, 8, 128, 60, 700, False, 1),          # clusters of one CTA,
    (12, 12, 64, 20, 900, False, 1),          # head_dim 64
    (8, 1, 128, 1, 70001, False, 2),          # few rows: workers and merge, 8 rows,
    (8, 1, 128, 2, 30011, False, 2),          # 16 rows,
    (4, 4, 64, 1, 60007, False, 2),           # head_dim 64
    (32, 32, 128, 40, 6001, False, 2),        # one CTA of 128 rows,
    (12, 12, 64, 60, 5003, False, 2),         # head_dim 64,
    (16, 2, 128, 10, 4003, True, 2),          # with chunk sums
    (16, 2, 128, 40, 9001, False, 2),         # pairs: two row blocks, the last ragged,
    (32, 8, 128, 60, 4096, False, 2),         # one,
    (32, 8, 128, 33, 20011, True, 3),         # with chunk sums by a launch of their own
]


@pytest.mark.parametrize("Hq,Hkv,D,T,L,scored,want", FORMS)
def test_forms(cuda_device, Hq, Hkv, D, T, L, scored, want):
    dev = cuda_device
    c = _filled(Hkv, D, L, 32, dev, T + L)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, L)
    parent = random_forest(np.random.default_rng(L), T)
    before = api.specext_launch_count()
    hp.verify_attn_q8(t, c, torch.from_numpy(parent).to(dev), scored)
    assert api.specext_launch_count() - before == want
    assert hp.read_status() == 0
    hp.check()
    K, V = values(c)
    check_attention(t["Q"], K, V, t["K_tree"], t["V_tree"], parent, 32, hp.O, hp.lse, hp.chunk_score(L) if scored else None)


@pytest.mark.parametrize("Hq,Hkv,D,T,L,scored,want", [FORMS[0], FORMS[6], FORMS[10], FORMS[12]])
def test_behind_a_kernel_longer_than_the_waits(cuda_device, Hq, Hkv, D, T, L, scored, want):
    dev = cuda_device
    c = _filled(Hkv, D, L, 32, dev, T)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, L)
    parent = random_forest(np.random.default_rng(L), T)
    par = torch.from_numpy(parent).to(dev)
    hp.verify_attn_q8(t, c, par, scored)
    want_O, want_lse = hp.O.clone(), hp.lse.clone()
    hp.O.fill_(float("nan"))
    par[0] = 5                                # no tree: an entry that a call must not see
    torch.cuda.synchronize()
    slow_then(par, int(parent[0]))
    hp.verify_attn_q8(t, c, par, scored)
    assert hp.read_status() == 0
    assert torch.equal(hp.O, want_O) and torch.equal(hp.lse, want_lse)


def test_logprobs_behind_a_kernel_longer_than_the_waits(cuda_device):
    dev = cuda_device
    x = torch.randn((1, 128256), device=dev)
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=dev)
    want = hp.token_logprobs(x, None, 5)[1:]
    bits = x.view(torch.int32)
    first = int(bits[0, 0])
    bits[0, 0] = 0x7fc00000                   # NaN
    torch.cuda.synchronize()
    slow_then(bits[0], first)
    got = hp.token_logprobs(x, None, 5)[1:]
    assert hp.read_status() == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T,L", [(2, 300), (60, 5000)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_values_that_are_not_finite_stay_with_their_rows(cuda_device, T, L, value):
    """A query of one node and head, and a key of the last node (a leaf): those rows are not finite, all others as before."""
    dev, Hq, Hkv, D = cuda_device, 8, 2, 128
    c = _filled(Hkv, D, L, 32, dev, 3)
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, 4)
    par = torch.from_numpy(random_forest(np.random.default_rng(T), T)).to(dev)
    hp.verify_attn_q8(t, c, par, False)
    O, lse = hp.O.clone(), hp.lse.clone()
    t["Q"][0, 5, 7] = value
    t["K_tree"][T - 1, 0, 9] = value
    hp.verify_attn_q8(t, c, par, False)
    assert hp.read_status() == 0
    hit = torch.zeros((T, Hq), dtype=torch.bool, device=dev)
    hit[0, 5] = True
    hit[T - 1, :4] = True
    same = ~hit
    assert torch.equal(hp.O[same], O[same]) and torch.equal(hp.lse.t()[same], lse.t()[same])
    if value != value:
        assert hp.O[hit].isnan().all() and hp.lse.t()[hit].isnan().all()
    else:
        # an infinite logit: NaN, or the key's weight is 0 or 1; never a finite stand-in for the infinity
        assert torch.equal(hp.O[hit].isnan().any(dim=1), hp.O[hit].isnan().all(dim=1))


@pytest.mark.parametrize("Hq,Hkv,D,T,L", [(4, 4, 128, 100, 32), (4, 4, 128, 128, 16), (4, 4, 64, 128, 160), (8, 4, 128, 100, 32),
                                          (2, 2, 128, 128, 0), (2, 1, 64, 65, 70)])
def test_workers_that_have_only_tree_keys_behind_a_row(cuda_device, Hq, Hkv, D, T, L):
    """Large trees on short prefixes: some workers have no key that the first nodes see."""
    dev = cuda_device
    c = _filled(Hkv, D, max(L, 1), 32, dev, T + L)
    c.length = L
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, max(L, 1), device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, L)
    parent = random_forest(np.random.default_rng(L), T)
    hp.verify_attn_q8(t, c, torch.from_numpy(parent).to(dev), False)
    assert hp.read_status() == 0
    hp.check()
    K, V = values(c, L)
    check_attention(t["Q"], K, V, t["K_tree"], t["V_tree"], parent, 32, hp.O, hp.lse, None)


@pytest.mark.parametrize("L", [0, 130, 500, 900, 1300, 1900, 2400, 3000, 3500, 4200])
@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 32, 128, 33), (64, 16, 128, 40), (36, 36, 64, 70)])
def test_tree_behind_runs_of_any_length(cuda_device, Hq, Hkv, D, T, L):
    """Workers of one to nine tiles, so that the tree's comes first, second, .. in its rings (one CTA, pairs, head_dim 64); a chain."""
    dev = cuda_device
    c = _filled(Hkv, D, max(L, 1), 64, dev, T + L)
    c.length = L
    hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, max(L, 1), device=dev)
    t = _tensors(Hq, Hkv, D, T, dev, L)
    for parent in (random_forest(np.random.default_rng(L), T), np.arange(-1, T - 1, dtype=np.int32)):
        hp.verify_attn_q8(t, c, torch.from_numpy(parent).to(dev), True)
        assert hp.read_status() == 0
        hp.check()
        K, V = values(c, L)
        check_attention(t["Q"], K, V, t["K_tree"], t["V_tree"], parent, 32, hp.O, hp.lse, hp.chunk_score(L) if L else None)


def test_trees_that_are_none(cuda_device):
    """A parent behind its node or below -1 is reported, by either kernel; the rows whose path it is not on are as before."""
    dev, Hq, Hkv, D, T, L = cuda_device, 16, 4, 128, 70, 2100
    c = _filled(Hkv, D, L, 32, dev, 9)
    t = _tensors(Hq, Hkv, D, T, dev, 9)
    good = random_forest(np.random.default_rng(9), T)
    for scored in (False, True):
        hp = GuardedHotPath(Hq, Hkv, D, T, 32, 4, L, device=dev)
        hp.verify_attn_q8(t, c, torch.from_numpy(good).to(dev), scored)
        assert hp.read_status() == 0
        O = hp.O.clone()
        for value in (T + 5, T - 1, -2, 2 ** 31 - 1, -2 ** 31):
            bad = good.copy()
            bad[T - 1] = value
            hp.verify_attn_q8(t, c, torch.from_numpy(bad).to(dev), scored)
            assert "BAD_TREE" in api.status_bits(hp.read_status())
            hp.status.zero_()
            assert torch.equal(hp.O[: T - 1], O[: T - 1])
            hp.check()
