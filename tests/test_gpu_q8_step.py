"""A decoding step with the target's cache in 8 bits, its operators together as a program runs them: the prompt into the cache, the
verification of a tree with its chunk scores, retrieval, log probabilities of the children's tokens, the accepted nodes into the
cache, the next step; and the same captured into a graph, on another stream, and behind a kernel that still runs."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle
from oracle import specext_oracle as orc
from paper_2505_20776_b200 import api
from tests.guards import GuardedHotPath
from tests.q8_util import GuardedCache8, check_attention, garbage, values
from tests.testing_lib import load_testing_lib
from tests.util import bf16_bits, f64, random_forest

pytestmark = pytest.mark.gpu

HQ, HKV, D, T, C, K_TOP, VOCAB = 16, 4, 128, 20, 32, 6, 5003


def _inputs(dev, seed, n=1):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(dev)
    t = {"Q": r(T, HQ, D), "K_tree": r(T, HKV, D), "V_tree": r(T, HKV, D)}
    parent = random_forest(np.random.default_rng(seed), T)
    logits = (torch.randn((T, VOCAB), generator=g) * 3).to(dev)
    tokens = torch.randint(0, VOCAB, (T, 2), generator=g, dtype=torch.int32).to(dev)
    return t, parent, logits, tokens


def _path(parent, node):
    out = []
    while node >= 0:
        out.append(int(node))
        node = parent[node]
    return out[::-1]


def test_three_steps(cuda_device):
    dev = cuda_device
    cache, hp = GuardedCache8(HKV, D, 1500, 32, dev), GuardedHotPath(HQ, HKV, D, T, C, K_TOP, 1500, device=dev)
    garbage(cache)
    g = torch.Generator().manual_seed(0)
    prompt = [torch.randn((1001, HKV, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2)]
    cache.append(prompt[0][:700], prompt[1][:700])
    cache.append(prompt[0][700:], prompt[1][700:])
    dK, dV = (torch.randn((1, 1500, HKV, D), generator=g).to(torch.bfloat16) for _ in range(2))
    for step in range(3):
        t, parent, logits, tokens = _inputs(dev, 10 + step)
        L = cache.length
        hp.verify_attn_q8(t, cache, torch.from_numpy(parent).to(dev), True)
        lp, ent, lse, ids, best = hp.token_logprobs(logits, tokens, 10, 0.8)
        row = T - 1 - step
        hp.select_gather(row, L, dK.to(dev), dV.to(dev))
        K, V = values(cache)
        accepted = torch.tensor(_path(parent, row), dtype=torch.int32, device=dev)
        cache.append(t["K_tree"], t["V_tree"], accepted)
        assert hp.read_status() == 0 and cache.read_status() == 0
        hp.check()
        cache.check()
        _, _, cs = check_attention(t["Q"], K, V, t["K_tree"], t["V_tree"], parent, C, hp.O, hp.lse, hp.chunk_score(L))
        idx = orc.select_chunks(cs[row], L, C, K_TOP, key_dtype=np.float64)
        np.testing.assert_array_equal(hp.idx.cpu().numpy(), idx)
        Kr, Vr, n = orc.gather_kv(dK.view(torch.int16).numpy(), dV.view(torch.int16).numpy(), idx, L, C)
        np.testing.assert_array_equal(bf16_bits(hp.K_compact)[:, :n], Kr)
        np.testing.assert_array_equal(bf16_bits(hp.V_compact)[:, :n], Vr)
        r_lp, r_ent, _, r_ids, _ = q8_oracle.token_logprobs(f64(logits), tokens.cpu().numpy(), 10, 0.8)
        np.testing.assert_array_equal(ids.cpu().numpy(), r_ids)
        np.testing.assert_allclose(f64(lp), r_lp, rtol=1e-6, atol=2e-5)
        np.testing.assert_allclose(f64(ent), r_ent, rtol=1e-6, atol=4e-6)
        assert cache.length == L + len(_path(parent, row))
        K2, _ = values(cache)
        new = f64(t["K_tree"])[_path(parent, row)]
        # e4m3: half a step is 2^-4 of the value; below 2^-6 of a scale (448 of them hold the block's largest) half a step of 2^-9
        assert np.all(np.abs(K2[L:] - new) <= 2.0 ** -4 * np.abs(new) + 2.0 ** -10 * 2 * np.abs(K2).max() / 448 * 8)


@pytest.mark.parametrize("nodes,L", [(1, 300), (1, 20000), (6, 3000), (20, 3000)])
def test_captured_calls_replay(cuda_device, nodes, L):
    """One graph of append, attention (with and without scores) and log probabilities; replayed on new inputs it gives what the
    calls give one by one.  A second graph with its own workspace is replayed in between."""
    dev = cuda_device
    g = torch.Generator().manual_seed(nodes)
    KV = [torch.randn((L, HKV, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2)]
    graphs = []
    s = torch.cuda.Stream()
    for k in range(2):
        cache = GuardedCache8(HKV, D, L, 32, dev)
        cache.append(*KV)
        hp = GuardedHotPath(HQ, HKV, D, nodes, C, K_TOP, L, device=dev)
        t, _, logits, tokens = _inputs(dev, k)
        t = {n: v[:nodes].contiguous() for n, v in t.items()}
        par = torch.arange(-1, nodes - 1, dtype=torch.int32, device=dev)
        new = [x[:3].clone() for x in KV]
        out = [torch.empty((T, 2), device=dev), torch.empty(T, device=dev), torch.empty(T, device=dev),
               torch.empty((T, 5), dtype=torch.int32, device=dev), torch.empty((T, 5), device=dev)]

        def step(cache=cache, hp=hp, t=t, logits=logits, tokens=tokens, par=par, new=new, out=out):
            cache.append(*new, start=L - 3)
            hp.verify_attn_q8(t, cache, par, False)
            hp.verify_attn_q8(t, cache, par, True)
            api.specext_token_logprobs(logits, tokens, *out, hp.status)

        with torch.cuda.stream(s):
            step()                                       # (allocates the workspace)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        graphs.append((graph, step, cache, hp, t, logits, new, out))
    for i in range(4):
        graph, step, cache, hp, t, logits, new, out = graphs[i % 2]
        for x in list(t.values()) + new:
            x.copy_(torch.randn(x.shape, generator=g).to(torch.bfloat16))
        logits.copy_(torch.randn(logits.shape, generator=g))
        graph.replay()
        graphs[1 - i % 2][0].replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (hp.O, hp.lse, hp.chunk_score(L), cache.K.view(torch.uint8), cache.K_scale.view(torch.uint8), *out)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (hp.O, hp.lse, hp.chunk_score(L), cache.K.view(torch.uint8), cache.K_scale.view(torch.uint8), *out)):
            assert torch.equal(a, b)
        assert hp.read_status() == 0 and cache.read_status() == 0
        hp.check()
        cache.check()


@pytest.mark.parametrize("nodes,L", [(1, 500), (1, 9000), (20, 2000)])
def test_behind_a_kernel_that_still_runs(cuda_device, nodes, L):
    """Every call waits for the kernel before it in the stream, whose last write is an input of the call."""
    dev, lib = cuda_device, load_testing_lib()
    cache, hp = GuardedCache8(HKV, D, L + 64, 32, dev), GuardedHotPath(HQ, HKV, D, nodes, C, K_TOP, L + 64, device=dev)
    g = torch.Generator().manual_seed(1)
    KV = [torch.randn((L, HKV, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2)]
    t, _, logits, tokens = _inputs(dev, 3)
    t = {n: v[:nodes].contiguous() for n, v in t.items()}
    par = torch.arange(-1, nodes - 1, dtype=torch.int32, device=dev)

    def slow(where, value):
        assert lib.specext_test_slow_kernel(2_000_000, where.data_ptr(), value, torch.cuda.current_stream().cuda_stream) == 0

    def run(late):
        word = KV[0].view(torch.int32)[5, 1]
        word[0] = 0
        if late:
            slow(word, 0x41404140)
        else:
            word[0] = 0x41404140
        cache.append(*KV, start=0)
        scale = cache.V_scale.view(torch.uint8).view(-1)[:4].view(torch.int32)
        if late:
            slow(scale, 0x7a7b7c7d)
        else:
            scale[0] = 0x7a7b7c7d
        hp.verify_attn_q8(t, cache, par, False)
        x = logits.view(torch.int32)[0]
        x[7] = 0
        if late:
            slow(x[7:], 0x41a00000)
        else:
            x[7] = 0x41a00000
        rest = hp.token_logprobs(logits, tokens, 5)
        return [v.clone() for v in (hp.O, hp.lse, cache.K.view(torch.uint8)[:L], *rest)]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)
    assert hp.read_status() == 0


def test_on_another_stream_beside_other_work(cuda_device):
    """Two sequences on two streams at once, each with its own buffers."""
    dev = cuda_device
    sides = []
    for k in range(2):
        g = torch.Generator().manual_seed(k)
        L = 2000 + 500 * k
        cache, hp = GuardedCache8(HKV, D, L, 32, dev), GuardedHotPath(HQ, HKV, D, T, C, K_TOP, L, device=dev)
        KV = [torch.randn((L, HKV, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2)]
        t, parent, logits, tokens = _inputs(dev, 20 + k)
        sides.append((cache, hp, KV, t, torch.from_numpy(parent).to(dev), logits, tokens, torch.cuda.Stream()))

    def run(side):
        cache, hp, KV, t, par, logits, tokens, _ = side
        cache.append(*KV, start=0)
        hp.verify_attn_q8(t, cache, par, True)
        return [v.clone() for v in (hp.O, hp.lse, hp.chunk_score(cache.length), *hp.token_logprobs(logits, tokens, 7))]

    want = [run(s) for s in sides]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(10):
        for k in (0, 1):
            with torch.cuda.stream(sides[k][7]):
                got[k] = run(sides[k])
    torch.cuda.synchronize()
    for a, b in zip(want[0] + want[1], got[0] + got[1]):
        assert torch.equal(a, b)
    for s in sides:
        assert s[0].read_status() == 0 and s[1].read_status() == 0
        s[0].check()
        s[1].check()


def test_a_graph_keeps_its_workspace(cuda_device):
    """A graph of a call with a small workspace is replayed after calls that need larger ones."""
    dev, L = cuda_device, 6001
    g = torch.Generator().manual_seed(21)
    cache = GuardedCache8(HKV, D, L, 32, dev)
    cache.append(*(torch.randn((L, HKV, D), generator=g).to(torch.bfloat16).to(dev) for _ in range(2)))
    hp = GuardedHotPath(HQ, HKV, D, T, C, K_TOP, L, device=dev)
    t, parent, _, _ = _inputs(dev, 22)
    par = torch.from_numpy(parent).to(dev)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hp.verify_attn_q8(t, cache, par, False)
    torch.cuda.synchronize()
    want, graph = hp.O.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hp.verify_attn_q8(t, cache, par, False)
    captured = hp._ws_q8[-1]
    hp.verify_attn_q8(t, cache, par, True)
    assert hp._ws_q8[-1] is not captured and any(w is captured for w in hp._ws_q8)
    hp.O.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert hp.read_status() == 0 and torch.equal(hp.O, want)
    hp.check()
