"""Operators of a decoding program whose target cache is held in 8 bits, as measurable cases.

Three operators, each in a plain form (elementary torch operations in 32 bits) and through the entry points of
`paper_2505_20776_b200`:

  append   new keys and values (a prompt, or the accepted nodes of a draft tree) go into a cache of e4m3 codes with a power
           of two as the scale of each block of tokens and head (e8m0).
  attend   attention of the draft tree's nodes, or of a single token, over that cache and over the tree itself; the last
           layer of a step also yields the chunk scores.
  score    log probabilities of given tokens under rows of logits, with the rows' entropy and their best alternatives.

A case is a dict of plain values: `prepare` makes what a program holds before the call, `run` is one pass, `work` what a
pass cannot do without, `exact` the definition in 64 bits.
"""
import math

import torch

own = False

_GQA8B = (32, 8, 128)             # Llama-3.1-8B layer shape: query heads, KV heads, head dimension
_GQA70B = (64, 8, 128)            # 70B-class layer shape
_MHA = (32, 32, 128)              # one query head per KV head (Vicuna-7B layer shape)
_SMALL = (12, 12, 64)             # 68M-class draft model
_FEW = (16, 2, 128)               # eight query heads per KV head
_WIDTH = 10                       # nodes per level of a draft tree
_FLOOR = 27                       # smallest scale: code 27 of e8m0 stands for 2^-100


def _append(name, heads, block, start, tokens, accepted):
    return {"name": name, "kind": "append", "kv_heads": heads[1], "dim": heads[2], "block": block, "start": start,
            "tokens": tokens, "accepted": accepted}


def _attend(name, heads, block, prefix, spare, nodes, chunk, scored):
    return {"name": name, "kind": "attend", "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "block": block,
            "prefix": prefix, "spare": spare, "nodes": nodes, "chunk": chunk, "scored": scored}


def _score(name, rows, vocab, dtype, given, best, temperature):
    return {"name": name, "kind": "score", "rows": rows, "vocab": vocab, "dtype": dtype, "given": given, "best": best,
            "temperature": temperature}


def listed():
    return [
        # the five accepted nodes of a verification step go behind a ragged 16K cache
        _append("append_accepted", _GQA8B, 32, 16391, 5, True),
        # a 16K prompt goes into an empty cache
        _append("append_prompt_16k", _GQA8B, 64, 0, 16391, False),
        # the second piece of a prompt, for 64-wide heads: it begins inside a block
        _append("append_piece_2k", _SMALL, 32, 1001, 2048, False),
        # single-token decoding of a small model on a short cache
        _attend("attend_token_1k", _SMALL, 32, 1021, 3, 1, 32, False),
        # single-token decoding of the 8B-class target at 16K
        _attend("attend_token_16k", _GQA8B, 32, 16391, 100, 1, 32, False),
        # the same at 128K
        _attend("attend_token_128k", _GQA8B, 64, 131072, 0, 1, 32, False),
        # a level of ten nodes on a 4K cache, eight query heads per KV head
        _attend("attend_level_4k", _FEW, 128, 4003, 93, 10, 32, False),
        # the last layer of a verification step at 16K: a 60-node tree, with the chunk scores
        _attend("attend_tree_16k", _GQA8B, 32, 16384, 0, 60, 32, True),
        # a target without grouped heads at 8K
        _attend("attend_mha_8k", _MHA, 32, 8201, 55, 60, 32, False),
        # one sampled token of a 32000-word model, and the runner-up
        _score("score_token", 1, 32000, "bf16", 1, 2, 1.0),
        # every node of a 60-node tree: its children's tokens and the ten best continuations
        _score("score_tree", 60, 128256, "bf16", 10, 10, 0.5),
        # the tokens of a prompt, from 32-bit logits
        _score("score_prompt", 2047, 32000, "fp32", 1, 5, 1.0),
    ]


def _spread(rng, lo, hi):
    """A whole number, spread over the logarithm of the range."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges, without a name."""
    kind = rng.choice(("append", "attend", "attend", "score"))
    if kind == "append":
        heads = rng.choice((_GQA8B, _GQA8B, _SMALL, _MHA, _FEW))
        accepted = rng.random() < 0.4
        tokens = rng.randint(1, 11) if accepted else min(_spread(rng, 1, 16384), 16000 * 1024 // (heads[1] * heads[2]))
        c = _append("", heads, rng.choice((32, 64, 128)), rng.choice((0, _spread(rng, 1, 8192))), tokens, accepted)
    elif kind == "attend":
        heads = rng.choice((_GQA8B, _GQA8B, _GQA70B, _MHA, _SMALL, _FEW))
        nodes = rng.choice((1, 1, rng.randint(2, 12), rng.randint(13, 64), 60, rng.randint(65, 128)))
        most = min(130000, 130000 * 1024 // (heads[1] * heads[2]), int(16e9 / (4 * heads[0] * heads[2] * nodes)))
        c = _attend("", heads, rng.choice((32, 32, 64, 128)), _spread(rng, 33, most), rng.choice((0, rng.randint(1, 300))),
                    nodes, rng.choice((16, 32, 32, 64)), rng.random() < 0.3)
    else:
        vocab = rng.choice((32000, 128256, _spread(rng, 1000, 160000)))
        dtype = rng.choice(("bf16", "bf16", "fp32"))
        rows = _spread(rng, 1, min(2047, int(2.6e8 / (vocab * (2 if dtype == "bf16" else 4)))))
        c = _score("", rows, vocab, dtype, rng.choice((1, 1, rng.randint(2, 10))), rng.choice((1, 2, 5, 10, rng.randint(3, 20))),
                   rng.choice((1.0, 0.5, 0.8)))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------
# the cache's numbers: a value is code * 2^(scale - 127); of the new values in a block the largest is at most 448 scales


def _needed(x):
    """The e8m0 code of the smallest power of two s with |x| <= 448 s for all x of a block (the last two dimensions but
    the head's: [blocks][block][heads][dim] -> [blocks][heads]); 448 = 0.875 * 2^9."""
    f, e = torch.frexp(x.abs().amax(dim=(1, 3)))
    return torch.where(f == 0, torch.full_like(e, _FLOOR), (e - 9 + (f > 0.875).to(e.dtype) + 127).clamp_min(_FLOOR))


def _power(code):
    """2^(code - 127) as fp32, for [blocks][heads] codes, against [blocks][block][heads][dim]."""
    return torch.ldexp(torch.ones(code.shape, device=code.device), code.to(torch.int32) - 127)[:, None, :, None]


def _blocks(x, block, lead, n_blocks):
    """[tokens][heads][dim] -> [n_blocks][block][heads][dim] in fp32, zeros in front (`lead` tokens) and behind."""
    out = torch.zeros((n_blocks * block,) + x.shape[1:], device=x.device)
    out[lead:lead + x.shape[0]] = x
    return out.view((n_blocks, block) + x.shape[1:])


def _append_plain(x, start, block, codes, scale):
    """Appends x [n][heads][dim] to codes [>= start+n][heads][dim] (e4m3) and scale [blocks][heads] (e8m0 as uint8)."""
    n, b0, lead = x.shape[0], start // block, start % block
    nb = (start + n + block - 1) // block - b0
    new = _blocks(x, block, lead, nb)
    code = _needed(new)
    if lead:
        # the block that the first new token falls into keeps its scale or gets a larger one
        code[0] = torch.maximum(code[0], scale[b0].to(code.dtype))
        new[0, :lead] = codes[start - lead:start].float() * _power(scale[b0:b0 + 1])[0]
    out = (new / _power(code)).to(torch.float8_e4m3fn).flatten(0, 1)
    codes[start - lead:start + n] = out[:lead + n]
    scale[b0:b0 + nb] = code.to(torch.uint8)


def _values(codes, scale, block):
    """The cache's values as fp32: codes [L][heads][dim], scale [blocks][heads]."""
    at = torch.arange(codes.shape[0], device=codes.device) // block
    return codes.float() * torch.ldexp(torch.ones(scale.shape, device=scale.device), scale.to(torch.int32) - 127)[at, :, None]


# ---------------------------------------------------------------------------------------------------------
# inputs


def _randn(shape, gen, device, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device=device, dtype=torch.float32).to(dtype)


def _tree(nodes, gen, device):
    """parent[]: levels of 10 nodes, each node's parent anywhere in the level above (-1 = the last prefix token)."""
    i = torch.arange(nodes, device=device)
    pick = torch.randint(0, _WIDTH, (nodes,), generator=gen, device=device)
    return torch.where(i < _WIDTH, torch.full_like(i, -1), (i // _WIDTH - 1) * _WIDTH + pick).to(torch.int32)


def _spoken(shape, gen, device):
    """Keys or values as a model makes them: channels of different size, some tokens larger than others."""
    tokens, heads, dim = shape
    channel = torch.exp(0.5 * torch.randn((1, heads, dim), generator=gen, device=device))
    token = torch.exp(0.2 * torch.randn((tokens, heads, 1), generator=gen, device=device))
    return (torch.randn(shape, generator=gen, device=device) * channel * token).to(torch.bfloat16)


def _cache(capacity, filled, c, gen, device):
    """An 8-bit cache of `capacity` tokens, the first `filled` of them written."""
    heads, dim, block = c["kv_heads"], c["dim"], c["block"]
    nb = (capacity + block - 1) // block
    k, v = (torch.zeros((capacity, heads, dim), dtype=torch.float8_e4m3fn, device=device) for _ in range(2))
    ks, vs = (torch.zeros((nb, heads), dtype=torch.uint8, device=device) for _ in range(2))
    if filled:
        _append_plain(_spoken((filled, heads, dim), gen, device), 0, block, k, ks)
        _append_plain(_spoken((filled, heads, dim), gen, device), 0, block, v, vs)
    return k, v, ks.view(torch.float8_e8m0fnu), vs.view(torch.float8_e8m0fnu)


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    c = dict(case)
    s = {"case": c, "status": torch.zeros(1, dtype=torch.int32, device=dev)}
    if c["kind"] == "score":
        rows, vocab = c["rows"], c["vocab"]
        dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        # a few words of every row stand out, as in a model's predictions; the given tokens are often among them
        x = torch.randn((rows, vocab), generator=gen, device=dev) * 2.0
        stand = torch.randint(0, vocab, (rows, 40), generator=gen, device=dev)
        x.scatter_add_(1, stand, 6.0 * torch.rand((rows, 40), generator=gen, device=dev) + 4.0)
        s["logits"] = x.to(dtype)
        tokens = torch.randint(0, vocab, (rows, c["given"]), generator=gen, device=dev)
        tokens[:, ::2] = stand[:, :c["given"]:2]
        s["tokens"] = tokens.to(torch.int32)
        return s
    heads, dim, block = c["kv_heads"], c["dim"], c["block"]
    if c["kind"] == "append":
        n, start = c["tokens"], c["start"]
        capacity = (start + n + block) // block * block
        s["K_codes"], s["V_codes"], s["K_scale"], s["V_scale"] = _cache(capacity, start, c, gen, dev)
        n_src = 60 if c["accepted"] else n
        s["K"], s["V"] = (_spoken((n_src, heads, dim), gen, dev) for _ in range(2))
        s["rows"] = torch.sort(torch.randperm(n_src, generator=gen, device=dev)[:n])[0].to(torch.int32) if c["accepted"] else None
        return s
    nodes, q, L = c["nodes"], c["q_heads"], c["prefix"]
    s["K_codes"], s["V_codes"], s["K_scale"], s["V_scale"] = _cache(L + c["spare"], L, c, gen, dev)
    s["Q"] = _randn((nodes, q, dim), gen, dev)
    s["K_tree"], s["V_tree"] = (_spoken((nodes, heads, dim), gen, dev) for _ in range(2))
    s["parent"] = _tree(nodes, gen, dev)
    return s


# ---------------------------------------------------------------------------------------------------------
# one pass


def _append_run(s):
    c = s["case"]
    if own:
        from paper_2505_20776_b200 import api
        api.specext_quantize_kv(s["K"], s["V"], c["start"], s["K_codes"], s["V_codes"], s["K_scale"], s["V_scale"], c["block"],
                                s["status"], s["rows"])
    else:
        K, V = (s["K"], s["V"]) if s["rows"] is None else (s["K"][s["rows"].long()], s["V"][s["rows"].long()])
        _append_plain(K.float(), c["start"], c["block"], s["K_codes"], s["K_scale"].view(torch.uint8))
        _append_plain(V.float(), c["start"], c["block"], s["V_codes"], s["V_scale"].view(torch.uint8))
    return {"K_codes": s["K_codes"], "V_codes": s["V_codes"], "K_scale": s["K_scale"], "V_scale": s["V_scale"]}


def _attend_own(s):
    from paper_2505_20776_b200 import api
    c = s["case"]
    nodes, q, dim, L = c["nodes"], c["q_heads"], c["dim"], c["prefix"]
    if "O" not in s:
        # what a program keeps from step to step: its outputs and the scratch
        dev = s["Q"].device
        s["O"] = torch.empty_like(s["Q"])
        s["lse"] = torch.empty((q, nodes), dtype=torch.float32, device=dev)
        s["chunk_score"] = torch.empty((nodes, -(-L // c["chunk"])), dtype=torch.float32, device=dev) if c["scored"] else None
        d = api.make_attn_desc(s["Q"], s["K_codes"], s["K_tree"], s["O"], L, c["chunk"], 0.0, c["scored"])
        s["ws"] = torch.empty(api.specext_verify_attn_q8_workspace(d, c["block"]), dtype=torch.uint8, device=dev)
    d = api.make_attn_desc(s["Q"], s["K_codes"], s["K_tree"], s["O"], L, c["chunk"], 0.0, c["scored"])
    api.specext_verify_attn_q8(d, s["Q"], s["K_codes"], s["V_codes"], s["K_scale"], s["V_scale"], c["block"], s["K_tree"],
                               s["V_tree"], s["parent"], s["O"], s["lse"], s["chunk_score"], s["ws"], s["status"])
    out = {"O": s["O"], "lse": s["lse"]}
    if c["scored"]:
        out["chunk_score"] = s["chunk_score"]
    return out


def _attend_plain(s):
    c = s["case"]
    nodes, q, heads, dim, L = c["nodes"], c["q_heads"], c["kv_heads"], c["dim"], c["prefix"]
    K = _values(s["K_codes"][:L], s["K_scale"].view(torch.uint8), c["block"])
    V = _values(s["V_codes"][:L], s["V_scale"].view(torch.uint8), c["block"])
    K = torch.cat((K, s["K_tree"].float())).permute(1, 2, 0)                       # [heads][dim][L + nodes]
    V = torch.cat((V, s["V_tree"].float())).permute(1, 0, 2)                       # [heads][L + nodes][dim]
    G = q // heads
    Q = s["Q"].float().view(nodes, heads, G, dim).permute(1, 2, 0, 3).reshape(heads, G * nodes, dim)
    S = (torch.matmul(Q, K) * dim ** -0.5).view(q, nodes, L + nodes)
    # a node sees itself and its ancestors: the powers of (self + parent) reach them all
    i = torch.arange(nodes, device=Q.device)
    step = (s["parent"].long()[:, None] == i[None, :]) | (i[:, None] == i[None, :])
    seen = torch.linalg.matrix_power(step.double(), nodes) > 0.5
    S[:, :, L:] = torch.where(seen, S[:, :, L:], torch.full_like(S[:, :, L:], -math.inf))
    top = S.amax(dim=2, keepdim=True)
    P = torch.exp(S - top)
    total = P.sum(dim=2, keepdim=True)
    P = P / total
    O = torch.matmul(P.view(heads, G * nodes, L + nodes), V).view(q, nodes, dim).permute(1, 0, 2)
    out = {"O": O.to(torch.bfloat16), "lse": (top + torch.log(total)).squeeze(2)}
    if c["scored"]:
        C, n = c["chunk"], -(-L // c["chunk"])
        mass = torch.zeros((nodes, n * C), device=Q.device)
        mass[:, :L] = P[:, :, :L].mean(dim=0)
        out["chunk_score"] = mass.view(nodes, n, C).sum(dim=2)
    return out


def _score_run(s):
    c = s["case"]
    rows, k = c["rows"], c["best"]
    if own:
        from paper_2505_20776_b200 import api
        if "lse" not in s:
            dev = s["logits"].device
            s["logprob"] = torch.empty((rows, c["given"]), dtype=torch.float32, device=dev)
            s["entropy"], s["lse"] = (torch.empty(rows, dtype=torch.float32, device=dev) for _ in range(2))
            s["top_ids"] = torch.empty((rows, k), dtype=torch.int32, device=dev)
            s["top_logprob"] = torch.empty((rows, k), dtype=torch.float32, device=dev)
        api.specext_token_logprobs(s["logits"], s["tokens"], s["logprob"], s["entropy"], s["lse"], s["top_ids"], s["top_logprob"],
                                   s["status"], c["temperature"])
        return {n: s[n] for n in ("logprob", "entropy", "lse", "top_ids", "top_logprob")}
    raw = s["logits"].float()
    x = raw / c["temperature"]
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    # minus the sum of p log p, with log p = (x - top) - log(total)
    entropy = torch.log(total[:, 0]) - (e * (x - top)).sum(dim=1) / total[:, 0]
    best, ids = torch.sort(raw, dim=1, descending=True, stable=True)              # equal logits: the lower word first
    return {"logprob": x.gather(1, s["tokens"].long()) - lse, "entropy": entropy, "lse": lse[:, 0],
            "top_ids": ids[:, :k].to(torch.int32), "top_logprob": best[:, :k] / c["temperature"] - lse}


def run(s):
    kind = s["case"]["kind"]
    if kind == "append":
        return _append_run(s)
    if kind == "score":
        return _score_run(s)
    return _attend_own(s) if own else _attend_plain(s)


# ---------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and the definitions in 64 bits


def work(case):
    c = case
    if c["kind"] == "score":
        size = 2 if c["dtype"] == "bf16" else 4
        n = c["rows"] * c["vocab"]
        # per word: the difference to the maximum, the exponential, two sums
        return {"bytes": n * size + c["rows"] * (8 * c["given"] + 8 + 8 * c["best"]), "flops": 5 * n}
    heads, dim, block = c["kv_heads"], c["dim"], c["block"]
    if c["kind"] == "append":
        values = 2 * c["tokens"] * heads * dim
        nb = (c["start"] + c["tokens"] - 1) // block - c["start"] // block + 1
        return {"bytes": values * 3 + 2 * nb * heads + (4 * c["tokens"] if c["accepted"] else 0), "flops": 3 * values}
    nodes, q, L = c["nodes"], c["q_heads"], c["prefix"]
    nb = -(-L // block)
    nbytes = 2 * (L * heads * dim + nb * heads) + 4 * nodes * heads * dim + 4 * nodes * q * dim + 4 * q * nodes + 4 * nodes
    if c["scored"]:
        nbytes += 4 * nodes * -(-L // c["chunk"])
    return {"bytes": nbytes, "flops": 4 * q * dim * (nodes * L + sum(i // _WIDTH + 1 for i in range(nodes)))}


def _power64(exponent):
    return torch.ldexp(torch.ones(exponent.shape, dtype=torch.float64, device=exponent.device), exponent.to(torch.int32))


def _scale64(code):
    """e8m0 as float64 (code 0 of blocks that were never written stands for 2^-127)."""
    return _power64(code.view(torch.uint8).to(torch.int32) - 127)


def _exact_append(x, rows, start, block, codes, scale):
    x = x.double() if rows is None else x[rows.long()].double()
    n = x.shape[0]
    values, sc = codes.double(), _scale64(scale)
    for b in range(start // block, (start + n - 1) // block + 1):
        lo, hi = max(b * block, start), min((b + 1) * block, start + n)
        part = x[lo - start:hi - start]
        # (a bf16 value that is not 448 times a power of two is 0.2 % off one: the margin is for the logarithm's last bit)
        exponent = torch.ceil(torch.log2(part.abs().amax(dim=(0, 2)) / 448) - 1e-9).clamp_min(_FLOOR - 127)
        new = _power64(exponent)
        if lo > b * block:
            new = torch.maximum(new, sc[b])
            values[b * block:lo] *= (sc[b] / new)[None, :, None]
        values[lo:hi] = part / new[None, :, None]
        sc[b] = new
    return values, sc


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "append":
        K, ks = _exact_append(s["K"], s["rows"], c["start"], c["block"], s["K_codes"], s["K_scale"])
        V, vs = _exact_append(s["V"], s["rows"], c["start"], c["block"], s["V_codes"], s["V_scale"])
        return {"K_codes": K, "V_codes": V, "K_scale": ks, "V_scale": vs}
    if c["kind"] == "score":
        got = {"logprob": [], "entropy": [], "lse": [], "top_ids": None, "top_logprob": []}
        for lo in range(0, c["rows"], 64):
            x = s["logits"][lo:lo + 64].double() / c["temperature"]
            lse = torch.logsumexp(x, dim=1, keepdim=True)
            lp = x - lse
            got["logprob"].append(lp.gather(1, s["tokens"][lo:lo + 64].long()))
            got["entropy"].append(-(lp.exp() * lp).sum(dim=1))
            got["lse"].append(lse[:, 0])
            got["top_logprob"].append(torch.topk(lp, c["best"], dim=1).values)
        return {k: v and torch.cat(v) for k, v in got.items()}
    nodes, q, heads, dim, L = c["nodes"], c["q_heads"], c["kv_heads"], c["dim"], c["prefix"]
    dev, G = s["Q"].device, q // heads
    parent = s["parent"].tolist()
    seen = torch.zeros((nodes, nodes), dtype=torch.bool)
    for t in range(nodes):
        u = t
        while u >= 0:
            seen[t, u] = True
            u = parent[u]
    seen = seen.to(dev)
    at = torch.arange(L, device=dev) // c["block"]
    O = torch.empty((nodes, q, dim), dtype=torch.float64, device=dev)
    lse = torch.empty((q, nodes), dtype=torch.float64, device=dev)
    mass = torch.zeros((nodes, L), dtype=torch.float64, device=dev)
    for h in range(q):
        g = h // G
        K = s["K_codes"][:L, g].double() * _scale64(s["K_scale"])[at, g][:, None]
        V = s["V_codes"][:L, g].double() * _scale64(s["V_scale"])[at, g][:, None]
        x = s["Q"][:, h].double() @ torch.cat((K, s["K_tree"][:, g].double())).T / math.sqrt(dim)
        x[:, L:].masked_fill_(~seen, -math.inf)
        p = torch.softmax(x, dim=1)
        O[:, h] = p @ torch.cat((V, s["V_tree"][:, g].double()))
        lse[h] = torch.logsumexp(x, dim=1)
        mass += p[:, :L] / q
    out = {"O": O, "lse": lse}
    if c["scored"]:
        out["chunk_score"] = torch.stack([p.sum(dim=1) for p in mass.split(c["chunk"], dim=1)], dim=1)
    return out
