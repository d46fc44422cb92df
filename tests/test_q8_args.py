"""What the operators of the 8-bit cache and the token log probabilities refuse, by return code and by exception; no GPU."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2505_20776_b200 import api, build
from paper_2505_20776_b200.cache8 import KvCache8
from tests.test_abi import _desc

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 1 << 20                                     # an aligned address that is never used: every call here is refused


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


def _q8(block=32, sb=8, sh=1):
    return api.Q8Desc(block, 0, sb, sh)


def test_workspace_and_descriptors(lib):
    plain, scored = (api.specext_verify_attn_q8_workspace(_desc(want_chunk_score=w), 32) for w in (0, 1))
    assert 0 < plain < scored
    for bad in (dict(head_dim=96), dict(n_tree=0), dict(n_tree=129), dict(chunk_size=3), dict(n_kv_heads=5), dict(prefix_len=-4),
                dict(kv_stride_l=1032), dict(kv_stride_h=120), dict(kv_stride_l=64), dict(softmax_scale=float("inf"))):
        assert api.specext_verify_attn_q8_workspace(_desc(**bad), 32) == 0
    for block in (0, 16, 31, 48, 256, -32):
        assert api.specext_verify_attn_q8_workspace(_desc(), block) == 0
    assert lib.specext_verify_attn_q8_workspace(None, ctypes.byref(_q8())) == 0
    assert lib.specext_verify_attn_q8_workspace(ctypes.byref(_desc()), None) == 0
    assert api.specext_verify_attn_q8_workspace(_desc(prefix_len=0), 128) > 0


def _verify(lib, d=None, q=None, ptrs=None, ws=P, bytes_=1 << 40):
    d = d or _desc(want_chunk_score=0)
    args = [P] * 11 if ptrs is None else ptrs   # Q, K, V, K_scale, V_scale, K_tree, V_tree, parent, O, lse, chunk_score
    return lib.specext_verify_attn_q8(ctypes.byref(d), None if q == 0 else ctypes.byref(q or _q8()), *args, ws, bytes_, P, None)


def test_verify_q8_refusals(lib):
    assert _verify(lib, q=0) == INVALID
    assert _verify(lib, q=_q8(48)) == UNSUPPORTED
    for q in (_q8(sb=0), _q8(sh=-1)):
        assert _verify(lib, q=q) == INVALID
    assert _verify(lib, d=_desc(kv_stride_l=8 * 128 + 8)) == INVALID
    for i in range(10):
        assert _verify(lib, ptrs=[None if j == i else P for j in range(11)]) == INVALID
    assert _verify(lib, d=_desc(), ptrs=[P] * 10 + [None]) == INVALID
    for i in (0, 1, 2, 5, 6, 8):                # (the scales may lie anywhere)
        assert _verify(lib, ptrs=[P + 8 if j == i else P for j in range(11)]) == INVALID
    assert _verify(lib, bytes_=64) == WORKSPACE
    assert _verify(lib, ws=P + 64) == INVALID


def _quantize(lib, **kw):
    a = dict(K=P, V=P, n_src=40, heads=8, dim=128, sl=1024, sh=128, rows=None, n=40, start=5, Kc=P, Vc=P, cl=1024, ch=128, Ks=P, Vs=P,
             q=ctypes.byref(_q8()))
    a.update(kw)
    return lib.specext_quantize_kv(a["K"], a["V"], a["n_src"], a["heads"], a["dim"], a["sl"], a["sh"], a["rows"], a["n"], a["start"],
                                   a["Kc"], a["Vc"], a["cl"], a["ch"], a["Ks"], a["Vs"], a["q"], P, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(K=None), INVALID), (dict(V=None), INVALID), (dict(Kc=None), INVALID), (dict(Vs=None), INVALID), (dict(q=None), INVALID),
    (dict(heads=0), INVALID), (dict(n=-1), INVALID), (dict(n=41), INVALID), (dict(start=-1), INVALID), (dict(start=1 << 24), INVALID),
    (dict(n_src=-1), INVALID), (dict(dim=96), UNSUPPORTED), (dict(sl=1023), INVALID), (dict(sh=64), INVALID), (dict(cl=1032), INVALID),
    (dict(ch=64), INVALID), (dict(K=P + 8), INVALID), (dict(Vc=P + 1), INVALID), (dict(rows=P + 2), INVALID),
    (dict(q=ctypes.byref(_q8(16))), UNSUPPORTED), (dict(q=ctypes.byref(_q8(32, 0, 1))), INVALID), (dict(n=0), OK),
])
def test_quantize_refusals(lib, kw, rc):
    assert _quantize(lib, **kw) == rc


def _logprobs(lib, **kw):
    a = dict(x=P, f=0, rows=4, V=1000, stride=1000, T=1.0, tokens=P, given=2, best=5, lp=P, ent=P, lse=P, ids=P, top=P)
    a.update(kw)
    return lib.specext_token_logprobs(a["x"], a["f"], a["rows"], a["V"], a["stride"], a["T"], a["tokens"], a["given"], a["best"],
                                      a["lp"], a["ent"], a["lse"], a["ids"], a["top"], P, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(x=None), INVALID), (dict(rows=-1), INVALID), (dict(V=0), INVALID), (dict(stride=999), INVALID), (dict(given=-1), INVALID),
    (dict(best=-1), INVALID), (dict(best=33), UNSUPPORTED), (dict(V=4, stride=4, best=5), INVALID), (dict(T=0.0), INVALID),
    (dict(T=-1.0), INVALID), (dict(T=float("nan")), INVALID), (dict(T=float("inf")), INVALID), (dict(T=1e-45), INVALID),
    (dict(tokens=None), INVALID), (dict(lp=None), INVALID), (dict(ent=None), INVALID), (dict(lse=None), INVALID),
    (dict(ids=None), INVALID), (dict(top=None), INVALID), (dict(x=P + 1), INVALID), (dict(f=1, x=P + 2), INVALID),
    (dict(tokens=P + 2), INVALID), (dict(V=(1 << 30) + 1, stride=1 << 31), UNSUPPORTED), (dict(rows=0, x=None), OK),
])
def test_logprobs_refusals(lib, kw, rc):
    assert _logprobs(lib, **kw) == rc


# ---- the binding, on tensors without memory: a call that passes every check ends where a pointer is asked for ----


def _fake(*shape, dtype=torch.bfloat16):
    with FakeTensorMode(allow_non_fake_inputs=True):
        return torch.empty(*shape, dtype=dtype, device="cuda")


E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _call_quantize(K=None, V=None, start=0, Kc=None, Vc=None, Ks=None, Vs=None, block=32, rows=None):
    K = _fake(40, 2, 64) if K is None else K
    Kc, Ks = _fake(100, 2, 64, dtype=E4) if Kc is None else Kc, _fake(4, 2, dtype=E8) if Ks is None else Ks
    api.specext_quantize_kv(K, K if V is None else V, start, Kc, Kc if Vc is None else Vc, Ks, Ks if Vs is None else Vs, block,
                            _fake(1, dtype=torch.int32), rows)


@pytest.mark.parametrize("kw,text", [
    (dict(K=_fake(40, 2, 64, dtype=torch.float16)), "K must be a bf16"), (dict(V=_fake(39, 2, 64)), "share shape"),
    (dict(start=61), "does not hold"), (dict(start=-1), "out of range"), (dict(Kc=_fake(100, 2, 64)), "codes must be"),
    (dict(Ks=_fake(4, 2, dtype=torch.uint8)), "scales must be"), (dict(Ks=_fake(1, 2, dtype=E8)), "does not hold"),
    (dict(Vc=_fake(90, 2, 64, dtype=E4)), "must share"), (dict(Kc=_fake(100, 3, 64, dtype=E4)), "does not hold"),
    (dict(rows=_fake(4, dtype=torch.int64)), "rows must be"), (dict(rows=_fake(4, 1, dtype=torch.int32)), "rows must be"),
    (dict(rows=_fake(101, dtype=torch.int32)), "rows must be|does not hold"),
])
def test_quantize_binding_refusals(kw, text):
    with pytest.raises((ValueError, RuntimeError), match=text + "|data pointer" if "rows" in kw else text):
        _call_quantize(**kw)


def _call_logprobs(x=None, tokens=None, lp=None, ent=None, ids=None, top=None, T=1.0):
    f = torch.float32
    api.specext_token_logprobs(_fake(3, 100) if x is None else x, tokens, lp, _fake(3, dtype=f) if ent is None else ent,
                               _fake(3, dtype=f), ids, top, _fake(1, dtype=torch.int32), T)


@pytest.mark.parametrize("kw", [
    dict(x=_fake(3, 100, dtype=torch.float16)), dict(x=_fake(100)), dict(x=_fake(100, 3).t()), dict(tokens=_fake(3, 2, dtype=torch.int32)),
    dict(ids=_fake(3, 2, dtype=torch.int32)),
])
def test_logprobs_binding_refusals(kw):
    with pytest.raises(ValueError):
        _call_logprobs(**kw)


def test_cache_refusals():
    with pytest.raises(ValueError):
        KvCache8(2, 64, 100, 48, device="cpu")
    c = KvCache8(2, 64, 100, 32, device="cpu")
    K = torch.zeros((101, 2, 64), dtype=torch.bfloat16)
    for n, start in ((101, None), (1, 1), (1, -1)):
        with pytest.raises(ValueError):
            c.append(K[:n], K[:n], start=start)
    with pytest.raises(ValueError, match="CUDA"):                    # there is no CPU path
        c.append(K[:1], K[:1])


@pytest.mark.parametrize("rows,text", [
    (_fake(4, dtype=torch.int64), "rows must be"), (_fake(4, 1, dtype=torch.int32), "rows must be"),
    (_fake(8, dtype=torch.int32)[::2], "rows must be"), (_fake(101, dtype=torch.int32), "does not hold"),
])
def test_what_the_binding_says_of_rows(rows, text):
    """By its own message (a call that passes every check ends with another error, where the stream is asked for)."""
    with pytest.raises(ValueError, match=text):
        _call_quantize(rows=rows)


@pytest.mark.parametrize("kw,text", [
    (dict(tokens=_fake(3, 2, dtype=torch.int64), lp=_fake(3, 2, dtype=torch.float32)), "tokens must be"),
    (dict(tokens=_fake(2, 2, dtype=torch.int32), lp=_fake(2, 2, dtype=torch.float32)), "tokens must be"),
    (dict(tokens=_fake(3, 2, dtype=torch.int32), lp=_fake(3, 3, dtype=torch.float32)), "tokens must be"),
    (dict(tokens=_fake(3, 2, dtype=torch.int32), lp=_fake(3, 2)), "tokens must be"),
    (dict(tokens=_fake(3, dtype=torch.int32), lp=_fake(3, dtype=torch.float32)), "tokens must be"),
    (dict(tokens=_fake(2, 3, dtype=torch.int32).t(), lp=_fake(3, 2, dtype=torch.float32)), "tokens must be"),
    (dict(ids=_fake(3, 2, dtype=torch.int32), top=_fake(3, 1, dtype=torch.float32)), "top_ids must be"),
    (dict(ids=_fake(3, 2, dtype=torch.int64), top=_fake(3, 2, dtype=torch.float32)), "top_ids must be"),
    (dict(ent=_fake(2, dtype=torch.float32)), "entropy and lse"), (dict(ent=_fake(3)), "entropy and lse"),
    (dict(ids=_fake(3, 2, dtype=torch.int32)), "go together"),
])
def test_what_the_binding_says_of_tables(kw, text):
    with pytest.raises(ValueError, match=text):
        _call_logprobs(**kw)


@pytest.mark.parametrize("given", [(1 << 30) + 1, (1 << 31) - 1])
def test_more_given_tokens_than_a_loop_of_int32_counts(lib, given):
    """A loop over them in steps of a thread block would pass 2^31 and go on behind 0."""
    assert _logprobs(lib, given=given) == UNSUPPORTED
    assert _logprobs(lib, given=given, rows=0) == UNSUPPORTED


@pytest.mark.parametrize("T", [3e-39, 4e-39])
def test_temperatures_whose_factor_is_no_number(lib, T):
    """1 / T is a finite number there, log2(e) / T is not: 0 times it made every row NaN."""
    assert _logprobs(lib, T=T) == INVALID
    assert _logprobs(lib, T=T, rows=0) == INVALID and _logprobs(lib, T=4.3e-39, rows=0) == OK
