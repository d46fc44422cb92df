"""specext_token_logprobs against the fp64 oracle.

Bounds: a term of the sums is off by the rounding of (x - m) * log2(e) / T in fp32, 2^-24 of at most ~150, and by ex2's 2 ulp;
terms that weigh are those near the maximum, so lse and entropy are held to 2e-6 absolute and 1e-6 relative, and a log
probability to that and the two roundings of x / T and of the difference (2^-23 of |x| / T and of the result).
"""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2505_20776_b200 import api
from tests.guards import GuardedHotPath
from tests.util import f64

pytestmark = pytest.mark.gpu


def _check(logits, tokens, k, temperature=1.0):
    dev = logits.device
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=dev)
    t = None if tokens is None else torch.as_tensor(tokens, dtype=torch.int32, device=dev)
    lp, ent, lse, ids, top = hp.token_logprobs(logits, t, k, temperature)
    assert hp.read_status() == 0
    hp.check()
    x = f64(logits)
    given = np.zeros((x.shape[0], 0), dtype=np.int64) if tokens is None else np.asarray(tokens)
    r_lp, r_ent, r_lse, r_ids, r_top = orc.token_logprobs(x, given, k, temperature)
    np.testing.assert_array_equal(ids.cpu().numpy(), r_ids)
    size = np.max(np.abs(x[np.isfinite(x)]), initial=0.0) / temperature if np.isfinite(x).any() else 0.0
    size = min(size, 1e6)                                            # (the type's lowest value as a mask takes no part)
    # (results are fp32: bf16's lowest value / 0.7 is -4.84e38, past its range of 3.41e38, and rounds to -inf)
    with np.errstate(over="ignore"):
        r_lse = np.asarray(r_lse).astype(np.float32).astype(np.float64)
    np.testing.assert_allclose(f64(lse), r_lse, rtol=1e-6, atol=2e-6)
    np.testing.assert_allclose(f64(ent), r_ent, rtol=1e-6, atol=4e-6)
    np.testing.assert_allclose(f64(top), r_top, rtol=1e-6, atol=2e-6 + 2.0 ** -22 * size)
    if tokens is not None:
        np.testing.assert_allclose(f64(lp), r_lp, rtol=1e-6, atol=2e-6 + 2.0 ** -22 * size)


def _logits(R, V, dtype, dev, seed, stride=None, offset=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((R, V), generator=g) * 2.5
    x.scatter_add_(1, torch.randint(0, V, (R, 5), generator=g), 8 * torch.rand((R, 5), generator=g))
    stride = stride or V
    room = torch.full((offset + R * stride + 16,), float("nan"), dtype=dtype, device=dev)
    view = room[offset:offset + R * stride].view(R, stride)[:, :V]
    view.copy_(x.to(dtype))
    return view


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (2, 7), (1, 31), (5, 257), (2, 1000), (3, 2049), (7, 5003), (1, 16384), (2, 32000),
                                 (1, 50257), (60, 4099), (3, 128256), (600, 1111)])
def test_sizes(cuda_device, dtype, R, V):
    rng = np.random.default_rng(V)
    x = _logits(R, V, dtype, cuda_device, R + V)
    for k, given, temp in ((min(V, 10), 3, 1.0), (min(V, 32), 1, 0.5), (1, 12, 2.0)):
        _check(x, rng.integers(-1, V, (R, given)), k, temp)


@pytest.mark.parametrize("dtype,unit", [(torch.bfloat16, 8), (torch.float32, 4)])
def test_rows_at_any_alignment(cuda_device, dtype, unit):
    """Odd row strides and first words anywhere inside a 16-byte piece; NaN lies between the rows and behind the last."""
    for offset in range(unit):
        for V, stride in ((33, 35), (3000, 3001), (20011, 20011 + offset)):
            _check(_logits(3, V, dtype, cuda_device, offset, stride, offset), [[0], [V - 1], [V // 2]], min(20, V))


def test_equal_logits_go_to_the_lower_word(cuda_device):
    dev = cuda_device
    for V in (40, 3000, 128256):
        x = torch.zeros((4, V), device=dev)
        x[1, V // 2:] = 1
        x[2, ::7] = 3
        x[3, V - 20:] = -0.0                                          # the same as zero
        _check(x, [[0], [V - 1], [7], [V - 1]], 32)
        _check(x.to(torch.bfloat16), None, 17)
    x = torch.randint(0, 3, (5, 30000), device=dev).float()
    _check(x, None, 32)


@pytest.mark.parametrize("V", [500, 20000, 128256])
def test_best_words_all_in_one_place(cuda_device, V):
    """Rising, falling and stepped rows, and the words of one thread above all others."""
    dev = cuda_device
    up = torch.arange(V, device=dev, dtype=torch.float32) / V * 20
    step = 8 * 256
    one = torch.zeros(V, device=dev)
    for b in range(0, V, step):
        one[b:b + 8] = 5 + torch.arange(8, device=dev) * 0.25 + b / V
    _check(torch.stack([up, up.flip(0), (up * 4).floor(), one]), [[0], [1], [2], [3]], 32)
    crowd = torch.zeros((1, V), device=dev)
    crowd[0, : V // 2 : 1] = torch.rand(V // 2, device=dev)
    _check(crowd, None, 20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_words_and_rows(cuda_device, dtype):
    """-inf and the type's lowest value as masks: a few words left, one, none; entropy of a certain word is 0."""
    dev, V = cuda_device, 32003
    x = _logits(8, V, dtype, dev, 3).clone()
    low = torch.finfo(dtype).min
    for r, mask in ((0, float("-inf")), (1, low)):
        keep = x[r, [5, 31000, 777]].clone()
        x[r] = mask
        x[r, [5, 31000, 777]] = keep
    x[2] = float("-inf")
    x[2, 4321] = -3.0
    x[3] = float("-inf")
    x[4] = low
    x[5, :16000] = float("-inf")
    x[6, 16000:] = low
    _check(x, [[5, 6], [777, 0], [4321, 1], [0, V - 1], [0, 5], [0, 20000], [0, 20000], [3, -1]], 10)


def test_rows_with_nan_or_infinity(cuda_device):
    dev, V = cuda_device, 9000
    for dtype in (torch.bfloat16, torch.float32):
        x = _logits(4, V, dtype, dev, 4).clone()
        x[0, 8999] = float("nan")
        x[2, 17] = float("inf")
        x[3] = float("nan")
        _check(x, [[0], [1], [17], [5]], 5)


def test_only_what_is_asked_for(cuda_device):
    x = _logits(3, 1500, torch.bfloat16, cuda_device, 6)
    _check(x, None, 0)
    _check(x, None, 4)
    _check(x, [[1], [2], [3]], 0)


def test_tokens_outside_the_vocabulary_are_reported(cuda_device):
    dev = cuda_device
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=dev)
    lp = hp.token_logprobs(_logits(2, 100, torch.float32, dev, 1), torch.tensor([[100, 5], [-2, -1]], dtype=torch.int32, device=dev), 1)[0]
    assert "INVALID_ARG" in api.status_bits(hp.read_status())
    assert lp[0, 0] == float("-inf") and (lp[1] == float("-inf")).all() and torch.isfinite(lp[0, 1])
    hp.check()


def test_no_rows_is_no_launch(cuda_device):
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=cuda_device)
    before = api.specext_launch_count()
    hp.token_logprobs(torch.empty((0, 100), device=cuda_device), None, 4)
    assert api.specext_launch_count() == before


def test_the_same_call_gives_the_same_bits(cuda_device):
    hp = GuardedHotPath(1, 1, 64, 1, 32, 1, 1, device=cuda_device)
    for R, V in ((1, 128256), (60, 32000)):
        x = _logits(R, V, torch.bfloat16, cuda_device, 8)
        ref = hp.token_logprobs(x, None, 20)[1:]
        for _ in range(20):
            assert all(torch.equal(a, b) for a, b in zip(ref, hp.token_logprobs(x, None, 20)[1:]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_more_rows_than_run_at_once(cuda_device, dtype):
    """Odd row strides, and rows of masks, ties, one place, NaN and +inf among them."""
    dev, R, V = cuda_device, 640, 9001
    x = _logits(R, V, dtype, dev, 11, V + 2, 3)
    x[0], x[1], x[2] = float("-inf"), torch.finfo(dtype).min, 0
    x[3, 1:] = float("-inf")
    x[600, 4000:] = torch.finfo(dtype).min
    x[601, :] = torch.arange(V, device=dev).to(dtype) / 512
    x[602, 77], x[603, 8000] = float("nan"), float("inf")
    x[R - 1, : V - 3] = float("-inf")
    _check(x, np.random.default_rng(3).integers(-1, V, (R, 2)), 24, 0.7)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mask", [-1e4, -7.2e5, -7.3e5, -0.9e29, -1.1e29, -1e30, -3e38])
def test_masks_of_any_size(cuda_device, dtype, mask):
    """Rows with few words left, none (each word as likely as the next), or two levels of masks; the sums change their form at 2^20 / c."""
    dev, V = cuda_device, 20003
    x = _logits(5, V, dtype, dev, 12).clone()
    keep = x[:, [9, 12345, V - 1]].clone()
    x[0] = x[1] = x[2] = mask
    x[0, [9, 12345, V - 1]] = keep[0]
    x[1, 12345] = 0
    x[3, : V // 2] = mask
    x[4] = mask
    x[4, ::3] = float("-inf")
    _check(x, [[9, 0], [12345, 1], [5, 6], [0, V - 1], [0, 1]], 8)


@pytest.mark.parametrize("temperature", [1e-3, 30.0, 1e9, 1e25])
def test_temperatures(cuda_device, temperature):
    for dtype in (torch.bfloat16, torch.float32):
        x = _logits(3, 7001, dtype, cuda_device, 13).clone()
        x[2, ::2] = float("-inf")
        _check(x, [[0], [1], [2]], 6, temperature)


def test_references_that_rise_all_along(cuda_device):
    """Every turn of every thread brings a larger maximum: by less than a rescaling takes, by just as much, and by far more."""
    dev, V = cuda_device, 40000
    turn = torch.arange(V, device=dev, dtype=torch.float32) / 2048
    x = torch.stack([turn * 0.2, turn * 4 * 0.6931472, turn * 40, -turn * 0.2])
    _check(x, [[0], [V - 1], [V // 2], [3]], 12)
    _check(x.to(torch.bfloat16), [[0], [V - 1], [V // 2], [3]], 12)


def test_maxima_on_both_sides_of_the_change_of_form(cuda_device):
    """Logits around -2^20 / c and 2^20 / c, a few units wide: threads with the one form are joined with threads with the other."""
    dev, V = cuda_device, 30000
    at = 2.0 ** 20 * 0.6931471805599453
    g = torch.Generator().manual_seed(14)
    wide = (torch.rand((2, V), generator=g, dtype=torch.float64) * 6 - 3).to(dev)
    wide[:, : V // 2] += torch.arange(V // 2, device=dev) * (4.0 / V)
    _check(torch.stack([wide[0] - at, wide[1] + at]).float(), [[0], [V - 1]], 12)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 5, 33])
def test_many_rows_of_few_words(cuda_device, dtype, V):
    for offset in (0, 1):
        x = _logits(1300, V, dtype, cuda_device, 15, V + 1, offset)
        _check(x, np.zeros((1300, 1), dtype=np.int64), V if V < 33 else 32)
