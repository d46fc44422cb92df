"""specext_quantize_kv against the oracle, code for code."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2505_20776_b200 import api
from tests.q8_util import GuardedCache8, exponents, garbage
from tests.util import f64

pytestmark = pytest.mark.gpu


def _kv(n, H, D, dev, seed, spread=1.0, pad=0):
    """bf16 K and V [n][H][D], rows `pad` elements apart more than needed."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(2):
        x = torch.randn((n, H, D), generator=g) * torch.exp(spread * torch.randn((n, H, 1), generator=g))
        room = torch.zeros((n, H * D + pad), dtype=torch.bfloat16, device=dev)
        room[:, :H * D] = x.reshape(n, H * D).to(torch.bfloat16).to(dev)
        out.append(room[:, :H * D].view(n, H, D) if pad == 0 else room.as_strided((n, H, D), (H * D + pad, D, 1)))
    return out


class Mirror:
    """The cache and what the oracle says it holds."""

    def __init__(self, H, D, capacity, block, dev, seed=0):
        self.c = GuardedCache8(H, D, capacity, block, dev)
        garbage(self.c, seed)
        self.table = orc.e4m3_values()
        self.ref = [(self.table[t.view(torch.uint8).cpu().numpy()], exponents(s)) for t, s in
                    ((self.c.K, self.c.K_scale), (self.c.V, self.c.V_scale))]

    def append(self, K, V, rows=None, start=None):
        at = self.c.length if start is None else start
        idx = None if rows is None else torch.tensor(rows, dtype=torch.int32, device=self.c.device)
        self.c.append(K, V, idx, start)
        for (v, e), x in zip(self.ref, (K, V)):
            orc.append(v, e, f64(x) if rows is None else f64(x)[rows], at, self.c.block_tokens)

    def check(self):
        assert self.c.read_status() == 0
        self.c.check()
        for (v, e), t, s in zip(self.ref, (self.c.K, self.c.V), (self.c.K_scale, self.c.V_scale)):
            got_e = exponents(s)
            np.testing.assert_array_equal(got_e, e)                 # scales of blocks not touched are as they were
            fine = ~np.isnan(e)[np.arange(v.shape[0]) // self.c.block_tokens]
            np.testing.assert_array_equal(self.table[t.view(torch.uint8).cpu().numpy()][fine], v[fine])


@pytest.mark.parametrize("H,D,block,start,n", [
    (8, 128, 32, 0, 1), (8, 128, 32, 0, 32), (8, 128, 32, 0, 33), (8, 128, 64, 0, 1000), (12, 64, 32, 0, 77),
    (12, 64, 128, 0, 300), (2, 128, 128, 0, 129), (1, 64, 64, 0, 64), (32, 128, 32, 0, 200),
])
def test_from_empty(cuda_device, H, D, block, start, n):
    m = Mirror(H, D, n + 5, block, cuda_device, seed=n)
    m.append(*_kv(n, H, D, cuda_device, 5 + n))
    m.check()


@pytest.mark.parametrize("H,D,block", [(8, 128, 32), (3, 64, 32), (4, 128, 64), (12, 64, 64), (2, 128, 128), (5, 64, 128)])
def test_pieces_that_begin_and_end_inside_blocks(cuda_device, H, D, block):
    """Scales that stay, grow once and grow by much; a growing scale divides the codes before it, and nothing else."""
    m = Mirror(H, D, 5 * block + 7, block, cuda_device, seed=block + H)
    for i, (n, size) in enumerate([(3, 1.0), (1, 0.01), (block - 5, 1.0), (1, 300.0), (2 * block - 1, 1.0), (1, 1e5), (block, 1e-3), (2, 1e9)]):
        K, V = _kv(n, H, D, cuda_device, 100 + i)
        m.append((K.float() * size).to(torch.bfloat16), (V.float() / size).to(torch.bfloat16))
        m.check()
    m.append(*_kv(4, H, D, cuda_device, 7), start=block)             # behind a shorter prefix: a new scale
    m.append(*_kv(4, H, D, cuda_device, 8), start=block + 2)         # and inside it: at least the old one
    m.check()


def test_rows_of_a_tree_strides_and_the_same_row_twice(cuda_device):
    H, D = 8, 128
    m = Mirror(H, D, 500, 32, cuda_device)
    m.append(*_kv(61, H, D, cuda_device, 1, pad=8))
    K, V = _kv(60, H, D, cuda_device, 2, pad=24)
    m.append(K, V, rows=[0, 7, 7, 59, 12])
    m.append(K, V, rows=[3])
    m.check()


def test_codes_of_another_layout(cuda_device):
    """Codes head by head and scales transposed: any strides that are multiples of 16 bytes, any for the scales."""
    dev, H, D, n = cuda_device, 3, 64, 150
    K, V = _kv(n, H, D, dev, 3)
    a = GuardedCache8(H, D, n, 32, dev)
    a.append(K, V)
    codes = [torch.zeros((H, n, D), dtype=torch.float8_e4m3fn, device=dev).transpose(0, 1) for _ in range(2)]
    scales = [torch.zeros((H, 5), dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu).t() for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    api.specext_quantize_kv(K, V, 0, *codes, *scales, 32, status)
    for x, y in zip(codes + scales, (a.K, a.V, a.K_scale, a.V_scale)):
        np.testing.assert_array_equal(x.contiguous().view(torch.uint8).cpu().numpy(), y.view(torch.uint8).cpu().numpy())


def test_extremes(cuda_device):
    """Zeros, the limits of bf16, values at 448 times a power of two, and those that become subnormal."""
    dev = cuda_device
    x = torch.zeros((160, 1, 64), dtype=torch.bfloat16)
    big = torch.finfo(torch.bfloat16).max
    x[32, 0, :3] = torch.tensor([448.0, -3.5, 0.001])
    x[64, 0, :3] = torch.tensor([450.0, -448.0, 1e-3])               # bf16 450: one step above
    x[96, 0, :4] = torch.tensor([big, -big, 1.0, big / 1e4])
    x[128, 0, :3] = torch.tensor([1e-36, -1e-38, 1e-40])
    m = Mirror(1, 64, 160, 32, dev)
    m.append(x.to(dev), x.neg().to(dev))
    m.check()
    assert exponents(m.c.K_scale)[:, 0].tolist()[:3] == [-100, 0, 1]


def test_a_value_that_is_not_finite_makes_its_block_nan(cuda_device):
    dev, H, D = cuda_device, 4, 128
    m = Mirror(H, D, 300, 32, dev)
    K, V = _kv(40, H, D, dev, 4)
    K[35, 2, 7] = float("nan")
    V[3, 0, 0] = float("-inf")
    m.append(K, V)
    m.check()
    assert np.argwhere(np.isnan(exponents(m.c.K_scale)[:2])).tolist() == [[1, 2]]
    assert np.argwhere(np.isnan(exponents(m.c.V_scale)[:2])).tolist() == [[0, 0]]
    m.append(*_kv(30, H, D, dev, 5))                                  # the block stays so, the next one is fine
    m.check()
    assert np.isnan(exponents(m.c.K_scale)[1, 2]) and not np.isnan(exponents(m.c.K_scale)[2]).any()
    m.append(*_kv(30, H, D, dev, 6), start=32)                        # begun anew it is fine too
    m.check()


def test_rows_outside_the_source_are_zeros_and_reported(cuda_device):
    dev = cuda_device
    c = GuardedCache8(2, 64, 64, 32, dev)
    K, V = _kv(4, 2, 64, dev, 9)
    c.append(K, V, torch.tensor([1, 4, -1, 2], dtype=torch.int32, device=dev))
    assert "INVALID_ARG" in api.status_bits(c.read_status())
    c.check()
    assert (c.K[1:3].float() == 0).all() and (c.K[0].float() != 0).any()


def test_no_tokens_is_no_launch(cuda_device):
    c = GuardedCache8(2, 64, 64, 32, cuda_device)
    before = api.specext_launch_count()
    c.append(*_kv(1, 2, 64, cuda_device, 9), torch.empty(0, dtype=torch.int32, device=cuda_device))
    assert api.specext_launch_count() == before and c.length == 0
