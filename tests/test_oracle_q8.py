"""Pins of the oracle of the 8-bit cache and of the token log probabilities: the number format against torch's own
conversions, the scale rule by hand, the log probabilities against closed forms and torch in fp64."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc


def test_e4m3_values_are_those_of_the_format():
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(orc.e4m3_values(), codes.view(torch.float8_e4m3fn).double().numpy())


def test_rounding_is_to_nearest_even():
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(4000, generator=g, dtype=torch.float64) * s for s in (1e-3, 0.02, 1.0, 60.0)]).float()
    grid = torch.from_numpy(orc.e4m3_values()[:127].copy())
    x = torch.cat([x, ((grid[1:] + grid[:-1]) / 2).float(), -((grid[1:] + grid[:-1]) / 2).float(), grid.float()]).clamp(-448, 448)
    np.testing.assert_array_equal(orc.e4m3_round(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("m,e", [(448.0, 0), (448.5, 1), (896.0, 1), (1.75, -8), (1.7578125, -7), (0.0, -100), (1e-38, -100)])
def test_scale_is_the_smallest_power_of_two(m, e):
    assert orc.scale_exponent(np.array([0.0, -m, m / 2])) == e


def test_append_keeps_or_raises_the_scale_of_a_block_begun():
    values, exps = np.zeros((64, 1, 2)), np.full((2, 1), np.nan)
    exps[0, 0] = 9
    orc.append(values, exps, np.full((3, 1, 2), 448.0), 0, 32)
    assert exps[0, 0] == 0 and (values[:3] == 448).all()             # a block begun anew takes what its tokens need
    orc.append(values, exps, np.full((1, 1, 2), 1.0), 3, 32)
    assert exps[0, 0] == 0 and (values[3] == 1).all()
    orc.append(values, exps, np.full((1, 1, 2), 896.0 * 4), 4, 32)
    assert exps[0, 0] == 3 and (values[:3] == 56).all() and (values[3] == 0.125).all() and (values[4] == 448).all()
    orc.append(values, exps, np.full((28, 1, 2), np.inf), 5, 32)
    assert np.isnan(exps[0, 0]) and exps[1, 0] > 0 or np.isnan(exps[1, 0])
    np.testing.assert_array_equal(orc.cached(values, np.array([[3.0], [0.0]]), 3, 32), np.full((3, 1, 2), 448.0))


def test_logprobs_against_torch_and_closed_forms():
    g = torch.Generator().manual_seed(2)
    x = torch.randn((5, 1000), generator=g, dtype=torch.float64) * 3
    x[1, 300:] = -np.inf
    tokens = np.array([[0, 999], [5, 299], [7, -1], [1, 1], [500, 2]])
    lp, ent, lse, ids, top = orc.token_logprobs(x.numpy(), tokens, 4, 0.7)
    ref = torch.log_softmax(x / 0.7, dim=1)
    np.testing.assert_allclose(lse, torch.logsumexp(x / 0.7, dim=1).numpy(), rtol=1e-13)
    np.testing.assert_allclose(ent, torch.distributions.Categorical(logits=x / 0.7).entropy().numpy(), rtol=1e-9)
    np.testing.assert_allclose(top, torch.topk(ref, 4).values.numpy(), rtol=1e-12)
    np.testing.assert_array_equal(ids, torch.topk(ref, 4).indices.numpy())
    assert lp[2, 1] == -np.inf and lp[0, 0] == pytest.approx(ref[0, 0].item())
    lp, ent, lse, ids, top = orc.token_logprobs(np.zeros((1, 8)), np.array([[3]]), 3, 1.0)
    assert ent[0] == pytest.approx(np.log(8)) and lp[0, 0] == pytest.approx(-np.log(8)) and ids.tolist() == [[0, 1, 2]]
    lp, ent, lse, ids, top = orc.token_logprobs(np.full((1, 8), -np.inf), np.array([[3]]), 2, 1.0)
    assert lp[0, 0] == -np.inf and ent[0] == 0 and ids.tolist() == [[0, 1]] and (top == -np.inf).all()
    lp, ent, lse, ids, top = orc.token_logprobs(np.array([[0.0, np.nan]]), np.array([[0]]), 1, 1.0)
    assert np.isnan(lp).all() and np.isnan(ent).all() and ids.tolist() == [[-1]]
