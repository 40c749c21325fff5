"""The 8-bit rows' and the block choice's plain forms on the CPU."""

import numpy as np
import pytest
import torch

from oracle import blocks, quant


def test_grid_is_the_e4m3_format():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    assert np.array_equal(quant.e4m3_values(), codes.double().numpy())


def test_rounding_is_to_nearest_even():
    x = np.concatenate([np.linspace(-448, 448, 20001), quant.e4m3_values(),
                        (quant.e4m3_values()[1:] + quant.e4m3_values()[:-1]) / 2])
    want = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(quant.round_e4m3(x.astype(np.float32).astype(np.float64)), want)


@pytest.mark.parametrize("amax,code", [(1.0, 256.0), (1.75, 448.0), (1.7578125, 224.0),
                                       (1.9921875, 256.0), (2.0, 256.0)])
def test_the_largest_value_lands_in_the_top_of_the_range(amax, code):
    for e in (-100, -3, 0, 7, 100):
        row = np.zeros(128)
        row[5] = -amax * 2.0 ** e
        got = quant.held_rows(row)[5]
        s = quant.row_exponent(np.abs(row).max())
        assert got == -code * 2.0 ** int(s)
        # a rounding is off by at most half a step of 2^-3 of the value
        assert abs(got - row[5]) <= 2.0 ** -4 * abs(row[5])


def test_held_values_are_bf16_numbers_and_stay_as_they_are():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((400, 128)) * 2.0 ** rng.integers(-140, 127, (400, 1))
    x = torch.tensor(x, dtype=torch.float32).to(torch.bfloat16)
    x[0] = 0
    x[1, :] = torch.finfo(torch.bfloat16).max
    x[2, :3] = torch.tensor([np.inf, -np.inf, np.nan])
    held = quant.held_rows(x.double().numpy())
    back = torch.tensor(held).to(torch.bfloat16).double().numpy()
    assert np.array_equal(back, held, equal_nan=True)
    assert np.array_equal(quant.held_rows(held), held, equal_nan=True)
    assert np.isnan(held[2, 2]) and held[2, 0] == 240 * 2.0 ** 120


def test_scores_bound_the_products():
    rng = np.random.default_rng(4)
    for trial in range(20):
        k = rng.standard_normal((5 * 32, 128)) * rng.uniform(0.1, 8, 128)
        # queries that 8 bits hold exactly: the score is an upper bound of q . k
        q = rng.integers(-127, 128, (3, 128)).astype(np.float64)
        q[:, 0] = 127
        dots = (q @ k.T).reshape(3, 5, 32).max((0, 2))
        assert (blocks.scores(q, k) >= dots).all()


def test_choice_takes_the_lowest_of_equals_and_keeps_the_recent_rows():
    k = np.ones((200, 128))
    q = np.ones((2, 128))
    rows = blocks.attended(q, k, 199, 2, 64)       # 4 candidates: rows below 128
    assert rows.tolist() == list(range(64)) + list(range(128, 200))
    k[96:128, 3] = 2.0
    rows = blocks.attended(q, k, 199, 2, 64)
    assert rows.tolist() == list(range(32)) + list(range(96, 200))
    assert blocks.attended(q, k, 199, 4, 64).tolist() == list(range(200))
    assert blocks.attended(q, k, 199, 0, 1000).tolist() == list(range(200))
    assert blocks.attended(q, k, 199, 0, 0).tolist() == list(range(192, 200))
