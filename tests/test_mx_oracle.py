"""The oracle of numbers of 4 bits against the definition."""
import numpy as np
import torch

from oracle import mx_oracle as M


def test_all_numbers_of_the_format_come_back():
    for s in (2, 100, 127, 200, 252):
        x = np.zeros(128)
        x[:16] = np.concatenate((M.NUMBERS, -M.NUMBERS)) * 2.0 ** (s - 127)
        codes, scales = M.encode(x)
        assert scales[0] == s and list(scales[1:]) == [2, 2, 2]
        assert np.array_equal(codes[:16], np.arange(16)) and np.array_equal(M.decode(codes, scales), x)


def test_every_number_is_off_by_half_a_step():
    g = torch.Generator().manual_seed(2)
    x = (torch.randn(2000, 128, generator=g) * torch.exp(8 * torch.randn(2000, 1, generator=g))).to(torch.bfloat16).double().numpy()
    codes, scales = M.encode(x)
    y = M.decode(codes, scales)
    unit = np.repeat(2.0 ** (scales - 127.0), 32, -1)
    size = np.abs(x) / unit
    assert np.all(size < 7.0)
    step = np.where(size < 2, 0.5, np.where(size < 4, 1.0, 2.0))
    assert np.all(np.abs(x - y) <= step * unit / 2)
    assert np.all(np.abs(x).reshape(-1, 32).max(1) / unit.reshape(-1, 32)[:, 0] >= 3.5)


def test_ties_go_to_the_even_code():
    x = np.zeros(128)
    x[:9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    codes, scales = M.encode(x)
    assert scales[0] == 127 and list(codes[:9]) == [7, 0, 2, 2, 4, 4, 6, 6, 14]


def test_what_is_no_number():
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(128)
        x[40] = bad
        y = M.decode(*M.encode(x))
        assert np.isnan(y[32:64]).all() and np.array_equal(y[:32], x[:32]) and np.array_equal(y[64:], x[64:])


def test_the_smallest_and_the_largest():
    x = np.zeros(128)
    x[0], x[32], x[64] = 2.0 ** -133, 2.0 ** 127 * (2 - 2.0 ** -7), 2.0 ** -124
    codes, scales = M.encode(x)
    assert list(scales) == [2, 252, 2, 2] and list(codes[[0, 32, 64]]) == [0, 7, 4]
