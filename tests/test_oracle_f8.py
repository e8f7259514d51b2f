"""The fp64 definitions of the 8-bit floating-point operators: against torch's conversions and by hand."""
import numpy as np
import torch

from oracle import f8


def test_decode_is_e4m3():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = f8.decode(codes.numpy())
    assert np.array_equal(got, want, equal_nan=True) and np.isnan(got).sum() == 2 and np.nanmax(got) == f8.TOP


def test_half_step_is_half_the_distance_of_neighbours():
    values = np.unique(f8.decode(np.arange(127)))
    middle = (values[1:] + values[:-1]) / 2
    assert np.array_equal(f8.half_step(middle), (values[1:] - values[:-1]) / 2)


def test_rounding_to_codes_is_within_half_a_step():
    v = np.random.default_rng(0).normal(size=20000) * np.exp(np.random.default_rng(1).uniform(-8, 3, 20000))
    v = np.clip(v, -f8.TOP, f8.TOP)
    got = torch.from_numpy(v).float().to(torch.float8_e4m3fn).double().numpy()
    assert (np.abs(got - v) <= f8.half_step(v) * (1 + 1e-6)).all()


def test_scales_leave_out_what_is_not_finite():
    v = np.zeros((2, 300))
    v[0, 5], v[0, 6], v[0, 130], v[1, 299] = 3.0, np.inf, np.nan, -448.0
    assert np.array_equal(f8.scales(v), [[3.0 / 448, 2.0 ** -100, 2.0 ** -100], [2.0 ** -100, 2.0 ** -100, 1.0]])
    assert np.array_equal(f8.scales(v, 128), [[3.0 / 448, 2.0 ** -100, 1.0]])


def test_norm_gate_and_linear_by_hand():
    total, y = f8.rmsnorm(np.array([[3.0, 4.0]]), np.array([1.0, 2.0]), 0.0, np.array([[0.0, 0.0]]))
    assert np.allclose(total, [[3, 4]]) and np.allclose(y, np.array([[3, 8]]) / np.sqrt(12.5))
    assert np.allclose(f8.gated(np.array([2.0, 5.0, 1.0]), np.array([0.0, 1e4, -1e4])), [0.0, 5e4, 0.0])
    one, two = 0x38, 0x40
    y, size = f8.linear(np.array([[one, two]]), np.array([[0.5]]), np.array([[two, one | 128], [one, one]]), np.array([[3.0]]), np.array([1.0, 0.0]))
    assert np.array_equal(y, [[1.0, 4.5]]) and np.array_equal(size, [[7.0, 4.5]])
