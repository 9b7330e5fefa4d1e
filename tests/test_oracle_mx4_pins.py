"""CPU pins of oracle/mx4_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo


def case(seed=0, S=3, D=64, sections=(8, 12)):
    r = np.random.default_rng(seed)
    n = sum(sections)
    return r.standard_normal((2, 3, S, D)), r.standard_normal(D), r.integers(0, 500, (2, S, len(sections))), 100.0 ** (-np.arange(n) / n), sections


def test_norm_is_torchs():
    x, w, pos, inv, sections = case()
    got = mo.norm_rotary(x, w, 0 * pos, inv, sections, eps=1e-5)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(w), 1e-5).numpy()
    assert np.allclose(got, want, rtol=1e-13, atol=0)
    assert np.array_equal(mo.norm_rotary(x, None, 0 * pos, inv, sections, eps=1e-5, norm=False), x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    x, w, pos, inv, sections = case()
    r = np.random.default_rng(1)
    dy, u, uw = r.standard_normal(x.shape), r.standard_normal(x.shape), r.standard_normal(64)
    f = lambda x, w: np.sum(dy * mo.norm_rotary(x, w, pos, inv, sections, eps=1e-3, interleaved=interleaved))
    dx, dw, dx_size, dw_size = mo.norm_rotary_gradient(x, w, dy, pos, inv, sections, eps=1e-3, interleaved=interleaved)
    h = 1e-5                                       # error of the quotient: h^2 times a third derivative, roundings 1e-16 / h
    assert abs((f(x + h * u, w) - f(x - h * u, w)) / (2 * h) - np.sum(dx * u)) <= 1e-7
    assert abs((f(x, w + h * uw) - f(x, w - h * uw)) / (2 * h) - np.sum(dw * uw)) <= 1e-7
    assert (np.abs(dx) <= dx_size * (1 + 1e-12)).all() and (np.abs(dw) <= dw_size * (1 + 1e-12)).all()


def test_what_the_format_has_is_held():
    for e in (1, 100, 127, 252):
        row = np.concatenate([mo.VALUES, -mo.VALUES, np.full(16, 6.0)]) * 2.0 ** (e - 127)
        codes, scales, _ = mo.hold(row)
        assert scales.tolist() == [e] and np.array_equal(mo.values(codes, scales), row)
        assert codes[:16].tolist() == list(range(16))


def test_ties_go_to_the_even_code():
    t = np.zeros(32)
    t[:8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]
    codes, scales, gap = mo.hold(t)
    assert scales.tolist() == [127] and codes[:8].tolist() == [0, 2, 2, 4, 4, 6, 6, 7] and (gap[:7] == 0).all()


def test_scale_is_the_smallest_that_the_largest_is_below_seven_of():
    for most, e, code in ((6.0, 127, 7), (6.99, 127, 7), (7.0, 128, 6), (3.5, 127 - 1 + 1, None), (3.49, 126, 7), (12.0, 128, 7)):
        x = np.zeros(32)
        x[5] = -most
        codes, scales, _ = mo.hold(x)
        assert scales.tolist() == [e], most
        if code is not None:
            assert codes[5] == 8 + code


def test_errors_are_half_a_step():
    x = np.random.default_rng(3).standard_normal((50, 64)) * np.exp(np.random.default_rng(4).standard_normal((50, 1)) * 20)
    codes, scales, _ = mo.hold(x)
    unit = np.repeat(2.0 ** (scales - 127.0), 32, axis=-1)
    step = np.where(np.abs(x) < 2 * unit, 0.5, np.where(np.abs(x) < 4 * unit, 1.0, 2.0)) * unit
    assert (np.abs(mo.values(codes, scales) - x) <= step / 2).all()


def test_what_is_not_finite():
    x = np.ones((4, 32))
    x[0, 3], x[1, 4], x[2, 5], x[3, 6] = np.inf, -np.inf, np.nan, -np.nan
    codes, scales, _ = mo.hold(x)
    v = mo.values(codes, scales)
    assert v[0, 3] == 6 * 2.0 ** 125 and v[1, 4] == -6 * 2.0 ** 125 and v[2, 5] == v[3, 6] == 0 and np.isfinite(v).all()
    assert scales[:, 0].tolist() == [252, 252, 125, 125] and (v[2, :5] == 1).all()
    zero, e, _ = mo.hold(np.zeros(32))
    assert not zero.any() and e.tolist() == [1]


@pytest.mark.parametrize("D,page", [(64, 8), (128, 16)])
def test_pages_round_trip(D, page):
    r = np.random.default_rng(5)
    codes, scales = r.integers(0, 16, (3, 2, page, D)).astype(np.uint8), r.integers(1, 253, (3, 2, page, D // 32)).astype(np.uint8)
    cache = mo.pages_of(codes, scales)
    back = mo.rows_of(cache, page, D)
    assert np.array_equal(back[0], codes) and np.array_equal(back[1], scales)
    assert cache[1, 1, 2 * (D // 2) + 3] == codes[1, 1, 2, 6] + 16 * codes[1, 1, 2, 7] and cache[2, 0, page * D // 2 + page + 4] == scales[2, 0, 4, 1]
    assert mo.dense(cache, page, D).shape == (3, page, 2, D)
