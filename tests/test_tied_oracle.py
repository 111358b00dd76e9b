"""Pins of the plain definitions around the tied weight: published test vectors, closed forms, library special cases,
and planted mistakes that must show."""
import numpy as np
import pytest
import torch

from oracle import tied_oracle as o


def test_generator_known_answers():
    # the three vectors published with the generator for ten rounds of the 4 x 32 form
    assert o.philox4x32((0, 0, 0, 0), (0, 0)) == (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)
    full = 0xffffffff
    assert o.philox4x32((full,) * 4, (full, full)) == (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)
    assert o.philox4x32((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == (
        0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)


def test_factor_follows_the_generator_and_keeps_the_expectation():
    seed, offset, p = 0x123456789ABCDEF, (5 << 32) + 9, 0.3
    k = o.drop_factor(40, 37, p, seed, offset, row_offset=3)
    cut = round(p * 65536)
    for r, c in ((0, 0), (0, 7), (11, 8), (39, 36), (20, 31)):
        word = o.philox4x32((c // 8, 3 + r, 9, 5), (seed & 0xffffffff, seed >> 32))[(c % 8) // 2]
        half = (word >> 16) if c % 2 else word & 0xffff
        assert k[r, c] == (65536 / (65536 - cut) if half >= cut else 0)
    big = o.drop_factor(1000, 1000, p, seed)
    assert abs(big.mean() - 1) < 5 * np.sqrt(p / (1 - p) / 1e6)          # five standard deviations
    assert o.drop_factor(3, 5, 0.0, 1).min() == 1 and o.drop_factor(3, 5, 1.0, 1).max() == 0
    assert not np.array_equal(o.drop_factor(8, 64, p, 1, 0), o.drop_factor(8, 64, p, 1, 1))
    assert np.array_equal(o.drop_factor(9, 64, p, 1)[4:], o.drop_factor(5, 64, p, 1, row_offset=4))


def test_codes_are_the_library_cast():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * s for s in (1e-3, 1e-2, 1, 100)]).clip(-448, 448).astype(np.float32)
    mids = o.e4m3_values()[:127]
    x = np.concatenate([x, ((mids[1:] + mids[:-1]) / 2).astype(np.float32), mids.astype(np.float32), -mids.astype(np.float32)])
    assert np.array_equal(o.to_e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(o.e4m3_values(), codes, equal_nan=True)


def test_scales_are_the_smallest_power_of_two_that_fits():
    for amax, want in ((448.0, 1.0), (449.0, 2.0), (1.75, 2.0 ** -8), (1.7501, 2.0 ** -7), (1.0, 2.0 ** -8), (0.0, 2.0 ** -108)):
        _, s = o.quantize(np.full((1, 3), amax), 1)
        assert s[0, 0] == want
    x = np.random.default_rng(1).standard_normal((130, 300))
    for rows in (1, 128):
        q, s = o.quantize(x, rows)
        assert s.shape == (3, 130 if rows == 1 else 2)
        assert np.abs(o.dequantize(q, s, rows) - x).max() <= np.abs(x).max() / 448 * 2 * 16    # half of the widest step


@pytest.mark.parametrize("seed", range(4))
def test_sampling_matches_a_direct_reading_on_small_rows(seed):
    """Rows of a few entries against filters written entry by entry with Python integers and fractions."""
    from fractions import Fraction
    rng = np.random.default_rng(seed)
    for _ in range(200):
        n = int(rng.integers(1, 9))
        x = np.round(rng.standard_normal(n) * 2, 1).astype(np.float32)                       # ties occur
        t, k, p, mp = float(rng.choice([0.5, 1.0, 2.0])), int(rng.integers(0, n + 2)), float(rng.choice([0.0, 0.25, 0.5, 0.75, 1.0])), float(rng.choice([0.0, 0.125, 0.5]))
        u = float(rng.integers(0, 1 << 24)) / (1 << 24)
        token, prob, _ = o.sample(x, u, t, k, p, mp)
        z = (x - x.max()) * np.float32(1 / np.float32(t))
        w = [int(np.rint(np.exp(np.float64(v)) * 2 ** 31)) for v in z]
        keep = sorted(range(n), key=lambda i: (-x[i], i))[:k if k > 0 else n]
        if p < 1:
            total, run, first = sum(w[i] for i in keep), 0, []
            for i in keep:
                if run < max(1, int(Fraction(p) * total)):
                    first.append(i)
                run += w[i]
            keep = first
        keep = sorted(i for i in keep if np.exp(np.float64(z[i])) >= mp)
        at, run = int(Fraction(u) * sum(w[i] for i in keep)), 0
        for i in keep:
            run += w[i]
            if run > at:
                break
        assert token == i and prob == pytest.approx(w[i] / sum(w[j] for j in keep))


def test_sampling_special_rows():
    inf = np.inf
    assert o.sample(np.array([-inf, np.nan, -inf]), 0.5)[:2] == (-1, 0.0)
    assert o.sample(np.array([-inf, 3.0, -inf]), 0.99)[0] == 1
    assert o.sample(np.array([1.0, inf, 0.0, inf]), 0.6)[0] == 3
    assert o.sample(np.array([1.0, 2.0, 2.0]), 0.9, temperature=0.0)[0] == 1
    assert o.sample(np.array([2.0, 1.0, 2.0, 2.0]), 0.999, top_k=2)[0] == 2
    low = np.finfo(np.float32).min
    assert o.sample(np.array([low, 0.0, low]), 0.999)[0] == 1
    assert o.sample(np.array([low, low]), 0.75)[0] == 1


def test_planted_mistakes_show():
    k = o.drop_factor(64, 64, 0.5, 77)
    assert not np.array_equal(k, np.roll(k, 1, 1)) and not np.array_equal(k, o.drop_factor(64, 64, 0.5, 78))
    x = np.random.default_rng(2).standard_normal((4, 200))
    q, s = o.quantize(x, 1)
    wrong = s[::-1]                                                                             # scales of the other block
    assert np.abs(o.dequantize(q, wrong, 1) - x).max() > np.abs(o.dequantize(q, s, 1) - x).max() or np.array_equal(s, wrong)
    y = np.array([0.0, 1.0, 1.0, -1.0], np.float32)
    assert o.sample(y, 0.0, top_k=1)[0] == 1                                                   # last among equals would be 2
    assert o.sample(y, 0.0)[0] == 0                                                             # descending order would give 1
