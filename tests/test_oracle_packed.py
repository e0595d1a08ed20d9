"""Pins of the 4-bit oracle (CPU): hand values, borders, bounds of the error, and the performance cases' plain form against it."""
import numpy as np
import pytest
import torch

from oracle import packed as O


def _group(*x):
    g = np.zeros(32, np.float32)
    g[:len(x)] = x
    return g


def test_hand_values():
    """0 .. 15: step 1, base -16, every code its own number."""
    n, s, b = O.quantise_group(np.arange(32) % 16)
    assert s == 1 and b == -16 and np.array_equal(n, np.arange(32) % 16)
    assert np.array_equal(O.values(n, [s], [b]), np.arange(32) % 16)


def test_borders_go_up():
    """Half way between two codes is the upper one's; the next fp16 number below is the lower one's (x + 16 keeps it
    in float32: its last bit there is 2^-19, that of an fp16 number below 0.5 is 2^-12)."""
    x = _group(0, 15, 0.5, np.nextafter(np.float16(0.5), np.float16(0)), 14.5, 7.5, np.nextafter(np.float16(7.5), np.float16(0)))
    n, s, b = O.quantise_group(x)
    assert s == 1 and list(n[:7]) == [0, 15, 1, 0, 15, 8, 7]


def test_constant_and_far_groups():
    for c in (0.0, -3.25, 16384.0):
        n, s, b = O.quantise_group(np.full(32, c, np.float32))
        assert s == 0 and not n.any() and np.all(O.values(n, [s], [b]) == c)
    n, s, b = O.quantise_group(_group(1e6, -1e6))            # clamped to +-16384
    assert np.all(np.isfinite(O.values(n, [s], [b]))) and n[0] == 15 and n[1] == 0


def test_a_zero_base_has_no_sign():
    """-0, and what rounds to it: fp16's smallest number is 2^-24, a half of it or less is 0."""
    for c in (-0.0, -1e-8, -2.0**-25, -1e-30):
        n, s, b = O.quantise_group(np.full(32, c, np.float32))
        assert s == 0 and b == 0 and not np.signbit(b) and not n.any()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_non_finite_group(bad):
    n, s, b = O.quantise_group(_group(1, bad))
    assert s == 0 and np.isnan(b) and np.all(np.isnan(O.values(n, [s], [b])))


def error_bound(x, s, b):
    """Inside the codes' range an element lies within s/2 of its code's number; at the ends what s (15 steps of it)
    and b lost by rounding adds; then the value's own rounding.  fp16 rounds by 2^-11 of a number, 2^-25 at least."""
    def half(y):
        return np.maximum(2.0**-11 * np.abs(y), 2.0**-25)
    s, b = (np.repeat(np.asarray(y, np.float64), 32, -1) for y in (s, b))
    return s / 2 + 15 * half(s) + half(b) + half(np.abs(x) + s) + 2.0**-24 * np.abs(x)


@pytest.mark.parametrize("scale", [1e-8, 1e-5, 1e-3, 1.0, 300.0, 16384.0])
@pytest.mark.parametrize("offset", [0.0, 1.0, 100.0])
def test_error_is_half_a_step(scale, offset):
    x = np.random.default_rng(0).uniform(-1, 1, (50, 64)).astype(np.float32) * np.float32(scale) + np.float32(offset)
    x = np.clip(x, -16384, 16384).astype(np.float32)
    n, s, b = O.quantise(x)
    assert np.all(np.abs(O.values(n, s, b) - x) <= error_bound(x, s, b))


@pytest.mark.parametrize("d", [64, 128])
def test_rows_round_trip(d):
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 7, 3, d)).astype(np.float32)
    rows = O.pack(k, v)
    assert rows.shape == (7, 3, O.row_bytes(d)) and O.row_bytes(d) == 5 * d // 4
    for x, got in zip((k, v), O.unpack(rows)):
        assert np.array_equal(got, O.values(*O.quantise(x)))


def test_layout_of_a_row():
    """Width 8j + 2p in bits 4p of word j, width 8j + 2p + 1 in bits 16 + 4p."""
    k = np.tile(np.arange(32) % 16, 2).astype(np.float32)        # codes are the widths modulo 16
    w = O.pack(k, k).view("<u4")
    assert w[0] == 0x75316420 and w[1] == 0xFDB9ECA8 and w[8] == w[0]
    assert list(O.pack(k, k)[64:68].view("<f2")) == [1, -16]


@pytest.mark.parametrize("type", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
def test_plain_form_of_the_performance_cases(d, type):
    from perf import more_operators as M
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((40, 2, d), generator=g).to(type) * s for s in (3, 0.01))
    k[3, 0, 5], v[7, 1, 40] = float("nan"), float("inf")
    k[9], v[9] = 2.0, 0.0
    k[10, 0, 0] = 30000.0
    rows = M._pack(k, v).numpy()
    assert np.array_equal(rows, O.pack(k.float().numpy(), v.float().numpy()))
    for a, b in zip(M._values(torch.from_numpy(rows)), O.unpack(rows)):
        assert np.array_equal(a.double().numpy(), b, equal_nan=True)
