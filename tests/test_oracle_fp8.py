"""Pins of the 8-bit oracle: its tables and encoder against torch's 8-bit
types, the block rule against hand-worked blocks, the mask words against the
generator's own pins."""

import numpy as np
import pytest
import torch

from oracle import fp8, philox

TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_tables_and_encoder(fmt):
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(TYPES[fmt]).double().numpy()
    fin = np.isfinite(want)
    got = fp8.decode(codes, fmt)
    assert np.array_equal(got[fin], want[fin]) and np.isnan(got[~fin]).all()
    assert fp8.values(fmt)[-1] == fp8.TOP[fmt]
    t = fp8.values(fmt)
    mid = (t[1:] + t[:-1]) / 2
    probe = np.concatenate([t, mid, np.nextafter(mid, 0), np.nextafter(mid, np.inf)]).astype(np.float64)
    probe = np.concatenate([probe, -probe, np.random.default_rng(0).standard_normal(10000) * 10])
    probe = probe[np.abs(probe) <= t[-1]]
    # torch rounds through binary32; keep what binary32 holds
    probe = probe.astype(np.float32)
    want = torch.from_numpy(probe).to(TYPES[fmt]).view(torch.uint8).numpy()
    assert np.array_equal(fp8.encode(probe.astype(np.float64), fmt), want)
    assert fp8.encode(np.array([1e9, -1e9, np.nan]), fmt).tolist() == [t.size - 1, 0x80 | (t.size - 1), 0xFF]


def test_block_rule():
    x = np.zeros((1, 300))
    x[0, 3], x[0, 5], x[0, 7] = 28.0, -14.0, 0.8125        # block 0: a = 28 = 448 / 16
    x[0, 128:256] = 0.0                                     # block 1: nothing
    x[0, 256] = 3.0                                         # block 2 (short): a = 3
    q, s = fp8.quantize_rows(x, "e4m3", "f32")
    assert q.shape == (1, 384) and s.shape == (3, 1)
    assert s[0, 0] == 1 / 16 and s[1, 0] == 1.0 and s[2, 0] == float(np.float32(3.0) / np.float32(448.0))
    d = fp8.decode(q, "e4m3")[0]
    assert d[3] == 448 and d[5] == -224 and d[7] == 13 and d[256] == 448 and not d[300:].any()
    q, s = fp8.quantize_rows(x, "e4m3", "e8m0")
    # 28 / 448 = 2^-4 exactly; 3 / 448 lies between 2^-8 and 2^-7
    assert s[0, 0] == 2.0 ** -4 and s[1, 0] == 1.0 and s[2, 0] == 2.0 ** -7
    assert fp8.decode(q, "e4m3")[0, 256] == 384
    x[0, 3] = np.inf
    x[0, 4] = np.nan
    q, s = fp8.quantize_rows(x, "e5m2", "e8m0")
    d = fp8.decode(q, "e5m2")[0]
    assert np.isnan(d[3]) and np.isnan(d[4]) and s[0, 0] == 2.0 ** -12 and d[5] == -14 * 4096
    q, s = fp8.quantize_tiles(np.full((130, 2), 7.0), "e8m0")
    assert s.shape == (2, 1) and s[0, 0] == 2.0 ** -6 and (fp8.decode(q, "e4m3")[:, :2] == 448).all()


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_relative_error(fmt, scale):
    """Values in the format's normal range come back within half a step."""
    x = np.random.default_rng(1).standard_normal((5, 256))
    q, s = fp8.quantize_rows(x, fmt, scale)
    back = fp8.decoded_rows(q, s, fmt)
    held = np.repeat(s.T, 128, 1)
    least = 2.0 ** (-6 if fmt == "e4m3" else -14)
    big = np.abs(x) >= least * held
    step = 2.0 ** -4 if fmt == "e4m3" else 2.0 ** -3
    assert (np.abs(back - x)[big] <= step * (1 + 2.0 ** -20) * np.abs(x)[big]).all()


def test_dropout_words():
    w = philox.philox4x32_10(np.array([[5, 0, 7, 1]], np.uint64), (11, 13))[0]
    got = fp8.dropout_words(11 + (13 << 32), 7, np.arange(40, 48))
    want = [v for x in w for v in (int(x) & 0xFFFF, int(x) >> 16)]
    assert got.tolist() == want
    big = fp8.dropout_words(1, 2, np.array([8 * (2 ** 32 + 3) + 5]))
    assert big[0] == int(philox.philox4x32_10(np.array([[3, 1, 2, 1]], np.uint64), (1, 0))[0][2]) >> 16
