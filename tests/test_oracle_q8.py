"""Pins of the 8-bit cache's oracle: the types against torch's conversions and
known values, the scale rule at its borders, hand-made partial writes, the
rotation against complex numbers."""
import math

import numpy as np
import pytest
import torch

from oracle import q8
from q8_util import DTYPES, Pool, bf16


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_codes_are_torchs(fmt):
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(DTYPES[fmt]).double().numpy()
    assert np.array_equal(q8.decode_table(fmt), want, equal_nan=True)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_rounding_is_torchs(fmt):
    rng = np.random.default_rng(1)
    top = q8.FORMATS[fmt][3]
    vals = q8.decode_table(fmt)[:128]
    vals = vals[np.isfinite(vals)]
    mids = (vals[1:] + vals[:-1]) / 2                       # every tie
    x = np.concatenate([vals, mids, np.nextafter(mids, 0), np.nextafter(mids, 1e9),
                        rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 8, 4000)])
    x = np.concatenate([x, -x]).astype(np.float32).astype(np.float64)
    x = np.clip(x, -top, top)
    want = torch.from_numpy(x).float().to(DTYPES[fmt]).view(torch.uint8).numpy()
    assert np.array_equal(q8.encode(x, fmt), want)


def test_known_values():
    assert q8.decode_table("e4m3")[0x7E] == 448 and q8.decode_table("e4m3")[1] == 2.0 ** -9
    assert q8.decode_table("e5m2")[0x7B] == 57344 and q8.decode_table("e5m2")[1] == 2.0 ** -16
    assert q8.encode([math.inf, -math.inf, math.nan], "e4m3").tolist() == [0x7E, 0xFE, 0x7F]
    assert q8.encode([17.0, 19.0], "e4m3").tolist() == [0x58, 0x5A]      # ties between 16, 18 and 20: even codes


@pytest.mark.parametrize("fmt,top", [("e4m3", 448.0), ("e5m2", 57344.0)])
def test_scale_borders(fmt, top):
    assert q8.page_scale(top, fmt) == 1.0
    assert q8.page_scale(np.nextafter(top, 1e9), fmt) == 2.0
    assert q8.page_scale(top / 2, fmt) == 0.5
    assert q8.page_scale(0.0, fmt) == 2.0 ** -100
    assert q8.page_scale(3.3895313892515355e38, fmt) == (2.0 ** 120 if fmt == "e4m3" else 2.0 ** 113)


def test_partial_writes_by_hand():
    """One head: 16 ones, then a token of 900 over slot 3 with the rest kept
    (scale 2^-8 -> 4: ones become 0.25, exact), then an append."""
    rng = np.random.default_rng(0)
    pool = Pool(rng, [20], 1, 64, "e4m3")
    one = torch.ones(16, 1, 64, dtype=torch.bfloat16)
    pool.set(q8.kv_write_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, [0], [16], one, one, "e4m3"))
    pid = pool.table[0, 0]
    assert pool.ks[pid, 0] == 2.0 ** -8 and pool.vs[pid, 0] == 2.0 ** -8          # 1 / 2^-8 = 256 <= 448 < 512
    big = torch.full((1, 1, 64), 900.0, dtype=torch.bfloat16)                      # 900 = 2^9 * 1.7578: above 448 * 2
    pool.set(q8.kv_write_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, [3], [1], big, big, "e4m3", kv_lens=[16]))
    assert pool.ks[pid, 0] == 4.0
    K, V = pool.values()
    want = np.ones(16)
    want[3] = 896.0                                                                # 225 between 224 and 240
    assert np.array_equal(K[pid, 0, :, 0].numpy(), want) and np.array_equal(V[pid, 0, 5].numpy(), want)
    # without kv_lens the tokens behind slot 3 are not kept: their bytes stay, their scale is gone
    k2, _, ks2, _ = q8.kv_write_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, [3], [1], one[:1], one[:1], "e4m3")
    assert ks2[pid, 0] == 4.0 and np.array_equal(k2[pid, 0, 4:], pool.k[pid, 0, 4:].numpy())
    k3, _, ks3, _ = q8.kv_write_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, [0], [1], one[:1], one[:1], "e4m3")
    assert ks3[pid, 0] == 2.0 ** -8


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_round_trip_error(fmt):
    """Written and read back, a normal value is off by half a step at most."""
    rng = np.random.default_rng(2)
    lens = [37, 0, 5]
    pool = Pool(rng, lens, 2, 64, fmt)
    k, v = bf16(rng, 42, 2, 64), bf16(rng, 42, 2, 64)
    pool.set(q8.kv_write_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, [0, 0, 0], lens, k, v, fmt))
    K, V = q8.kv_read_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, [0, 0, 0], lens, fmt)
    half = torch.finfo(DTYPES[fmt]).eps / 2
    floor = {"e4m3": 2.0 ** -10, "e5m2": 2.0 ** -17}[fmt] * float(max(pool.ks[pool.ks == pool.ks].max(), 0))
    for got, x in ((K, k), (V, v)):
        x = x.double().numpy()
        assert np.all(np.abs(got - x) <= half * np.abs(x) + floor)


def test_rotary_is_a_complex_product():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 2, 32))
    turns = [int(2.0 ** 64 * 10000.0 ** (-i / 8) / (2 * math.pi)) for i in range(8)]
    pos = np.array([0, 1, 7, 4095, 100000])
    for inter in (False, True):
        y = q8.rotary(x, pos, turns, 1.25, inter)
        a, b = (x[..., 0:16:2], x[..., 1:16:2]) if inter else (x[..., :8], x[..., 8:16])
        ang = pos[:, None] * np.array([10000.0 ** (-i / 8) for i in range(8)])
        z = (a + 1j * b) * 1.25 * np.exp(1j * ang)[:, None]
        ya, yb = (y[..., 0:16:2], y[..., 1:16:2]) if inter else (y[..., :8], y[..., 8:16])
        assert np.allclose(ya, z.real, atol=1e-9) and np.allclose(yb, z.imag, atol=1e-9)
        assert np.array_equal(y[..., 16:], x[..., 16:])
        assert np.allclose(q8.rotary(y, pos, turns, 1 / 1.25, inter, inverse=True), x, atol=1e-12)
