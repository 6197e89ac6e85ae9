"""The quantising write and the read-back against the 64-bit oracle, bit for
bit: codes and scales are exact, so nothing here has a tolerance."""
import numpy as np
import pytest
import torch

from oracle import q8
from q8_util import Pool, bf16, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _write(gpu, pool, start, lens, k, v, *, kv_lens=None, flags=None, block=None, rows=None):
    """One call on the device and by the oracle; compares the whole pools."""
    args = pool.on(DEV)
    rows = k.shape[0] if rows is None else rows
    gpu.kv_write_q8(*args, i32(start, DEV), i32(lens, DEV), k.to(DEV), v.to(DEV), max_len=max(max(lens), 1),
                    kv_lens=None if kv_lens is None else i32(kv_lens, DEV),
                    block_flags=None if flags is None else torch.as_tensor(flags, dtype=torch.uint8).to(DEV),
                    block_size=block)
    torch.cuda.synchronize()
    want = q8.kv_write_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, start, lens, k, v, pool.fmt, kv_lens, flags, block)
    got = [args[0].cpu().view(torch.uint8), args[1].cpu().view(torch.uint8), args[2].cpu(), args[3].cpu()]
    table = q8.decode_table(pool.fmt)
    for g, w, name in zip(got, want, ("K", "V", "K scales", "V scales")):
        g = g.numpy()
        if g.dtype == np.uint8:       # (a NaN code's sign is not specified)
            same = (g == w) | (np.isnan(table[g]) & np.isnan(table[w]))
        else:
            same = (g == w) | (np.isnan(g) & np.isnan(w))
        assert same.all(), f"{name}: {int((~same).sum())} of {same.size} differ, first at {np.argwhere(~same)[0]}"
    pool.set([np.where(np.isnan(table[w]), g.numpy(), w) if w.dtype == np.uint8 else w for g, w in zip(got, want)])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("hkv,d", [(1, 64), (3, 64), (2, 128), (5, 128)])
def test_ragged_prompts_then_tokens(gpu, fmt, hkv, d):
    """Prompts of ragged lengths, then single tokens behind them whose size
    grows, so that kept slots are requantised several times."""
    rng = np.random.default_rng(hkv * d)
    lens = [1, 15, 16, 0, 17, 33, 130]
    pool = Pool(rng, [n + 6 for n in lens], hkv, d, fmt)
    n = sum(lens)
    _write(gpu, pool, [0] * len(lens), lens, bf16(rng, n, hkv, d), bf16(rng, n, hkv, d))
    held = list(lens)
    for step in range(5):
        one = [1] * len(lens)
        _write(gpu, pool, held, one, bf16(rng, len(lens), hkv, d, scale=3.0 ** step), bf16(rng, len(lens), hkv, d))
        held = [h + 1 for h in held]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [1, 7, 16, 32])
def test_blocks_written_over(gpu, fmt, d, block):
    """Flagged blocks in the middle of sequences, from any slot, with tokens
    behind them on the same pages; one row of flags empty."""
    rng = np.random.default_rng(block)
    start, lens, held = [3, 16, 40, 0], [64, 50, 33, 20], [100, 66, 73, 21]
    pool = Pool(rng, held, 2, d, fmt).fill(rng, held, sigma=0.5)
    nblk = -(-64 // block)
    flags = rng.integers(0, 2, (4, nblk))
    flags[2] = 0
    _write(gpu, pool, start, lens, bf16(rng, sum(lens), 2, d, scale=20.0), bf16(rng, sum(lens), 2, d, scale=20.0),
           kv_lens=held, flags=flags.tolist(), block=block)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_extreme_values(gpu, fmt):
    """Zeros, subnormals, the largest bf16, infinities and NaN, a page of each,
    and mixed with ordinary values."""
    rng = np.random.default_rng(7)
    x = bf16(rng, 16 * 10, 2, 64)
    pages = x.view(10, 16, 2, 64)
    pages[0] = 0
    pages[1] = 2.0 ** -133                       # a bf16 subnormal
    pages[2] = 3.3895313892515355e38
    pages[3, 5] = float("inf")
    pages[3, 6, :, ::3] = float("-inf")
    pages[4, :, 0] = float("nan")
    pages[5, 2, 1, 7] = float("nan")
    pages[6] = float("inf")
    pages[7, :, :, :] *= 2.0 ** -120
    pages[8, 0, 0, 0] = 448 * 2.0 ** 5           # the border: the largest value itself
    pages[9, 0, 0, 0] = 450 * 2.0 ** 5           # and just above
    pool = Pool(rng, [160], 2, 64, fmt)
    _write(gpu, pool, [0], [160], x, x.flip(0).contiguous())
    # infinities next to kept tokens of a larger scale
    y = bf16(rng, 1, 2, 64)
    y[0, 0, 0] = float("inf")
    _write(gpu, pool, [47], [1], y, y, kv_lens=[160])


def test_tokens_off_the_table_are_not_written(gpu):
    """A table row that ends early, page ids out of the pool, rows beyond the
    input: the other tokens are written, nothing else changes."""
    rng = np.random.default_rng(9)
    pool = Pool(rng, [64, 64, 64], 2, 128, "e4m3")
    pool.table[0, 1] = -1
    pool.table[1, 2] = pool.k.shape[0]
    lens = [64, 64, 90]                       # the last one runs off its row of 4 pages
    n = sum(lens)
    _write(gpu, pool, [0, 0, 0], lens, bf16(rng, n, 2, 128), bf16(rng, n, 2, 128))


def test_zero_lengths_do_nothing(gpu):
    rng = np.random.default_rng(10)
    pool = Pool(rng, [20, 20], 2, 64, "e4m3").fill(rng, [20, 20])
    _write(gpu, pool, [20, 3], [0, 0], bf16(rng, 1, 2, 64), bf16(rng, 1, 2, 64))


def test_a_foreign_scale_is_kept_under_appends(gpu):
    """A pool whose scales are no powers of two: a larger one stays, the kept
    bytes with it; new values are rounded at that scale."""
    rng = np.random.default_rng(11)
    pool = Pool(rng, [8], 1, 64, "e4m3").fill(rng, [4], sigma=4.0)
    pid = pool.table[0, 0]
    pool.ks[pid] = 0.3
    kept = pool.k[pid, 0, :4].clone()
    args = pool.on(DEV)
    one = torch.full((1, 1, 64), 0.9, dtype=torch.bfloat16)
    gpu.kv_write_q8(*args, i32([4], DEV), i32([1], DEV), one.to(DEV), one.to(DEV), max_len=1)
    torch.cuda.synchronize()
    assert float(args[2][pid, 0]) == np.float32(0.3)
    assert torch.equal(args[0][pid, 0, :4].cpu().view(torch.uint8), kept)
    # 0.9 (bf16) / 0.3 = 3 within fp32 rounding, far from a tie of e4m3
    assert torch.equal(args[0][pid, 0, 4].float().cpu(), torch.full((64,), 3.0))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("hkv,d", [(1, 128), (3, 64), (4, 128)])
def test_read_back(gpu, fmt, hkv, d):
    """Ranges from any slot; rows behind the last sequence stay as they were;
    tokens off the table read as zeros."""
    rng = np.random.default_rng(hkv + d)
    held = [70, 16, 5, 300]
    pool = Pool(rng, held, hkv, d, fmt).fill(rng, held)
    pool.table[2, 0] = pool.k.shape[0] + 3
    start, lens = [3, 0, 1, 150], [60, 16, 4, 150]
    n = sum(lens)
    out = [torch.full((n + 3, hkv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    k, v = gpu.kv_read_q8(*pool.on(DEV), i32(start, DEV), i32(lens, DEV), max_len=150, out=out)
    torch.cuda.synchronize()
    K, V = q8.kv_read_q8(pool.k, pool.v, pool.ks, pool.vs, pool.table, start, lens, fmt)
    for got, want in ((k, K), (v, V)):
        assert np.array_equal(got[:n].cpu().double().numpy(), want)          # exact: powers of two
        assert bool((got[n:] == 7).all())
    # sizes read from the device
    k2, v2 = gpu.kv_read_q8(*pool.on(DEV), i32(start, DEV), i32(lens, DEV))
    assert torch.equal(k2, k[:n]) and torch.equal(v2, v[:n])


def test_read_rounds_foreign_scales_to_bf16(gpu):
    rng = np.random.default_rng(12)
    pool = Pool(rng, [16], 1, 64, "e4m3").fill(rng, [16])
    pool.ks[pool.table[0, 0]] = 0.37
    k, _ = gpu.kv_read_q8(*pool.on(DEV), i32([0], DEV), i32([16], DEV))
    want = (pool.on("cpu")[0][pool.table[0, 0], 0].float() * torch.tensor(0.37)).to(torch.bfloat16)
    assert torch.equal(k[:, 0].cpu(), want)


def test_positions_past_32_bits_of_bytes(gpu):
    """A pool of more than 2^31 bytes: its last pages are written and read."""
    hkv, d = 8, 128
    pages = (1 << 31) // (hkv * 16 * d) + 3
    rng = np.random.default_rng(13)
    args = [torch.zeros(pages, hkv, 16, d, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn),
            torch.zeros(pages, hkv, d, 16, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn),
            torch.ones(pages, hkv, device=DEV), torch.ones(pages, hkv, device=DEV),
            i32([[pages - 1, 0, pages - 2]], DEV)]
    k, v = bf16(rng, 40, hkv, d).to(DEV), bf16(rng, 40, hkv, d).to(DEV)
    gpu.kv_write_q8(*args, i32([2], DEV), i32([40], DEV), k, v, max_len=40)
    a, b = gpu.kv_read_q8(*args, i32([2], DEV), i32([40], DEV), max_len=40, total=40)
    torch.cuda.synchronize()
    for got, x in ((a, k), (b, v)):
        err = (got.double() - x.double()).abs()
        # half a step of e4m3, or of its subnormals: 2^-10 of the page's scale.  That is 1 on the first
        # page, whose slots 0 and 1 are kept at the pool's scale of 1 (max(s, 1) = 1, as values below
        # 448 give s <= 1), and s <= 2^-6 (8 / 448 < 2^-5) on the others, so 2^-10 covers both
        assert bool((err <= x.double().abs() * 2.0 ** -4 + 2.0 ** -10).all())
    assert float(args[0][1].float().abs().max()) == 0
