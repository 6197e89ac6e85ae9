"""Window attention over an 8-bit cache against the 64-bit oracle on the pool's
exact values.

Tolerance, for every output value o = sum p v / sum p: o is rounded to bf16
(2^-8 |o|); each probability is rounded to bf16 before P.V (2^-8 of sum p |v| /
sum p =: A); exponents are fp32 numbers below 2^8 in magnitude, so exp2's
argument is off by 2^-16 and p by 2^-16 ln 2, and the fp32 sums of the scores
(q exact, keys exact) by 2^-23 of sum |q k|, at most 2^-23 * 2^9 here: together
under 2^-12 A.  So |error| <= 2^-8 |o| + (2^-8 + 2^-12) A, A >= |o|."""
import numpy as np
import pytest
import torch

import oracle
from q8_util import Pool, bf16, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    def __init__(self, seed, prefix, window, block, hq, hkv, d, fmt="e4m3", sigma_q=1.0, sigma_kv=1.0, width=None):
        rng = np.random.default_rng(seed)
        self.prefix, self.window, self.block = list(prefix), list(window), block
        held = [p + w for p, w in zip(prefix, window)]
        self.pool = Pool(rng, held, hkv, d, fmt, width=width).fill(rng, held, sigma=sigma_kv)
        self.q = bf16(rng, int(sum(window)), hq, d, scale=sigma_q)

    def run(self, gpu, mode="bidir", q=None, args=None, **kw):
        kw.setdefault("max_prefix_len", max(self.prefix, default=0))
        kw.setdefault("max_window_len", max(self.window, default=0))
        return gpu.window_attention_q8(self.q.to(DEV) if q is None else q, *(args or self.pool.on(DEV)),
                                       i32(self.prefix, DEV), i32(self.window, DEV), self.block, mask_mode=mode, **kw)

    def want(self, mode="bidir", scale=None):
        """Output, and A of the tolerance (kept while the inputs stay the same)."""
        key = (mode, scale, self.q.view(torch.int16).numpy().tobytes(), self.pool.k.numpy().tobytes())
        if getattr(self, "_key", None) != key:
            self._key, self._want = key, self._compute(mode, scale)
        return self._want

    def _compute(self, mode, scale):
        k, v = self.pool.values()
        m = oracle.MASK_BIDIR if mode == "bidir" else oracle.MASK_BLOCK_CAUSAL
        rest = self.pool.table, self.prefix, self.window, self.block, m, scale
        return (oracle.window_attention(self.q, k, v, *rest), oracle.window_attention(self.q, k, v.abs(), *rest))

    def check(self, out, mode="bidir", scale=None, what=""):
        want, size = self.want(mode, scale)
        got = out.cpu().double().numpy()
        err = np.abs(got - want)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * size
        assert np.isfinite(got).all(), f"{what}: {int((~np.isfinite(got)).sum())} values are not finite"
        assert (err <= tol).all(), f"{what}: max error {err.max():.3e}, {float((err / tol).max()):.2f} of the tolerance"


@pytest.mark.parametrize("keys", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 128, 129, 511, 513, 1100])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_key_counts(gpu, keys, d, fmt):
    """Sequences that end at and around pages and tiles; NaN codes behind."""
    c = Case(keys, [keys - 1, max(keys - 2, 0), 0], [1, 1, 1], 1, 8, 2, d, fmt)
    c.check(c.run(gpu), what=f"{keys} keys")
    w = min(keys, 16)
    for hq in (4, 8, 16, 32):                # units of 32 to 256 rows
        c = Case(keys, [keys - w, 3], [w] * 2, w, hq, 2 if hq < 32 else 1, d, fmt)
        for split in (0, 1 << 20):
            c.check(c.run(gpu, kv_split_tokens=split), what=f"{keys} keys, {hq} heads, split {split}")


@pytest.mark.parametrize("group,window,block", [(1, 1, 1), (1, 33, 33), (3, 11, 11), (4, 8, 4), (4, 9, 3), (4, 16, 16),
                                                (4, 17, 17), (4, 32, 16), (3, 43, 43), (4, 64, 32), (8, 48, 16),
                                                (4, 128, 32), (16, 8, 8), (1, 300, 50), (8, 65, 13)])
@pytest.mark.parametrize("d", [64, 128])
def test_row_counts(gpu, group, window, block, d):
    """1 to 520 packed rows: part of a wave's rows, of a workgroup's, several; in
    the small units of short calls, and in the units that go by the rows (whole,
    and cut)."""
    c = Case(group * window, [77, 600, 0], [window] * 3, block, 2 * group, 2, d)
    for mode in ("bidir", "block_causal"):     # (units by split)
        for split in (0, 1 << 20, 64):
            c.check(c.run(gpu, mode, kv_split_tokens=split), mode, what=f"{mode}, split {split}")


@pytest.mark.parametrize("split", [64, 128, 320, 1024])
@pytest.mark.parametrize("mode", ["bidir", "block_causal"])
@pytest.mark.parametrize("group,window", [(4, 1), (4, 12), (4, 32), (4, 72), (8, 72)])
def test_split_sequences(gpu, split, mode, group, window):
    """Units cut between many workgroups, ragged: several borders in one unit,
    several units in one share, windows of nothing between them."""
    prefix, win = [1500, 3, 0, 700, 64, 2049], [window, window, 0, window, 0, window]
    c = Case(split, prefix, win, window // 4 if window > 1 else 1, 2 * group, 2, 128)
    c.check(c.run(gpu, mode, kv_split_tokens=split), mode, what=f"split {split}")


def test_ragged_batch_of_many(gpu):
    """150 sequences (several rounds of the 64-lane scans), windows of 0 to 5
    blocks, bounds far above the lengths."""
    rng = np.random.default_rng(1)
    n = 150
    prefix, win = rng.integers(0, 400, n), 4 * rng.integers(0, 6, n)
    c = Case(2, prefix.tolist(), win.tolist(), 4, 4, 1, 64)
    for mode in ("bidir", "block_causal"):
        c.check(c.run(gpu, mode, max_prefix_len=100000, max_window_len=64), mode, what=mode)
    c.check(c.run(gpu, kv_split_tokens=64), what="forced splits")


@pytest.mark.parametrize("window", [1, 16, 64])
def test_sharp_rising_and_flat_scores(gpu, window):
    """Scores of hundreds, keys whose scores rise along the sequence (the
    reference maximum is raised again and again), equal scores, a zero q."""
    c = Case(3, [900], [window], window, 4, 1, 128, sigma_q=20.0, sigma_kv=3.0)
    for split in (0, 1 << 20, 128):
        c.check(c.run(gpu, kv_split_tokens=split), what=f"sharp, split {split}")
    rng = np.random.default_rng(4)
    c = Case(4, [900], [window], window, 4, 1, 128)
    n = 900 + window
    k = torch.ones(n, 1, 128, dtype=torch.bfloat16) * (torch.arange(n) / 64).floor().view(-1, 1, 1).to(torch.bfloat16)
    v = bf16(rng, n, 1, 128)
    from oracle import q8
    c.pool.set(q8.kv_write_q8(c.pool.k, c.pool.v, c.pool.ks, c.pool.vs, c.pool.table, [0], [n], k, v, "e4m3"))
    c.q = torch.full_like(c.q, 0.25)
    c.q[0, 1] = 0
    c.q[0, 2] = -0.25
    for split in (0, 1 << 20, 128):
        c.check(c.run(gpu, kv_split_tokens=split), what=f"rising, split {split}")


def test_scales_far_apart(gpu):
    """Pages whose scales differ by 2^40, rows of q by 2^60, zero pages."""
    rng = np.random.default_rng(5)
    c = Case(5, [300], [4], 4, 4, 1, 128)
    n = 304
    from oracle import q8
    k, v = bf16(rng, n, 1, 128), bf16(rng, n, 1, 128)
    for page in range(0, 19):
        k[16 * page:16 * page + 16] *= 2.0 ** -(2 * page)
        v[16 * page:16 * page + 16] *= 2.0 ** (20 - 2 * page)
    k[32:48] = 0
    v[64:80] = 0
    c.pool.set(q8.kv_write_q8(c.pool.k, c.pool.v, c.pool.ks, c.pool.vs, c.pool.table, [0], [n], k, v, "e4m3"))
    c.q[1] *= 2.0 ** -60
    c.q[2, :, ::2] *= 2.0 ** -9            # values at both ends of a row's range
    c.check(c.run(gpu), what="scales")
    c.check(c.run(gpu, softmax_scale=0.5), scale=0.5, what="softmax scale")
    for rows in (64, 256):                    # the kernels of larger units
        c.q = c.q[:, :1].expand(4, rows // 4, 128).contiguous()
        c.check(c.run(gpu, kv_split_tokens=1 << 20), what=f"scales, {rows} rows")


@pytest.mark.parametrize("heads", [2, 4, 8, 16])
def test_block_flags_and_gate(gpu, heads):
    """Only flagged blocks' rows are written; nothing is when the gate is 0.  (32
    to 256 rows per KV head)"""
    c = Case(6, [100, 2000], [32, 32], 8, heads, 2, 128)
    flags = torch.tensor([[1, 0, 0, 1], [0, 0, 0, 0]], dtype=torch.uint8, device=DEV)
    for split in (0, 64, 1 << 20):
        out = torch.full(c.q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
        c.run(gpu, "block_causal", out=out, block_flags=flags, kv_split_tokens=split)
        full = c.run(gpu, "block_causal", kv_split_tokens=split)
        keep = flags.bool().repeat_interleave(8, 1).flatten()
        assert torch.equal(out[keep], full[keep]) and bool((out[~keep] == 9).all())
        c.check(full, "block_causal")
        gate = torch.zeros(1, dtype=torch.int32, device=DEV)
        out.fill_(9.0)
        c.run(gpu, "block_causal", out=out, run_if_nonzero=gate, kv_split_tokens=split)
        assert bool((out == 9).all())
        gate.fill_(3)
        c.run(gpu, "block_causal", out=out, run_if_nonzero=gate, kv_split_tokens=split)
        assert torch.equal(out, full)


def test_rows_behind_the_last_sequence_stay(gpu):
    c = Case(7, [50, 60], [8, 8], 8, 4, 2, 64)
    q = torch.cat([c.q, c.q]).to(DEV)
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
    c.run(gpu, q=q, out=out)
    c.check(out[:16])
    assert bool((out[16:] == 9).all())


def test_bad_page_ids_are_clamped(gpu):
    """Ids outside the pool and lengths beyond the table give wrong numbers,
    never an access outside; other sequences are not touched by them."""
    c = Case(8, [50, 500], [8, 8], 8, 4, 2, 64, width=33)
    args = c.pool.on(DEV)
    args[4][0] = -5
    args[4][0, ::2] = 1 << 30
    out = c.run(gpu, args=args)
    c.prefix[0] = 20000                       # past its 33 pages
    out2 = c.run(gpu, args=args)
    c.prefix[0] = 50
    want, size = c.want()
    for o in (out, out2):
        err = np.abs(o[8:].cpu().double().numpy() - want[8:])
        assert (err <= 2.0 ** -8 * np.abs(want[8:]) + (2.0 ** -8 + 2.0 ** -12) * size[8:]).all()


def test_same_inputs_same_bits(gpu):
    for heads, split in ((16, 0), (8, 64), (16, 64), (32, 128)):
        c = Case(9, [5000, 777, 3000], [32, 16, 8], 8, heads, 4, 128)
        a = c.run(gpu, "block_causal", kv_split_tokens=split)
        for _ in range(3):
            assert torch.equal(a, c.run(gpu, "block_causal", kv_split_tokens=split))


def test_q_that_is_not_finite_stays_in_its_row(gpu):
    c = Case(10, [200], [4], 4, 4, 1, 128)
    c.q[1, 2, 5] = float("inf")
    c.q[3, 0, 0] = float("nan")
    bad = torch.zeros(4, 4, dtype=torch.bool)
    bad[1, 2] = bad[3, 0] = True
    for rep in (1, 3, 16):                    # 16, 48 and 256 rows
        q = c.q.repeat(1, rep, 1)
        out = c.run(gpu, q=q.to(DEV), kv_split_tokens=0 if rep == 1 else 1 << 20).cpu()
        b = bad.repeat(1, rep)
        assert bool(torch.isnan(out[b]).all()) and bool(torch.isfinite(out[~b]).all())


def test_pool_past_32_bits(gpu):
    hkv, d = 8, 128
    pages = (1 << 31) // (hkv * 16 * d) + 5
    g = torch.Generator(DEV).manual_seed(1)
    raw = torch.randint(0, 256, (64, hkv, 16, d), generator=g, device=DEV, dtype=torch.uint8)
    raw &= 0xBF                                   # magnitudes below 2
    args = [torch.zeros(pages, hkv, 16, d, dtype=torch.uint8, device=DEV),
            torch.zeros(pages, hkv, d, 16, dtype=torch.uint8, device=DEV),
            torch.ones(pages, hkv, device=DEV), torch.ones(pages, hkv, device=DEV)]
    args[0][-64:], args[1][-64:] = raw, raw.transpose(2, 3)
    table = torch.arange(pages - 64, pages, dtype=torch.int32, device=DEV).view(1, 64)
    small = [a[-64:].contiguous() for a in args]
    for a in (args, small):
        a[0], a[1] = a[0].view(torch.float8_e4m3fn), a[1].view(torch.float8_e4m3fn)
    for heads, split in ((32, 0), (32, 64), (64, 64), (128, 64), (256, 128)):
        q = torch.randn(8, heads, d, generator=g, device=DEV, dtype=torch.bfloat16)
        kw = dict(max_prefix_len=1016, max_window_len=8, kv_split_tokens=split)
        a = gpu.window_attention_q8(q, *args, table, i32([1016], DEV), i32([8], DEV), 8, **kw)
        b = gpu.window_attention_q8(q, *small, table - (pages - 64), i32([1016], DEV), i32([8], DEV), 8, **kw)
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


def test_random_shapes(gpu):
    rng = np.random.default_rng(20)
    for i in range(60):
        d, fmt = int(rng.choice([64, 128])), str(rng.choice(["e4m3", "e5m2"]))
        hkv, group = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 5, 8]))
        block = int(rng.choice([1, 3, 16, 32]))
        n = int(rng.integers(1, 6))
        win = (block * rng.integers(0, 5, n)).tolist()
        prefix = [int(x) for x in np.exp(rng.uniform(0, 8, n))]
        split = int(rng.choice([0, 64, 256, 1 << 20]))
        if sum(win) == 0:
            continue
        c = Case(100 + i, prefix, win, block, hkv * group, hkv, d, fmt, sigma_q=float(rng.choice([0.3, 1.0, 4.0])))
        mode = str(rng.choice(["bidir", "block_causal"]))
        c.check(c.run(gpu, mode, kv_split_tokens=split), mode,
                what=f"case {i}: d {d} {fmt} heads {hkv}x{group} block {block} windows {win} prefixes {prefix} split {split}")
