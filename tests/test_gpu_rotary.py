"""The rotation against the 64-bit oracle.  Tolerance: the result is rounded
once to bf16 (2^-8 of it at most), and the fp32 arithmetic before that is off
by the sine's and cosine's error, taken as 2^-18 each, times the pair's length
(|x| + |y|) * scale, and a few fp32 roundings (2^-22)."""
import numpy as np
import pytest
import torch

from oracle import q8
from q8_util import bf16, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(got, x, pos, turns, scale, inter, inverse, what):
    want = q8.rotary(x, pos, turns, scale, inter, inverse)
    x = x.double().abs().numpy()
    size = np.zeros_like(want)
    half = len(turns)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + half)
        size[..., a] = size[..., b] = (x[..., a] + x[..., b]) * abs(scale)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -18 + 2.0 ** -22) * size
    err = np.abs(got.cpu().double().numpy() - want)
    assert (err <= tol).all(), f"{what}: {err.max():.3e}, {float((err / np.maximum(tol, 1e-30)).max()):.2f} of the tolerance"


def _positions(start, lens):
    return np.concatenate([s + np.arange(n) for s, n in zip(start, lens)]) if sum(lens) else np.zeros(0)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 16), (64, 64), (128, 32), (128, 48), (128, 112), (128, 128)])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1), (16, 4), (6, 0)])
def test_shapes(gpu, inter, d, rot, hq, hkv):
    rng = np.random.default_rng(d + rot)
    start, lens = [0, 5, 100000, (1 << 31) - 40], [3, 0, 33, 17]
    n = sum(lens)
    turns = gpu.rotary_turns(gpu.rotary_frequencies(rot), DEV)
    q, k = bf16(rng, n + 2, hq, d), bf16(rng, n + 2, hkv, d) if hkv else None
    oq = torch.full((n + 2, hq, d), 5.0, dtype=torch.bfloat16, device=DEV)
    ok = torch.full((n + 2, hkv, d), 5.0, dtype=torch.bfloat16, device=DEV) if hkv else None
    gpu.rotary(q.to(DEV), None if k is None else k.to(DEV), i32(start, DEV), i32(lens, DEV), turns, scale=1.1,
               layout="interleaved" if inter else "half", max_len=33, out=(oq, ok))
    torch.cuda.synchronize()
    pos, t = _positions(start, lens), turns.cpu().numpy().astype(object)
    _check(oq[:n], q[:n], pos, t, np.float32(1.1), inter, False, "q")
    assert bool((oq[n:] == 5).all())                       # rows behind the last sequence
    if hkv:
        _check(ok[:n], k[:n], pos, t, np.float32(1.1), inter, False, "k")
        assert bool((ok[n:] == 5).all())
    assert torch.equal(oq[:n, :, rot:].cpu(), q[:n, :, rot:])


@pytest.mark.parametrize("inter", [False, True])
def test_in_place_on_a_packed_projection(gpu, inter):
    """q and k are slices of one [rows, (Hq + 2 Hkv) * D] tensor; v stays."""
    rng = np.random.default_rng(5)
    hq, hkv, d, n = 8, 2, 64, 21
    packed = bf16(rng, n, hq + 2 * hkv, d)
    dev = packed.to(DEV)
    q, k = dev[:, :hq], dev[:, hq:hq + hkv]
    turns = gpu.rotary_turns(gpu.rotary_frequencies(d), DEV)
    layout = "interleaved" if inter else "half"
    a, b = gpu.rotary(q, k, i32([7], DEV), i32([n], DEV), turns, layout=layout, max_len=n, out=(q, k))
    torch.cuda.synchronize()
    assert a is q and b is k
    pos, t = _positions([7], [n]), turns.cpu().numpy().astype(object)
    _check(dev[:, :hq], packed[:, :hq], pos, t, 1.0, inter, False, "q")
    _check(dev[:, hq:hq + hkv], packed[:, hq:hq + hkv], pos, t, 1.0, inter, False, "k")
    assert torch.equal(dev[:, hq + hkv:].cpu(), packed[:, hq + hkv:])


@pytest.mark.parametrize("inter", [False, True])
def test_inverse_is_the_gradient(gpu, inter):
    """d/dx of <w, rotary(x)> is rotary(w, inverse): against the formula, and
    <w, R x> = <R' w, x> with fp64 sums of the rounded outputs."""
    rng = np.random.default_rng(6)
    n, h, d = 40, 3, 128
    x, w = bf16(rng, n, h, d), bf16(rng, n, h, d)
    turns = gpu.rotary_turns(gpu.rotary_frequencies(96, scaling="ramp", factor=8.0), DEV)
    kw = dict(scale=1.2, layout="interleaved" if inter else "half", max_len=n)
    args = i32([1 << 20], DEV), i32([n], DEV), turns
    y, _ = gpu.rotary(x.to(DEV), None, *args, **kw)
    g, _ = gpu.rotary(w.to(DEV), None, *args, inverse=True, **kw)
    pos, t = _positions([1 << 20], [n]), turns.cpu().numpy().astype(object)
    _check(g, w, pos, t, np.float32(1.2), inter, True, "gradient")
    left = (w.double() * y.cpu().double()).sum().item()
    right = (g.cpu().double() * x.double()).sum().item()
    # each side's roundings: at most 2^-8 of every output, times the other factor
    tol = 2.0 ** -8 * ((w.double() * y.cpu().double()).abs().sum() + (g.cpu().double() * x.double()).abs().sum()).item()
    assert abs(left - right) <= tol
    # differences: the map is linear, so a step in one value moves the output by step * column
    e = x.clone()
    e[3, 1, 5] += 1.0
    step = float(e[3, 1, 5].double() - x[3, 1, 5].double())
    y2, _ = gpu.rotary(e.to(DEV), None, *args, **kw)
    diff = ((y2.double() - y.double()).cpu() * w.double()).sum().item() / step
    size = float((y2.double().abs() + y.double().abs()).cpu()[3, 1].max() * w[3, 1].double().abs().sum())
    assert abs(diff - float(g[3, 1, 5])) <= 2.0 ** -8 * (size / step + abs(float(g[3, 1, 5])))


def test_frequencies(gpu):
    """The scalings, at both ends of their ranges, and the table's rounding."""
    f = gpu.rotary_frequencies(64)
    assert f[0] == 1.0 and abs(f[31] - 10000.0 ** (-31 / 32)) < 1e-15
    assert torch.equal(gpu.rotary_frequencies(64, scaling="linear", factor=4.0), f / 4)
    b = gpu.rotary_frequencies(64, scaling="base", factor=4.0)
    assert b[0] == 1.0 and abs(b[31] * 4 / f[31] - 1) < 1e-12
    r = gpu.rotary_frequencies(64, scaling="ramp", factor=4.0, original_len=4096)
    assert r[0] == f[0] and abs(r[31] * 4 / f[31] - 1) < 1e-15
    with pytest.raises(ValueError, match="scaling"):
        gpu.rotary_frequencies(64, scaling="other")
    t = gpu.rotary_turns([0.0, 3 * np.pi, -np.pi / 2, 2 * np.pi], "cpu")
    # 0, half a turn over one, a quarter back, one turn: modulo one turn (fp64 of f / 2 pi)
    got = [int(v) % (1 << 64) / 2.0 ** 64 for v in t.tolist()]
    assert np.allclose(got[:3], [0.0, 0.5, 0.75], atol=1e-15) and min(got[3], 1 - got[3]) < 1e-15


def test_empty(gpu):
    turns = gpu.rotary_turns(gpu.rotary_frequencies(64), DEV)
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    a, b = gpu.rotary(q, q, i32([], DEV), i32([], DEV), turns)
    assert a.shape == q.shape and b.shape == q.shape
    q = torch.ones(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    a, _ = gpu.rotary(q, None, i32([5, 6], DEV), i32([0, 0], DEV), turns, out=(q.clone() * 3, None))
    assert bool((a == 3).all())
