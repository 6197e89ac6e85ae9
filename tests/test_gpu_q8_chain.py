"""The 8-bit cache's calls as a decoding loop makes them: rotation of a packed
projection, quantising write, attention; prompts, tokens, an editing pass and
the refresh of its changed blocks; eagerly, in captured graphs, on streams."""
import numpy as np
import pytest
import torch

import oracle
from oracle import q8
from q8_util import DTYPES, Pool, bf16, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HKV, D = 8, 2, 128


class Loop:
    """A layer's state on the device, and the same by the oracle on the CPU."""

    def __init__(self, gpu, rng, cap, fmt="e4m3"):
        self.gpu, self.rng, self.n = gpu, rng, len(cap)
        self.pool = Pool(rng, cap, HKV, D, fmt)
        self.dev = self.pool.on(DEV)
        self.turns = gpu.rotary_turns(gpu.rotary_frequencies(D, scaling="ramp", factor=4.0), DEV)
        self.cap = max(cap)

    def project(self, rows):
        return bf16(self.rng, rows, HQ + 2 * HKV, D).to(DEV)

    def rotate_write(self, qkv, start, lens, **kw):
        """In place on the packed projection, then into the pool; the pool is
        compared with the oracle's, bit for bit."""
        q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
        s, n = i32(start, DEV), i32(lens, DEV)
        before = k.cpu()
        self.gpu.rotary(q, k, s, n, self.turns, max_len=max(lens), out=(q, k))
        pos = np.concatenate([a + np.arange(b) for a, b in zip(start, lens)])
        want = q8.rotary(before, pos, self.turns.cpu().numpy().astype(object))
        err = np.abs(k.cpu().double().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -14).all()      # (|x| + |y| < 16: 2^-18 of it, see the rotation's test)
        k, v = k.contiguous(), v.contiguous()
        args = {key: None if x is None else torch.as_tensor(x, dtype=torch.uint8 if key == "block_flags" else torch.int32).to(DEV)
                for key, x in kw.items() if key != "block_size"}
        self.gpu.kv_write_q8(*self.dev, s, n, k, v, max_len=max(lens), block_size=kw.get("block_size"), **args)
        p = self.pool
        p.set(q8.kv_write_q8(p.k, p.v, p.ks, p.vs, p.table, start, lens, k, v, p.fmt, kw.get("kv_lens"),
                             kw.get("block_flags"), kw.get("block_size")))
        for got, w in zip(self.dev[:4], (p.k, p.v, p.ks, p.vs)):
            got = got.cpu().view(torch.uint8) if w.dtype == torch.uint8 else got.cpu()
            assert np.array_equal(got.numpy(), w.numpy(), equal_nan=w.dtype != torch.uint8)
        return q.contiguous()

    def attend(self, q, prefix, window, block, mode="bidir", **kw):
        out = self.gpu.window_attention_q8(q, *self.dev, i32(prefix, DEV), i32(window, DEV), block, mask_mode=mode,
                                           max_prefix_len=self.cap, max_window_len=max(window), **kw)
        k, v = self.pool.values()
        m = oracle.MASK_BIDIR if mode == "bidir" else oracle.MASK_BLOCK_CAUSAL
        rest = self.pool.table, prefix, window, block, m
        want, size = oracle.window_attention(q, k, v, *rest), oracle.window_attention(q, k, v.abs(), *rest)
        err = np.abs(out.cpu().double().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * size).all()
        return out


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_prompts_tokens_edits_and_refresh(gpu, fmt):
    rng = np.random.default_rng(1)
    prompts = [37, 300, 5]
    loop = Loop(gpu, rng, [p + 80 for p in prompts], fmt)
    # prompts, block-causal from nothing
    q = loop.rotate_write(loop.project(sum(prompts)), [0, 0, 0], prompts)
    # (windows are whole blocks: blocks of one token, the causal scope)
    loop.attend(q, [0, 0, 0], prompts, 1, "block_causal")
    # tokens one by one
    held = list(prompts)
    for _ in range(3):
        q = loop.rotate_write(loop.project(3), held, [1, 1, 1])
        loop.attend(q, held, [1, 1, 1], 1)
        held = [h + 1 for h in held]
    # a window of four blocks of 16, an editing pass over it, and the refresh of the
    # blocks it changed, written over in place with nothing behind them lost
    window = [64, 64, 64]
    q = loop.rotate_write(loop.project(192), held, window)
    loop.attend(q, held, window, 16)
    flags = [[0, 1, 0, 1], [0, 0, 0, 0], [1, 0, 0, 0]]
    total = [h + 64 for h in held]
    q = loop.rotate_write(loop.project(192), held, window, kv_lens=total, block_flags=flags, block_size=16)
    loop.attend(q, held, window, 16, "block_causal")
    out = torch.full_like(q, 5.0)
    part = gpu.window_attention_q8(q, *loop.dev, i32(held, DEV), i32(window, DEV), 16, mask_mode="block_causal",
                                   max_prefix_len=400, max_window_len=64, out=out,
                                   block_flags=torch.tensor(flags, dtype=torch.uint8, device=DEV))
    keep = torch.tensor(flags, device=DEV).bool().repeat_interleave(16, 1).flatten()
    assert bool((part[~keep] == 5).all()) and bool(torch.isfinite(part[keep]).all())
    # the whole cache read back is what the oracle holds
    k, v = gpu.kv_read_q8(*loop.dev, i32([0, 0, 0], DEV), i32(total, DEV))
    p = loop.pool
    K, V = q8.kv_read_q8(p.k, p.v, p.ks, p.vs, p.table, [0, 0, 0], total, fmt)
    assert np.array_equal(k.cpu().double().numpy(), K) and np.array_equal(v.cpu().double().numpy(), V)


@pytest.mark.parametrize("window,prefix", [(1, 900), (32, 200), (64, 3000), (256, 2500)])
def test_captured_step(gpu, window, prefix):
    """Rotation, write and attention in one graph, replayed with other inputs,
    positions and lengths, eager calls and synchronisations between the replays;
    two graphs of it replayed on two streams at once."""
    rng = np.random.default_rng(2)
    n, cap = 4, prefix + window + 40
    pool = Pool(rng, [cap] * n, HKV, D, "e4m3").fill(rng, [cap] * n)
    turns = gpu.rotary_turns(gpu.rotary_frequencies(D), DEV)

    def state():
        return {"dev": pool.on(DEV), "qkv": torch.zeros(n * window, HQ + 2 * HKV, D, dtype=torch.bfloat16, device=DEV),
                "start": i32([0] * n, DEV), "lens": i32([window] * n, DEV), "held": i32([cap] * n, DEV),
                "q": torch.zeros(n * window, HQ, D, dtype=torch.bfloat16, device=DEV),
                "k": torch.zeros(n * window, HKV, D, dtype=torch.bfloat16, device=DEV),
                "out": torch.zeros(n * window, HQ, D, dtype=torch.bfloat16, device=DEV)}

    def step(s):
        q, k, v = s["qkv"][:, :HQ], s["qkv"][:, HQ:HQ + HKV], s["qkv"][:, HQ + HKV:].contiguous()
        gpu.rotary(q, k, s["start"], s["lens"], turns, max_len=window, out=(s["q"], s["k"]))
        gpu.kv_write_q8(*s["dev"], s["start"], s["lens"], s["k"], v, max_len=window, kv_lens=s["held"])
        gpu.window_attention_q8(s["q"], *s["dev"], s["start"], s["lens"], window, out=s["out"], max_prefix_len=prefix + 20,
                                max_window_len=window)

    def feed(s, seed):
        g = torch.Generator(DEV).manual_seed(seed)
        s["qkv"].copy_(torch.randn(s["qkv"].shape, generator=g, device=DEV))
        s["start"].copy_(torch.randint(prefix - 60, prefix + 20, (n,), generator=g, device=DEV))

    eager, a, b = state(), state(), state()
    graphs = []
    for s in (a, b):
        feed(s, 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(s)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    # (the warm-up wrote the pools of a and b; the eager one follows)
    feed(eager, 1)
    step(eager)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for seed in range(2, 7):
        feed(eager, seed)
        step(eager)
        torch.cuda.synchronize()
        for s in (a, b):
            feed(s, seed)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s in (a, b):
            assert torch.equal(s["out"], eager["out"]), (window, seed)
            for x, y in zip(s["dev"], eager["dev"]):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        assert bool(torch.isfinite(eager["out"]).all())


def test_calls_on_two_streams(gpu):
    """Split calls on two streams at once do not share memory."""
    rng = np.random.default_rng(3)
    pools = [Pool(rng, [6000], 2, 128, "e4m3").fill(rng, [6000]).on(DEV) for _ in range(2)]
    q = [bf16(rng, 16, 8, 128).to(DEV) for _ in range(2)]
    args = i32([5984], DEV), i32([16], DEV), 16
    kw = dict(max_prefix_len=5984, max_window_len=16)
    want = [gpu.window_attention_q8(q[i], *pools[i], *args, **kw) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(gpu.window_attention_q8(q[i], *pools[i], *args, **kw))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_own_workspace(gpu):
    rng = np.random.default_rng(4)
    pool = Pool(rng, [3000], 1, 64, "e5m2").fill(rng, [3000]).on(DEV)
    q = bf16(rng, 8, 4, 64).to(DEV)
    kw = dict(max_prefix_len=2992, max_window_len=8)
    need = gpu.workspace_bytes_window_attention_q8(q, pool[0], pool[4], 1, **kw)
    assert need > 0
    args = q, *pool, i32([2992], DEV), i32([8], DEV), 8
    want = gpu.window_attention_q8(*args, **kw)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)       # any contents
    assert torch.equal(gpu.window_attention_q8(*args, workspace=ws, **kw), want)
    assert torch.equal(gpu.window_attention_q8(*args, workspace=ws, **kw), want)
    with pytest.raises(gpu.MbeError, match="workspace"):
        gpu.window_attention_q8(*args, workspace=ws[:need - 256], **kw)
    with pytest.raises(ValueError, match="workspace"):
        gpu.window_attention_q8(*args, workspace=ws.float(), **kw)
