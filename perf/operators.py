"""The operators of an 8-bit KV cache, as a decoding loop calls them: their plain
forms, the library's calls, and the work that is timed.

Kinds of case:

  rotary  rotary: rotation of the queries and keys of ragged sequences by their
          absolute positions
  write   kv_write_q8: keys and values quantised into an 8-bit paged pool, with
          one scale for each page of 16 tokens and head
  read    kv_read_q8: ranges of such a pool read back as bf16
  attn    window_attention_q8: attention of the editing window's queries over
          such a pool

The pools hold float8_e4m3fn or float8_e5m2.  A page's scale is a power of two,
the smallest that keeps its largest magnitude within the type; tokens that a
partial write leaves in a page keep their values, at a scale that never shrinks
under them.  The slots no sequence covers hold NaN codes.

Inputs are N(0, 1) in bf16, some heads and some tokens larger than others, as
keys and values are; pages are in a random order.  Lengths go by the case alone,
spread over its range; all values, tables and flags go by the seed.
"""
import math

import torch

own = False

PAGE = 16
DEV = "cuda"
FMT = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}        # largest finite value, 0.875 * 2^9 and 0.875 * 2^16
TOP_EXP = {"e4m3": 9, "e5m2": 16}
MIN_SCALE_EXP = -100                          # scale of a page of zeros


def _case(name, kind, **kw):
    return dict(kw, kind=kind, name=name) if name else dict(kw, kind=kind)


def _rotary(name, batch, lo, hi, *, start=0, hq=16, hkv=4, d=128, rot=128, layout="half", base=10000.0, factor=1.0,
            inverse=False):
    """Rows lo..hi of each sequence, from position `start` on; `factor`: how
    much longer the context is than the one the frequencies were made for."""
    return _case(name, "rotary", batch=batch, lo=lo, hi=hi, start=start, hq=hq, hkv=hkv, d=d, rot=rot, layout=layout,
                 base=base, factor=factor, inverse=inverse)


def _write(name, batch, lo, hi, plo, phi, *, hkv=4, d=128, fmt="e4m3", block=0):
    """lo..hi tokens written behind plo..phi tokens.  With `block` the range is
    written over by block flags, and more tokens follow it."""
    return _case(name, "write", batch=batch, lo=lo, hi=hi, prefix_lo=plo, prefix_hi=phi, hkv=hkv, d=d, fmt=fmt,
                 block=block)


def _read(name, batch, lo, hi, plo, phi, *, hkv=4, d=128, fmt="e4m3"):
    return _case(name, "read", batch=batch, lo=lo, hi=hi, prefix_lo=plo, prefix_hi=phi, hkv=hkv, d=d, fmt=fmt)


def _attn(name, batch, plo, phi, klo, khi, *, hq=16, hkv=4, d=128, block=32, fmt="e4m3", causal=False):
    """Windows of klo..khi blocks behind prefixes of plo..phi tokens."""
    return _case(name, "attn", batch=batch, prefix_lo=plo, prefix_hi=phi, k_lo=klo, k_hi=khi, hq=hq, hkv=hkv, d=d,
                 block=block, fmt=fmt, causal=causal)


def listed():
    return [
        # the window of two users deep in a long context: half the head rotated
        _rotary("rotary_b2_w64", 2, 64, 64, start=100000, rot=64, factor=4.0),
        # the prompts of a serving batch
        _rotary("rotary_prefill_b32", 32, 500, 4096, layout="interleaved"),
        # one decoded token of eight users, at any slot of its page
        _write("write_token_b8", 8, 1, 1, 1000, 4000),
        # blocks that an editing pass changed, written over in place
        _write("write_refresh_b16", 16, 128, 128, 1000, 8192, block=32),
        # the prompts of a serving batch
        _write("write_prefill_b32", 32, 500, 4096, 0, 0, fmt="e5m2"),
        # one short prompt of a small model
        _read("read_b1_n96_d64", 1, 96, 96, 0, 0, d=64),
        # whole caches of mixed lengths, taken out of the pool
        _read("read_b32_ragged", 32, 500, 8192, 0, 0),
        # a small model's first window: nothing but latency and launches
        _attn("attn_b1_p64_d64", 1, 64, 64, 2, 2, hq=4, d=64),
        # one token per sequence, prompts that end anywhere
        _attn("attn_token_b32", 32, 1000, 8192, 1, 1, block=1),
        # the ordinary decoding step on long prompts, a block per sequence
        _attn("attn_block_b8_p16384", 8, 16384, 16384, 1, 1),
        # recomputed blocks under the standard scope, windows of one to eight blocks
        _attn("attn_causal_b12_odd", 12, 1000, 12000, 1, 8, fmt="e5m2", causal=True),
        # large batch on long contexts, four-block windows
        _attn("attn_b64_long", 64, 4096, 32768, 4, 4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["rotary", "write", "write", "read", "attn", "attn", "attn"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 4, 4, 8])
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    batch = _log_int(rng, 1, 64)
    if kind == "rotary":
        # at most the values of the largest listed case
        hi = _log_int(rng, 1, max(1, min(4096, int(1.5e8 / ((hq + hkv) * d * batch)))))
        lo = rng.randint(0, hi)
        return _rotary(None, batch, lo, hi, start=rng.choice([0, rng.randrange(0, 1 << 20)]), hq=hq, hkv=hkv, d=d,
                       rot=rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)]),
                       layout=rng.choice(["half", "interleaved"]), base=rng.choice([10000.0, 500000.0]),
                       factor=rng.choice([1.0, 1.0, 4.0, 32.0]), inverse=rng.random() < 0.2)
    if kind in ("write", "read"):
        hi = _log_int(rng, 1, max(1, min(8192, int((3.5e7 if kind == "write" else 6.5e7) / (hkv * d * batch)))))
        lo = rng.randint(0, hi)
        phi = rng.choice([0, _log_int(rng, 1, 8192)])
        if kind == "read":
            return _read(None, batch, lo, hi, phi // 4, phi, hkv=hkv, d=d, fmt=fmt)
        return _write(None, batch, lo, hi, phi // 4, phi, hkv=hkv, d=d, fmt=fmt, block=rng.choice([0, 0, 16, 32]))
    block = rng.choice([1, 1, 16, 32, 32])
    k_hi = rng.choice([1, 2, 4, 8])
    k_lo = rng.choice([1, k_hi])
    # the bytes of all keys and the work on them stay below the largest listed case's
    most = min(32768, int(1.1e9 / (2 * hkv * d * batch)), int(1.2e12 / (4 * d * hq * k_hi * block * batch)))
    hi = _log_int(rng, 64, max(64, most - k_hi * block))
    lo = hi if rng.random() < 0.3 else max(0, int(hi * rng.uniform(0.05, 1.0)))
    return _attn(None, batch, lo, hi, k_lo, k_hi, hq=hq, hkv=hkv, d=d, block=block, fmt=fmt, causal=rng.random() < 0.4)


# ------------------------------------------------------------------ lengths
def _spread(lo, hi, n, step):
    """n whole numbers spread over lo..hi; the first is hi."""
    return [hi - int((hi - lo + 1) * ((i * step) % 1.0)) for i in range(n)]


def _lens(case):
    """Tokens before the range, and of the range, of every sequence."""
    n = case["batch"]
    if case["kind"] == "rotary":
        return [case["start"] + 37 * b for b in range(n)], _spread(case["lo"], case["hi"], n, 0.6180339887)
    p = _spread(case["prefix_lo"], case["prefix_hi"], n, 0.6180339887)
    if case["kind"] == "attn":
        return p, [k * case["block"] for k in _spread(case["k_lo"], case["k_hi"], n, 0.7548776662)]
    return p, _spread(case["lo"], case["hi"], n, 0.7548776662)


TAIL = 40       # tokens that follow a range that is written over


def _covered(case):
    """Tokens of each sequence that the cache holds (after the call)."""
    p, w = _lens(case)
    more = TAIL if case["kind"] == "write" and case["block"] else 0
    return [a + b + more for a, b in zip(p, w)]


def work(case):
    p, w = _lens(case)
    if case["kind"] == "rotary":
        n = sum(w) * (case["hq"] + case["hkv"])
        return {"bytes": 4 * n * case["d"] + 8 * len(p) + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    hkv, d, n = case["hkv"], case["d"], len(p)
    if case["kind"] == "attn":
        seen = 0
        for a, b in zip(p, w):
            k = b // case["block"]
            seen += b * (a + b) if not case["causal"] else b * a + case["block"] ** 2 * (k * (k + 1) // 2)
        keys, pages = sum(p) + sum(w), sum(-(-(a + b) // PAGE) for a, b in zip(p, w))
        return {"bytes": 2 * hkv * d * keys + 12 * hkv * pages + 4 * sum(w) * case["hq"] * d + 8 * n,
                "flops": 4 * d * case["hq"] * seen}
    tokens = sum(w)
    if case["kind"] == "write" and case["block"]:
        tokens = tokens // 2          # every second block is flagged, on the average
    pages = sum(-(-b // PAGE) for b in w)
    return {"bytes": 6 * hkv * d * tokens + 12 * hkv * pages + 8 * n, "flops": 2 * hkv * d * tokens}


# ------------------------------------------------------------------- inputs
def _values(g, rows, heads, d):
    """bf16 [rows, heads, d]: N(0, 1), rows and heads of different sizes."""
    x = torch.randn(rows, heads, d, generator=g, device=DEV, dtype=torch.bfloat16)
    x *= torch.exp2(2 * torch.rand(rows, 1, 1, generator=g, device=DEV) - 1).to(torch.bfloat16)
    return x * torch.exp2(torch.randint(-3, 4, (1, heads, 1), generator=g, device=DEV).float()).to(torch.bfloat16)


def _scale_exp(amax, fmt):
    """Exponent of the smallest power of two s with amax / s within the type."""
    m, e = torch.frexp(amax)
    e = e - TOP_EXP[fmt] + (m > 0.875).to(e.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, MIN_SCALE_EXP)).clamp(MIN_SCALE_EXP, 120)


def _filled(g, pages, hkv, a, b, fmt):
    """A pool [pages, hkv, a, b] of 8-bit values and its scales."""
    x = torch.randn(pages, hkv, a, b, generator=g, device=DEV, dtype=torch.bfloat16)
    x *= torch.exp2(2 * torch.rand(pages, hkv, 1, 1, generator=g, device=DEV) - 1).to(torch.bfloat16)
    s = torch.exp2(_scale_exp(x.abs().amax((2, 3)).float(), fmt).float())
    x *= (1 / s).to(torch.bfloat16)[:, :, None, None]            # exact: powers of two
    return x.to(FMT[fmt]), s


def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    p, w = _lens(case)
    n, rows = case["batch"], sum(w)
    i32 = dict(dtype=torch.int32, device=DEV)
    s = {"case": case, "rows": rows, "max_len": max(w), "start": torch.tensor(p, **i32), "lens": torch.tensor(w, **i32)}
    if case["kind"] == "rotary":
        s["q"], s["k"] = _values(g, rows, case["hq"], case["d"]), _values(g, rows, case["hkv"], case["d"])
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        f = _frequencies(case)
        s["freq"] = f.to(DEV)
        # the table that the call takes: turns per position, in units of 2^-64
        s["turns"] = torch.tensor([int(v * 2.0 ** 64) for v in (f / (2 * math.pi)).tolist()], dtype=torch.int64).to(DEV)
        s["scale"] = 0.1 * math.log(case["factor"]) + 1.0
        return s
    # a pool for a batch of the longest sequences, pages in a random order
    cover, hkv, d = _covered(case), case["hkv"], case["d"]
    width = -(-max(max(cover), 1) // PAGE)
    total = n * width
    s["table"] = torch.randperm(total, generator=g, device=DEV).to(torch.int32).view(n, width)
    s["k_pages"], s["k_scales"] = _filled(g, total, hkv, PAGE, d, case["fmt"])
    s["v_pages"], s["v_scales"] = _filled(g, total, hkv, d, PAGE, case["fmt"])
    slot = torch.arange(width * PAGE, device=DEV).view(1, width, PAGE)
    held = s["start"] if case["kind"] == "write" and not case["block"] else torch.tensor(cover, **i32)
    void = (slot >= held.view(n, 1, 1)).view(total, 1, PAGE)                # slots that no sequence covers
    at = s["table"].view(-1).long()
    void = torch.zeros_like(void).index_copy_(0, at, void)
    s["k_pages"].view(torch.uint8).masked_fill_(void[..., None], 0x7F)      # NaN in both types
    s["v_pages"].view(torch.uint8).masked_fill_(void[:, :, None, :], 0x7F)
    if case["kind"] == "attn":
        s["q"] = _values(g, rows, case["hq"], d)
        s["out"] = torch.empty_like(s["q"])
        s["max_prefix"] = max(p)
        s["host_start"], s["host_lens"] = torch.tensor(p, dtype=torch.int32), torch.tensor(w, dtype=torch.int32)
    elif case["kind"] == "write":
        s["k_new"], s["v_new"] = _values(g, rows, hkv, d), _values(g, rows, hkv, d)
        s["kv_lens"] = s["flags"] = None
        if case["block"]:
            s["kv_lens"] = torch.tensor(cover, **i32)
            s["flags"] = torch.randint(0, 2, (n, -(-s["max_len"] // case["block"])), generator=g, device=DEV,
                                       dtype=torch.uint8)
    else:
        s["k_out"], s["v_out"] = (torch.empty(rows, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return s


def _frequencies(case):
    """Radians per position, in 64 bits.  For a context `factor` times longer,
    the slow frequencies are divided by it, the fast ones are kept, with a ramp
    between 32 turns and 1 turn of the original context."""
    half = case["rot"] // 2
    f = case["base"] ** (-torch.arange(half, dtype=torch.float64) / half)
    if case["factor"] == 1.0:
        return f
    turns = 4096 * f / (2 * math.pi)
    keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
    return f * keep + f / case["factor"] * (1 - keep)


# ---------------------------------------------------------------- one pass
def run(s):
    if own:
        return _run_own(s)
    return {"rotary": _plain_rotary, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[s["case"]["kind"]](s)


def _run_own(s):
    import paper_2607_22663_amd as mbe
    c = s["case"]
    if c["kind"] == "rotary":
        return mbe.rotary(s["q"], s["k"], s["start"], s["lens"], s["turns"], scale=s["scale"], layout=c["layout"],
                          inverse=c["inverse"], max_len=s["max_len"], out=(s["q_out"], s["k_out"]))
    pools = s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["table"]
    if c["kind"] == "write":
        mbe.kv_write_q8(*pools, s["start"], s["lens"], s["k_new"], s["v_new"], max_len=s["max_len"],
                        kv_lens=s["kv_lens"], block_flags=s["flags"], block_size=c["block"] or None)
        return pools[:4]
    if c["kind"] == "read":
        return mbe.kv_read_q8(*pools, s["start"], s["lens"], max_len=s["max_len"], out=(s["k_out"], s["v_out"]))
    return mbe.window_attention_q8(s["q"], *pools, s["start"], s["lens"], c["block"], out=s["out"],
                                   mask_mode="block_causal" if c["causal"] else "bidir", max_prefix_len=s["max_prefix"],
                                   max_window_len=s["max_len"], host_prefix_lens=s["host_start"],
                                   host_window_lens=s["host_lens"])


def _row_places(s):
    """Sequence and place within it of every row of the ragged inputs."""
    lens = s["lens"].long()
    seq = torch.repeat_interleave(torch.arange(lens.numel(), device=DEV), lens, output_size=s["rows"])
    return seq, torch.arange(s["rows"], device=DEV) - (lens.cumsum(0) - lens)[seq]


def _plain_rotary(s):
    c = s["case"]
    r, half = c["rot"], c["rot"] // 2
    seq, at = _row_places(s)
    angle = (s["start"].long()[seq] + at).double()[:, None] * s["freq"]
    cos, sin = (torch.cos(angle) * s["scale"]).float()[:, None], (torch.sin(angle) * s["scale"]).float()[:, None]
    if c["inverse"]:
        sin = -sin

    def turned(x):
        x = x.float()
        a, b = (x[..., :half], x[..., half:r]) if c["layout"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
        y = [a * cos - b * sin, b * cos + a * sin]
        y = torch.cat(y, -1) if c["layout"] == "half" else torch.stack(y, -1).flatten(-2)
        return torch.cat([y, x[..., r:]], -1).to(torch.bfloat16)

    return turned(s["q"]), turned(s["k"])


def _plain_write(s):
    c = s["case"]
    dt, top = FMT[c["fmt"]], TOP[c["fmt"]]
    n, width = s["table"].shape
    start, lens = s["start"].long(), s["lens"].long()
    row0 = (lens.cumsum(0) - lens).view(n, 1, 1)
    start, lens = start.view(n, 1, 1), lens.view(n, 1, 1)
    # the pages each range can touch, and their 16 slots: [batch, pages, 16]
    page = start // PAGE + torch.arange(-(-s["max_len"] // PAGE) + 1, device=DEV).view(1, -1, 1)
    pos = page * PAGE + torch.arange(PAGE, device=DEV)
    t = pos - start
    new = (t >= 0) & (t < lens)
    if s["flags"] is not None:
        block = (t // c["block"]).clamp(0, s["flags"].shape[1] - 1)
        new = new & (torch.gather(s["flags"], 1, block.flatten(1)).view_as(block) != 0)
    held = start if s["kv_lens"] is None else torch.maximum(start, s["kv_lens"].long().view(n, 1, 1))
    kept = ~new & (pos < held)
    hit = new.any(-1) & (page[..., 0] < width)
    pid = torch.gather(s["table"].long(), 1, page[..., 0].clamp(max=width - 1))
    row = (row0 + t).clamp(0, max(s["rows"] - 1, 0))
    for pages, scales, x, slot_dim in ((s["k_pages"], s["k_scales"], s["k_new"], 2), (s["v_pages"], s["v_scales"], s["v_new"], 3)):
        x = x.float()[row].movedim(2, 3)                                    # [batch, pages, heads, 16, d]
        new_, kept_ = new[:, :, None, :, None], kept[:, :, None, :, None]
        raw = pages.view(torch.uint8)[pid]
        raw = raw.transpose(3, 4) if slot_dim == 3 else raw                 # [batch, pages, heads, 16, d]
        old, was = raw.contiguous().view(dt).float(), scales[pid]
        amax = torch.where(new_, x, torch.zeros_like(x)).abs().amax((3, 4))
        scale = torch.exp2(_scale_exp(amax, c["fmt"]).float())
        scale = torch.where(kept.any(-1)[..., None], torch.maximum(scale, was), scale)
        y = torch.where(new_, x / scale[..., None, None], old * (was / scale)[..., None, None])
        y = y.clamp(-top, top).to(dt).view(torch.uint8)
        y = torch.where(new_ | kept_, y, raw)
        y = y.transpose(3, 4) if slot_dim == 3 else y
        pages.view(torch.uint8)[pid[hit]] = y[hit]
        scales[pid[hit]] = scale[hit]
    return s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"]


def _plain_read(s):
    seq, at = _row_places(s)
    pos = s["start"].long()[seq] + at
    pid, slot = s["table"].long()[seq, pos // PAGE], pos % PAGE
    k = s["k_pages"].view(torch.uint8)[pid, :, slot].view(s["k_pages"].dtype).float() * s["k_scales"][pid][..., None]
    v = s["v_pages"].view(torch.uint8)[pid, :, :, slot].view(s["v_pages"].dtype).float() * s["v_scales"][pid][..., None]
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_attn(s):
    c = s["case"]
    n, width = s["table"].shape
    hkv, d, group, wmax, block = c["hkv"], c["d"], c["hq"] // c["hkv"], s["max_len"], c["block"]
    seq, at = _row_places(s)
    q = torch.zeros(n, wmax, c["hq"], d, device=DEV)
    q[seq, at] = s["q"].float()
    q = q.view(n, wmax, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, group * wmax, d)
    pid = s["table"].long()
    total = (s["start"] + s["lens"]).long().view(n, 1)
    key = torch.arange(width * PAGE, device=DEV)
    held = (key < total)[:, None, :, None]                                  # slots that hold a token
    k = s["k_pages"].view(torch.uint8)[pid].view(s["k_pages"].dtype).float() * s["k_scales"][pid][..., None, None]
    k = k.transpose(1, 2).reshape(n, hkv, width * PAGE, d).masked_fill_(~held, 0)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(d)).view(n, hkv, group, wmax, width * PAGE)
    del k
    if c["causal"]:
        seen = (torch.arange(wmax, device=DEV) // block + 1) * block
        seen = torch.minimum(s["start"].long().view(n, 1) + seen, total)
    else:
        seen = total.expand(n, wmax)
    score.masked_fill_((key >= seen[..., None])[:, None, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True)).exp_()
    norm = score.sum(-1, keepdim=True)
    v = s["v_pages"].view(torch.uint8)[pid].view(s["v_pages"].dtype).float() * s["v_scales"][pid][..., None, None]
    v = v.permute(0, 2, 1, 4, 3).reshape(n, hkv, width * PAGE, d).masked_fill_(~held, 0)
    out = torch.matmul(score.view(n, hkv, group * wmax, -1), v).view(n, hkv, group, wmax, d) / norm
    out = out.permute(0, 3, 1, 2, 4).reshape(n, wmax, c["hq"], d)
    return out[seq, at].to(torch.bfloat16)


# --------------------------------------------------- the definition, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "write": _exact_write, "read": _exact_read, "attn": _exact_attn}[case["kind"]](case, s)


def _exact_rotary(c, s):
    """Pairs as complex numbers, multiplied by scale * exp(i * angle)."""
    p, w = _lens(c)
    r = c["rot"]
    pos = torch.cat([a + torch.arange(b, dtype=torch.float64) for a, b in zip(p, w)]).to(DEV)
    angle = pos[:, None] * s["freq"] * (-1 if c["inverse"] else 1)
    turn = torch.polar(torch.full_like(angle, s["scale"]), angle)[:, None]
    done = []
    for x in (s["q"].double(), s["k"].double()):
        y = x.clone()
        if c["layout"] == "half":
            z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        else:
            z = torch.view_as_complex(x[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn
            y[..., :r] = torch.view_as_real(z).flatten(-2)
        done.append(y)
    return tuple(done)


def _rounded(x, fmt):
    """x, in 64 bits, to the nearest value of the type; ties to the even one."""
    digits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    x = x.clamp(-TOP[fmt], TOP[fmt])
    e = (torch.frexp(x)[1] - 1).clamp(min=low).double()
    step = torch.exp2(e - digits)
    return torch.round(x / step) * step


def _exact_write(c, s):
    """Page by page, in the order of the tokens."""
    p, w = _lens(c)
    flags = s["flags"].tolist() if s["flags"] is not None else None
    table = s["table"].tolist()
    done = []
    for pages, scales, x, minor in ((s["k_pages"], s["k_scales"], s["k_new"], False), (s["v_pages"], s["v_scales"], s["v_new"], True)):
        out, sc, x = pages.double(), scales.double(), x.double()
        row0 = 0
        for b in range(c["batch"]):
            held = max(p[b], p[b] + w[b] + TAIL if flags else 0)
            for page in range(p[b] // PAGE, -(-(p[b] + w[b]) // PAGE)):
                span = range(page * PAGE, (page + 1) * PAGE)
                new = [t for t in span if p[b] <= t < p[b] + w[b] and (not flags or flags[b][(t - p[b]) // c["block"]])]
                if not new:
                    continue
                kept = [t - page * PAGE for t in span if t < held and t not in new]
                rows = x[[row0 + t - p[b] for t in new]]                    # [tokens, heads, d]
                top = rows.abs().amax((0, 2))
                need = torch.ceil(torch.log2(top / TOP[c["fmt"]])).clamp(MIN_SCALE_EXP, 120)
                need = need + (top > TOP[c["fmt"]] * torch.exp2(need))       # a logarithm next to a whole number
                need = need - (top <= TOP[c["fmt"]] * torch.exp2(need - 1)).double() * (need > MIN_SCALE_EXP)
                scale = torch.exp2(need)
                at = out[table[b][page]].transpose(1, 2) if minor else out[table[b][page]]   # [heads, 16, d], a view
                if kept:
                    was = sc[table[b][page]]
                    scale = torch.maximum(scale, was)
                    at[:, kept] = _rounded(at[:, kept] * (was / scale)[:, None, None], c["fmt"])
                at[:, [t - page * PAGE for t in new]] = _rounded(rows.transpose(0, 1) / scale[:, None, None], c["fmt"])
                sc[table[b][page]] = scale
            row0 += w[b]
        done += [out, sc]
    return done[0], done[2], done[1], done[3]


def _exact_read(c, s):
    p, w = _lens(c)
    ks, vs = [], []
    for b in range(c["batch"]):
        pid = s["table"][b].long()
        k = s["k_pages"].view(torch.uint8)[pid].view(FMT[c["fmt"]]).double() * s["k_scales"][pid].double()[..., None, None]
        v = s["v_pages"].view(torch.uint8)[pid].view(FMT[c["fmt"]]).double() * s["v_scales"][pid].double()[..., None, None]
        ks.append(k.transpose(1, 2).flatten(0, 1)[p[b]:p[b] + w[b]])
        vs.append(v.permute(0, 3, 1, 2).flatten(0, 1)[p[b]:p[b] + w[b]])
    return torch.cat(ks), torch.cat(vs)


def _exact_attn(c, s):
    """Sequence by sequence and head by head."""
    p, w = _lens(c)
    group, d = c["hq"] // c["hkv"], c["d"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    row0 = 0
    for b in range(c["batch"]):
        n = p[b] + w[b]
        pid = s["table"][b, : -(-n // PAGE)].long()
        blocks = torch.arange(w[b], device=DEV) // c["block"]
        for h in range(c["hkv"]):
            k = (s["k_pages"][:, h].view(torch.uint8)[pid].view(FMT[c["fmt"]]).double() * s["k_scales"][pid, h].double()[:, None, None])
            v = (s["v_pages"][:, h].view(torch.uint8)[pid].view(FMT[c["fmt"]]).double() * s["v_scales"][pid, h].double()[:, None, None])
            k, v = k.flatten(0, 1)[:n], v.transpose(1, 2).flatten(0, 1)[:n]
            q = s["q"][row0:row0 + w[b], h * group:(h + 1) * group].double()
            x = torch.matmul(q.reshape(-1, d), k.T.contiguous()).view(w[b], group, n) / math.sqrt(d)
            if c["causal"]:
                hidden = blocks[:, None] < blocks[None, :]                  # [queries, window keys]
                x[:, :, p[b]:] = x[:, :, p[b]:].masked_fill(hidden[:, None], -math.inf)
            out[row0:row0 + w[b], h * group:(h + 1) * group] = torch.matmul(torch.softmax(x, -1).view(-1, n), v).view(w[b], group, d)
        row0 += w[b]
    return out
