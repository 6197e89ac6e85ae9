"""The 8-bit cache's calls without a GPU: exports, the header as plain C, every
refusal of the C entry points (before any HIP call) and of the binding, and the
workspace sizes."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2607_22663_amd as mbe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    return mbe.load()


def _declared():
    src = open(os.path.join(ROOT, "include", "mbe_q8.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    return set(re.findall(r"\b(mbe_\w+)\s*\(", src))


def test_every_declared_symbol_is_exported(lib):
    assert _declared() == set(mbe.EXPORTS_Q8)
    for n in _declared():
        assert hasattr(lib, n), n


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text(r'''
#include <string.h>
#include "mbe_q8.h"
int main(void) {
  mbe_paged_kv_q8 kv;
  mbe_attn_opts o;
  memset(&kv, 0, sizeof(kv));
  memset(&o, 0, sizeof(o));
  kv.page_size = 16; kv.num_kv_heads = 4; kv.head_dim = 128; kv.num_pages = 10; kv.format = MBE_Q8_E5M2;
  o.batch = 1; o.num_q_heads = 16; o.max_pages_per_seq = 10; o.total_q = 64; o.max_prefix_len = 64;
  o.max_window_len = 64;
  if (mbe_window_attention_q8_workspace_size(&kv, &o) != 0) return 1;
  kv.head_dim = 96;
  if (mbe_window_attention_q8(NULL, &kv, NULL, NULL, NULL, 32, NULL, &o) != MBE_ERR_UNSUPPORTED) return 2;
  if (strstr(mbe_last_error(), "head_dim") == NULL) return 3;
  return 0;
}
''')
    exe, libdir = tmp_path / "use", os.path.dirname(mbe.LIB_PATH)
    r = subprocess.run([cc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"),
                        str(src), "-o", str(exe), "-L", libdir, "-lmbe", f"-Wl,-rpath,{libdir}"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


def _vp(x):
    return None if x is None else ctypes.c_void_p(x)


def _kv(**kw):
    a = dict(k_pages=16, v_pages=32, k_scales=16, v_scales=16, num_pages=10, page_size=16, num_kv_heads=4, head_dim=128,
             format=0)
    a.update(kw)
    return mbe.PagedKVQ8(**{k: _vp(v) if k.endswith(("pages", "scales")) and k != "num_pages" else v
                            for k, v in a.items()})


POOL_FAULTS = [(dict(head_dim=96), 3, "head_dim"), (dict(page_size=32), 3, "page_size"), (dict(format=2), 3, "format"),
               (dict(format=-1), 3, "format"), (dict(num_kv_heads=0), 2, "num_kv_heads"),
               (dict(num_kv_heads=70000), 2, "num_kv_heads"), (dict(num_pages=-1), 2, "num_pages"),
               (dict(num_pages=0), 2, "empty"), (dict(k_pages=None), 1, "non-NULL"), (dict(v_scales=None), 1, "non-NULL"),
               (dict(v_pages=24), 2, "16-byte"), (dict(k_scales=18), 2, "4-byte")]


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("kv,args,status,text", [(k, {}, s, t) for k, s, t in POOL_FAULTS] + [
    ({}, dict(batch=-1), 2, "batch"), ({}, dict(batch=70000), 2, "batch"), ({}, dict(max_len=-1), 2, "negative"),
    ({}, dict(total=-1), 2, "negative"), ({}, dict(max_pages=-1), 2, "negative"), ({}, dict(max_pages=0), 2, "empty"),
    ({}, dict(pt=None), 1, "non-NULL"), ({}, dict(k=None), 1, "non-NULL"), ({}, dict(lens=None), 1, "non-NULL"),
    ({}, dict(v=24), 2, "16-byte"), (dict(num_kv_heads=64), dict(max_len=1 << 30), 2, "too large"),
    (None, {}, 1, "paged_kv")])
def test_range_refusals(lib, read, kv, args, status, text):
    a = dict(pt=16, max_pages=8, start=16, lens=16, batch=2, max_len=64, total=96, k=16, v=32)
    a.update(args)
    ref = None if kv is None else ctypes.byref(_kv(**kv))
    if read:
        st = lib.mbe_kv_read_q8(ref, _vp(a["pt"]), a["max_pages"], _vp(a["start"]), _vp(a["lens"]), a["batch"],
                                a["max_len"], a["total"], _vp(a["k"]), _vp(a["v"]), None)
    else:
        st = lib.mbe_kv_write_q8(ref, _vp(a["pt"]), a["max_pages"], _vp(a["start"]), _vp(a["lens"]), None, a["batch"],
                                 a["max_len"], a["total"], _vp(a["k"]), _vp(a["v"]), None, 0, None)
    assert st == status and text in lib.mbe_last_error().decode(), (st, lib.mbe_last_error())


def test_flags_need_a_block_size(lib):
    st = lib.mbe_kv_write_q8(ctypes.byref(_kv()), _vp(16), 8, _vp(16), _vp(16), None, 2, 64, 96, _vp(16), _vp(16),
                             _vp(16), 0, None)
    assert st == 2 and "block_size" in lib.mbe_last_error().decode()


@pytest.mark.parametrize("args", [dict(batch=0), dict(max_len=0), dict(total=0)])
def test_empty_ranges_are_ok(lib, args):
    a = dict(batch=2, max_len=64, total=96)
    a.update(args)
    kv = _kv(k_pages=None, num_pages=0)
    assert lib.mbe_kv_write_q8(ctypes.byref(kv), None, 0, None, None, None, a["batch"], a["max_len"], a["total"], None,
                               None, None, 0, None) == 0
    assert lib.mbe_kv_read_q8(ctypes.byref(kv), None, 0, None, None, a["batch"], a["max_len"], a["total"], None, None,
                              None) == 0


def _opts(**kw):
    a = dict(batch=1, num_q_heads=16, max_pages_per_seq=10, total_q=64, max_prefix_len=64, max_window_len=64, mask_mode=0,
             softmax_scale=0.0, kv_split_tokens=0)
    a.update(kw)
    return mbe.AttnOpts(**a)


@pytest.mark.parametrize("kv,opts,call,status,text", [(k, {}, {}, s, t) for k, s, t in POOL_FAULTS] + [
    ({}, dict(num_q_heads=6), {}, 2, "multiple"), ({}, dict(num_q_heads=0), {}, 2, "multiple"),
    ({}, dict(max_window_len=48), {}, 2, "multiple of block_size"), ({}, dict(max_pages_per_seq=0), {}, 2, "empty"),
    ({}, dict(mask_mode=2), {}, 3, "mask_mode"), ({}, dict(kv_split_tokens=100), {}, 2, "multiple of 64"),
    ({}, dict(kv_split_tokens=-64), {}, 2, "multiple of 64"), ({}, dict(softmax_scale=math.nan), {}, 6, "finite"),
    ({}, dict(softmax_scale=math.inf), {}, 6, "finite"), ({}, dict(batch=-1), {}, 2, "batch"),
    ({}, dict(total_q=-1), {}, 2, "negative"), ({}, dict(max_prefix_len=-1), {}, 2, "negative"),
    ({}, dict(max_prefix_len=(1 << 30) + 1), {}, 2, "too large"), ({}, {}, dict(B=0), 2, "block_size"),
    ({}, {}, dict(q=None), 1, "non-NULL"), ({}, {}, dict(wl=None), 1, "non-NULL"), ({}, {}, dict(out=8), 2, "16-byte"),
    ({}, dict(max_prefix_len=65536, max_pages_per_seq=5000), {}, 4, "workspace"),
    ({}, dict(max_prefix_len=65536, max_pages_per_seq=5000, workspace=256, workspace_bytes=16), {}, 4, "workspace"),
    ({}, dict(max_prefix_len=65536, max_pages_per_seq=5000, workspace=264, workspace_bytes=1 << 40), {}, 4, "aligned"),
    (None, {}, {}, 1, "paged_kv"), ({}, None, {}, 1, "opts")])
def test_attention_refusals(lib, kv, opts, call, status, text):
    a = dict(q=16, pl=16, wl=16, out=32, B=32)
    a.update(call)
    ref = None if kv is None else ctypes.byref(_kv(**kv))
    st = lib.mbe_window_attention_q8(_vp(a["q"]), ref, _vp(16), _vp(a["pl"]), _vp(a["wl"]), a["B"], _vp(a["out"]),
                                     None if opts is None else ctypes.byref(_opts(**opts)))
    assert st == status and text in lib.mbe_last_error().decode(), (st, lib.mbe_last_error())


def test_attention_workspace(lib):
    def size(kv=None, **kw):
        return lib.mbe_window_attention_q8_workspace_size(ctypes.byref(kv or _kv()), ctypes.byref(_opts(**kw)))

    bad = ctypes.c_size_t(-1).value
    assert size() == 0                                                       # a few tiles: nothing is split
    big = dict(max_prefix_len=65536, max_pages_per_seq=5000)
    assert 0 < size(**big) != bad and size(**big) % 256 == 0
    assert size(batch=0, total_q=0) == 0
    assert size(num_q_heads=5) == bad
    assert lib.mbe_window_attention_q8_workspace_size(None, ctypes.byref(_opts())) == bad
    assert lib.mbe_window_attention_q8_workspace_size(ctypes.byref(_kv()), None) == bad
    # the largest bounds neither overflow nor ask for more than the shares hold
    wide = dict(max_window_len=256, max_pages_per_seq=1)
    assert 0 < size(batch=1024, max_prefix_len=1 << 20, total_q=1 << 18, **wide) < 1 << 28
    assert size(batch=1024, max_prefix_len=1 << 29, total_q=1 << 18, **wide) == 0      # (too many tiles to deal out)
    assert size(batch=1 << 30, max_prefix_len=1 << 29, total_q=2 ** 31 - 1, **wide) == bad
    # (units whose number wraps to nothing in 64 bits)
    assert size(_kv(num_kv_heads=4096), batch=1 << 30, num_q_heads=4096, max_prefix_len=0, max_window_len=1 << 30,
                total_q=2 ** 31 - 1) == bad
    # the binding's query agrees
    q = torch.empty(64, 16, 128, device="meta")
    k = torch.empty(10, 4, 16, 128, dtype=torch.float8_e4m3fn, device="meta")
    pt = torch.empty(1, 5000, device="meta")
    assert mbe.workspace_bytes_window_attention_q8(q, k, pt, 1, max_prefix_len=65536, max_window_len=64) == size(**big)


def test_attention_of_nothing_is_ok(lib):
    for kw in (dict(batch=0), dict(total_q=0), dict(max_window_len=0)):
        assert lib.mbe_window_attention_q8(None, ctypes.byref(_kv()), None, None, None, 32, None,
                                           ctypes.byref(_opts(**kw))) == 0


@pytest.mark.parametrize("args,status,text", [
    (dict(d=96), 3, "head_dim"), (dict(rot=24), 3, "rot_dim"), (dict(rot=0), 3, "rot_dim"), (dict(rot=144), 3, "rot_dim"),
    (dict(layout=2), 3, "layout"), (dict(scale=math.nan), 6, "finite"), (dict(scale=math.inf), 6, "finite"),
    (dict(hq=-1), 2, "num_q_heads"), (dict(hkv=70000), 2, "num_kv_heads"), (dict(batch=-1), 2, "batch"),
    (dict(batch=70000), 2, "batch"), (dict(max_len=-1), 2, "negative"), (dict(max_len=(1 << 27) + 1), 2, "too large"),
    (dict(total=-1), 2, "negative"), (dict(turns=None), 1, "non-NULL"), (dict(q=None), 1, "non-NULL"),
    (dict(ko=None), 1, "non-NULL"), (dict(k=8), 2, "16-byte"), (dict(qs=2052), 2, "multiples of 8"),
    (dict(qs=1024), 2, "smaller"), (dict(kos=-512), 2, "smaller")])
def test_rotary_refusals(lib, args, status, text):
    a = dict(q=16, qo=32, hq=16, qs=2048, qos=2048, k=48, ko=64, hkv=4, ks=512, kos=512, d=128, start=16, lens=16, batch=2,
             max_len=8, total=12, turns=16, rot=128, layout=0, scale=1.0)
    a.update(args)
    st = lib.mbe_rotary(_vp(a["q"]), _vp(a["qo"]), a["hq"], a["qs"], a["qos"], _vp(a["k"]), _vp(a["ko"]), a["hkv"], a["ks"],
                        a["kos"], a["d"], _vp(a["start"]), _vp(a["lens"]), a["batch"], a["max_len"], a["total"],
                        _vp(a["turns"]), a["rot"], a["layout"], a["scale"], 0, None)
    assert st == status and text in lib.mbe_last_error().decode(), (st, lib.mbe_last_error())


def _host_args(dev="cpu", fmt=torch.float8_e4m3fn):
    pool = [torch.zeros(6, 2, 16, 64, dtype=torch.uint8, device=dev).view(fmt),
            torch.zeros(6, 2, 64, 16, dtype=torch.uint8, device=dev).view(fmt), torch.ones(6, 2, device=dev),
            torch.ones(6, 2, device=dev), torch.arange(6, dtype=torch.int32, device=dev).view(1, 6)]
    lens = [torch.full((1,), 64, dtype=torch.int32, device=dev), torch.full((1,), 32, dtype=torch.int32, device=dev)]
    q = torch.zeros(32, 8, 64, dtype=torch.bfloat16, device=dev)
    return q, pool, lens


def _calls(m, q, pool, lens):
    kv = q[:, :2].contiguous()
    turns = torch.zeros(32, dtype=torch.int64, device=q.device)
    return [lambda: m.kv_write_q8(*pool, *lens, kv, kv, max_len=32),
            lambda: m.kv_read_q8(*pool, *lens, max_len=32, total=32),
            lambda: m.window_attention_q8(q, *pool, *lens, 32, max_prefix_len=64, max_window_len=32),
            lambda: m.rotary(q, kv, *lens, turns, max_len=32)]


def test_host_tensors_are_refused(lib):
    """By the binding, before the library is called."""
    reached = []

    class Lib:
        def __getattr__(self, name):
            f = getattr(lib, name)
            return f if "workspace" in name or name == "mbe_last_error" else lambda *x: reached.append(name) or 0

    mbe._lib = Lib()
    try:
        for call in _calls(mbe, *_host_args()):
            with pytest.raises((ValueError, RuntimeError, AssertionError)) as e:
                call()
            assert not isinstance(e.value, mbe.MbeError), e.value
    finally:
        mbe._lib = lib
    assert not reached, reached


@pytest.mark.gpu
def test_the_usual_calls_run_and_wrong_ones_are_named(gpu):
    q, pool, lens = _host_args("cuda:0")
    for call in _calls(gpu, q, pool, lens):
        call()
    torch.cuda.synchronize()
    names = ["k_pages", "v_pages", "k_scales", "v_scales", "page_table"]
    for i in range(5):
        t = pool[i]
        for fault in (t.cpu(), t.unsqueeze(0), t.to(torch.float64), None, [1], t.view(torch.uint8)[..., ::2].view(t.dtype)
                      if i < 2 else torch.stack([t, t], -1)[..., 0], t[:-1] if i < 4 else t[:0]):
            bad = pool[:i] + [fault] + pool[i + 1:]
            for call in _calls(gpu, q, bad, lens)[:3]:
                with pytest.raises((TypeError, ValueError, AttributeError)):
                    call()
    with pytest.raises(ValueError, match="v_pages"):           # token-major V is not a layout of this cache
        gpu.kv_read_q8(pool[0], pool[0], *pool[2:], *lens)
    with pytest.raises(TypeError, match="k_pages"):
        gpu.kv_read_q8(pool[0].view(torch.uint8), *pool[1:], *lens)
    kv = q[:, :2].contiguous()
    with pytest.raises(ValueError, match="k_new"):
        gpu.kv_write_q8(*pool, *lens, q, q, max_len=32)
    with pytest.raises(ValueError, match="kv_lens"):
        gpu.kv_write_q8(*pool, *lens, kv, kv, max_len=32, kv_lens=torch.zeros(2, dtype=torch.int32, device="cuda:0"))
    with pytest.raises(ValueError, match="block_flags"):
        gpu.kv_write_q8(*pool, *lens, kv, kv, max_len=32, block_size=16,
                        block_flags=torch.zeros(1, 3, dtype=torch.uint8, device="cuda:0"))
    with pytest.raises(ValueError, match="disagree"):
        gpu.window_attention_q8(q, *pool, lens[0], torch.zeros(2, dtype=torch.int32, device="cuda:0"), 32)
    with pytest.raises(ValueError, match="head_dim"):
        gpu.window_attention_q8(torch.zeros(32, 8, 128, dtype=torch.bfloat16, device="cuda:0"), *pool, *lens, 32)
    with pytest.raises(gpu.MbeError, match="multiple"):
        gpu.window_attention_q8(q[:, :3].contiguous(), *pool, *lens, 32)
    turns = torch.zeros(32, dtype=torch.int64, device="cuda:0")
    with pytest.raises(ValueError, match="contiguous"):
        gpu.rotary(q.transpose(0, 1), None, *lens, turns)
    with pytest.raises(ValueError, match="disagree"):
        gpu.rotary(q, kv[:5], *lens, turns)
    with pytest.raises(ValueError, match="out"):
        gpu.rotary(q, kv, *lens, turns, max_len=32, out=(q, None))
    with pytest.raises(gpu.MbeError, match="rot_dim"):
        gpu.rotary(q, kv, *lens, turns[:20], max_len=32)
    with pytest.raises(KeyError):
        gpu.rotary(q, kv, *lens, turns, max_len=32, layout="other")


@pytest.mark.gpu
def test_debug_checks_name_the_fault(gpu, monkeypatch):
    monkeypatch.setenv("MBE_DEBUG_CHECK", "1")
    q, pool, lens = _host_args("cuda:0")
    for call in _calls(gpu, q, pool, lens):
        call()
    short = [torch.full((1,), 80, dtype=torch.int32, device="cuda:0"), lens[1]]
    for call in _calls(gpu, q, pool, short)[:3]:
        with pytest.raises(gpu.MbeError, match="pages|outside"):
            call()
    pool[4][0, 5] = 6
    for call in _calls(gpu, q, pool, lens)[:3]:
        with pytest.raises(gpu.MbeError, match="page_table"):
            call()
    with pytest.raises(gpu.MbeError, match="add up"):
        gpu.kv_read_q8(*pool[:4], pool[4] * 0, *lens, max_len=32, total=31)
