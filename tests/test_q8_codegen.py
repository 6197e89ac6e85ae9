"""Properties of the 8-bit attention kernels' gfx950 code, on the assembly hipcc
writes for them with the library's own flags (no GPU is used): the key loops keep
their loads in flight across iterations, so no block of a loop that multiplies may
wait for every load, and none may touch scratch memory."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="needs hipcc")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from paper_2607_22663_amd import build as b
    flags = [f for f in b.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = tmp_path_factory.mktemp("asm") / "attn_q8.s"
    cmd = [b.hipcc(), *flags, "--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"), "-o", str(out),
           os.path.join(b.CSRC, "attn_q8.hip")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    asm = out.read_text()
    found = {}
    for m in re.finditer(r"^(_ZN3mbe12_GLOBAL__N_1\d+attn_q8_(\w+?)_kernel\w+):", asm, re.M):
        end = asm.index(".Lfunc_end", m.start())
        found[m.group(1)] = (m.group(2), asm[m.start():end], int(re.search(r"; ScratchSize: (\d+)", asm[end:]).group(1)))
    return found


def test_every_form_is_there(kernels):
    kinds = sorted(k for k, _, _ in kernels.values())
    # head_dim x type for the streaming and tile kernels, x row groups for the wide
    # one; head_dim x rows for the join
    assert kinds == ["join"] * 8 + ["stream"] * 4 + ["tile"] * 4 + ["wide"] * 8, kinds


def test_key_loops_keep_their_loads_in_flight(kernels):
    for name, (kind, body, scratch) in kernels.items():
        if kind == "join":
            assert scratch == 0, name
            continue
        assert scratch <= 64, f"{name}: {scratch} bytes of scratch per lane"
        for blk in re.split(r"\n(?=\.LBB)", body):
            ins = [l.strip() for l in blk.splitlines()[1:] if l.strip() and not l.strip().startswith((";", "."))]
            if sum(l.startswith("v_exp_f32") for l in ins) < 16 or sum("v_mfma" in l for l in ins) < 4:
                continue        # (a key block's scores, probabilities and products)
            assert not any(l.startswith(("scratch_", "buffer_")) for l in ins), name
            assert not any(re.search(r"s_waitcnt.*vmcnt\(0\)", l) for l in ins), name
