"""A check of the gfx950 assembly of the operators at a model's two ends (CPU only: hipcc
cross-compiles the kernel sources).

A store of more than 8 bytes reads its data registers over several cycles after it is
issued; a vector instruction right behind it must not write them.  The compiler puts a
wait state there, but not behind a buffer store with a scalar offset register, where it
takes none to be needed: there the store has written the later value of some lanes' first
word (a sum's registers cleared right after the sum was stored).  So no such store may be
followed at once by a write of its data."""
import concurrent.futures as cf
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_12500_amd import build as B

pytestmark = pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which("hipcc")),
                                reason="hipcc not installed")

SOURCES = ("mx4.hip", "verify_draft.hip", "embedding.hip")


def registers(text):
    out = set()
    for kind, a, b, kind1, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out |= {(kind1, int(one))} if kind1 else {(kind, i) for i in range(int(a), int(b) + 1)}
    return out


def overwritten_stores(asm):
    """(kernel, store, instruction) where the instruction behind a wide store writes its data."""
    bad, kernel, stored = [], None, None
    for line in asm.splitlines():
        s = line.split(";")[0].strip()
        m = re.match(r"(_Z\w+):", s)
        if m:
            kernel, stored = m.group(1), None
            continue
        if not s or s.startswith((".", "/")):
            continue                       # (a label does not wait)
        op, _, args = s.partition(" ")
        writes = op.startswith("v_") and not op.startswith(("v_cmp", "v_readlane", "v_readfirstlane"))
        if stored and writes and registers(args.split(",")[0]) & stored[1]:
            bad.append((kernel, stored[0], s))
        stored = None
        if re.match(r"(buffer|global|flat)_store_dwordx[34]", op):
            parts = args.split(",")
            stored = (s, registers(parts[0 if op.startswith("buffer") else 1]))
    return bad


def test_the_scan_finds_a_write_behind_a_store():
    store = "\tbuffer_store_dwordx4 v[2:5], v1, s[4:7], s36 offen sc0 sc1\n"
    assert len(overwritten_stores("_Zk:\n" + store + ".LBB0_1:  ; x\n\tv_mov_b32_e32 v2, 0\n")) == 1
    assert not overwritten_stores("_Zk:\n" + store + "\ts_nop 0\n\tv_mov_b32_e32 v2, 0\n")
    assert not overwritten_stores("_Zk:\n" + store + "\tv_mov_b32_e32 v6, v2\n")


def test_no_wide_store_is_overwritten(tmp_path):
    def compile_(src):
        out = str(tmp_path / (src + ".s"))
        r = subprocess.run([B.HIPCC, *B.CXXFLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, src),
                            "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        with open(out) as f:
            return f.read()
    with cf.ThreadPoolExecutor(max_workers=3) as ex:
        for src, asm in zip(SOURCES, ex.map(compile_, SOURCES)):
            assert asm.count("_store_dwordx4") > 10
            assert overwritten_stores(asm) == [], src
