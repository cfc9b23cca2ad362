"""A check of the gfx950 assembly of all kernels (CPU only: hipcc cross-compiles them): the
data of a store of more than 8 bytes is not overwritten before the store has read it.

Two wait states have to lie between such a store and a vector instruction that writes its data
registers; the compiler puts them there itself, but not behind a buffer store with a scalar
offset register (tests/test_store_hazards.py has what happened then).  Followed are all ways
from a store, over branches too, and both registers that a swap writes."""
import concurrent.futures as cf
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_12500_amd import build as B
from tests.test_store_hazards import registers

pytestmark = pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which("hipcc")),
                                reason="hipcc not installed")

WAIT_STATES = 2


def written(op, args):
    """Vector registers that a vector instruction writes (none for others)."""
    if not op.startswith("v_") or op.startswith(("v_cmp", "v_readlane", "v_readfirstlane")):
        return set()
    out = registers(args[0])
    if op.startswith(("v_swap", "v_permlane16_swap", "v_permlane32_swap")):
        out |= registers(args[1])
    return out


def functions(asm):
    """(name, instructions, index of each label) of every function."""
    name, code, labels = None, [], {}
    for line in asm.splitlines():
        s = line.split(";")[0].strip()
        m = re.match(r"([.\w$]+):", s)
        if m and not s.startswith("."):
            if code:
                yield name, code, labels
            name, code, labels = m.group(1), [], {}
        elif m:
            labels[m.group(1)] = len(code)
        elif s and not s.startswith((".", "/")):
            op, _, args = s.partition(" ")
            code.append((op, [a.strip() for a in args.split(",")]))
    if code:
        yield name, code, labels


def overwritten(asm):
    """(function, store, instruction) where the data is written too early on some way."""
    bad = []
    for name, code, labels in functions(asm):
        for i, (op, args) in enumerate(code):
            if not re.match(r"(buffer|global|flat|scratch)_store_dwordx[34]", op):
                continue
            data = registers(args[0 if op.startswith("buffer") else 1])
            ways = [(i + 1, 0)]
            while ways:
                at, waited = ways.pop()
                if waited >= WAIT_STATES or at >= len(code):
                    continue
                next_op, next_args = code[at]
                if written(next_op, next_args) & data:
                    bad.append((name, (op, args), (next_op, next_args)))
                if next_op in ("s_endpgm", "s_setpc_b64"):
                    continue
                waited += int(next_args[0], 0) + 1 if next_op == "s_nop" else 1
                if next_op.startswith(("s_branch", "s_cbranch")):
                    ways.append((labels[next_args[0]], waited))
                if next_op != "s_branch":
                    ways.append((at + 1, waited))
    return bad


STORE = "\tbuffer_store_dwordx4 v[2:5], v1, s[4:7], s36 offen sc0 sc1\n"


@pytest.mark.parametrize("behind,found", [
    ("\tv_mov_b32_e32 v2, 0\n", 1),
    ("\ts_nop 0\n\tv_mov_b32_e32 v5, 0\n", 1),
    ("\ts_nop 1\n\tv_mov_b32_e32 v5, 0\n", 0),
    ("\ts_add_i32 s0, s0, 1\n\ts_add_i32 s0, s0, 1\n\tv_mov_b32_e32 v2, 0\n", 0),
    ("\tv_mov_b32_e32 v6, v2\n", 0),
    ("\tv_swap_b32 v9, v3\n", 1),
    ("\tv_permlane32_swap_b32_e32 v9, v4\n", 1),
    ("\tv_permlane16_swap_b32_e32 v9, v10\n", 0),
    ("\ts_endpgm\n.L2:\n\tv_mov_b32_e32 v2, 0\n", 0),
    ("\ts_branch .L1\n\tv_mov_b32_e32 v2, 0\n", 1),          # (at .L1: v5)
    ("\ts_cbranch_scc0 .L1\n\tv_mov_b32_e32 v2, 0\n", 2),
    ("\ts_cbranch_scc0 .L1\n\ts_nop 0\n\tv_mov_b32_e32 v2, 0\n", 1)])
def test_the_scan(behind, found):
    assert len(overwritten("_Zk:\n.L1:\n\tv_mov_b32_e32 v5, 0\n\ts_nop 0\n\ts_nop 0\n" + STORE + behind)) == found


def test_no_kernel_overwrites_a_stores_data(tmp_path):
    def compile_(src):
        out = str(tmp_path / (src + ".s"))
        r = subprocess.run([B.HIPCC, *B.CXXFLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, src),
                            "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        with open(out) as f:
            return f.read()
    stores = 0
    # (the largest source first)
    sources = sorted(B.SOURCES, key=lambda s: -os.path.getsize(os.path.join(B.CSRC, s)))
    with cf.ThreadPoolExecutor(max_workers=4) as ex:
        for src, asm in zip(sources, ex.map(compile_, sources)):
            stores += asm.count("_store_dwordx4")
            assert overwritten(asm) == [], src
    assert stores > 1000
