"""The row kernels touch an element of the logits, lone or at a row's ragged end, as its
own type (CPU only: hipcc's front end).

Listed tokens' gradients are stored over what the main pass wrote, one element over a
part of a vector, and logits may be overwritten in place.  The compiler keeps two such
accesses in order only if their types may alias: the same type, or the 16-byte vectors,
which alias everything.  Accesses through another scalar type of the same size (a bfloat16
as a short, a float as an int) it may exchange."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_12500_amd import build as B

pytestmark = pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which("hipcc")),
                                reason="hipcc not installed")


def global_accesses(ir, kernel):
    """{TBAA type name} of the kernel's accesses through pointers that are not LDS."""
    names = dict(re.findall(r'^(!\d+) = !\{!"([^"]+)", !\d+, i64 0\}', ir, re.M))
    tags = dict(re.findall(r"^(!\d+) = !\{(!\d+), !\d+, i64 0\}", ir, re.M))
    body = re.findall(r"^define [^\n]*" + kernel + r"[^\n]*\{\n(.*?)^\}", ir, re.M | re.S)
    assert body, kernel
    used = set()
    for line in body[0].splitlines():
        m = re.search(r"(?:load|store) (i16|i32|half|bfloat|float)\b.*!tbaa (!\d+)", line)
        if m and m.group(2) in tags:
            used.add((m.group(1), names.get(tags[m.group(2)])))
    return used


@pytest.mark.parametrize("what,dtype,own", [("load_part", 1, "_Float16"), ("load_part", 2, "__bf16"),
                                            ("load_part", 3, "float"), ("store", 1, "_Float16"),
                                            ("store", 2, "__bf16"), ("store", 3, "float")])
def test_parts_of_vectors_are_of_the_elements_type(tmp_path_factory, what, dtype, own):
    where = tmp_path_factory.mktemp("types")
    src, out = str(where / "part.hip"), str(where / "part.ll")
    with open(src, "w") as f:
        f.write(f"""#include "logits_rows.h"
typedef logits::Segment<{dtype}, 2> S;
typedef logits::Elem<{dtype}>::type T;
extern "C" __global__ void load_part(const T* p, int n, symtile::u32x4* r) {{ *r = S::load_part(p, n); }}
extern "C" __global__ void store(T* p, int len, int at, symtile::u32x4 v) {{ S::store(p, len, at, v); }}
""")
    cmd = [B.HIPCC, *[f for f in B.CXXFLAGS if f != "-O3"], "-O1", "-S", "-emit-llvm",
           "--cuda-device-only", src, "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        names = {name for _, name in global_accesses(f.read(), what)}
    assert names and names <= {own, "omnipotent char"}      # (of a copy of the bytes)
