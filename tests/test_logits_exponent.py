"""The exponent that the row kernels compute (csrc/logits_rows.h), on the host: the
same code, compiled for the CPU, over all largest logits that bfloat16 has.

A row's sums hold 2^y with y = scale log2(e) (x - m) + shift, and the shift is taken
out of them afterwards: it has to stay a fraction of one, whatever m, or the sums
overflow, vanish, or lose the entropy's digits."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2511_12500_amd import build as B

pytestmark = pytest.mark.skipif(not (os.path.exists(B.HIPCC) or shutil.which("hipcc")),
                                reason="hipcc not installed")

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "logits_rows.h"
int main() {
    float in[3];   // largest logit, scale, another logit
    while (std::fread(in, 4, 3, stdin) == 3) {
        const logits::Exponent ex(in[0], in[1]);
        const float m = in[0] == -logits::kInf ? 0.0f : in[0];
        const float out[4] = {(float)ex.huge, ex.shift, ex.huge ? ex.y<true>(m) : ex.y<false>(m),
                              ex.huge ? ex.y<true>(in[2]) : ex.y<false>(in[2])};
        std::fwrite(out, 4, 4, stdout);
    }
}
"""


@pytest.fixture(scope="module")
def exponent(tmp_path_factory):
    """f(m, scale, x) -> (huge, shift, y(m), y(x)) of fp32 arrays."""
    where = tmp_path_factory.mktemp("exponent")
    src, exe = str(where / "exponent.hip"), str(where / "exponent")
    with open(src, "w") as f:
        f.write(PROGRAM)
    r = subprocess.run([B.HIPCC, *B.CXXFLAGS, src, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def call(m, scale, x):
        rows = np.stack(np.broadcast_arrays(m, scale, x), axis=-1).astype(np.float32)
        r = subprocess.run([exe], input=rows.tobytes(), capture_output=True)
        assert r.returncode == 0
        return np.frombuffer(r.stdout, np.float32).reshape(-1, 4).T
    return call


SCALES = np.float32([1e-38, 1e-30, 1e-3, 0.25, 0.7, 1.0, 1.25, 2.0, 17.0, 1e6, 1e30, 2.4e38, 3.4e38])


def largest():
    m = (np.arange(1 << 16, dtype=np.uint32) << 16).view(np.float32)
    return m[np.isfinite(m)]


@pytest.mark.parametrize("scale", SCALES, ids=lambda s: f"{s:g}")
def test_the_shift_is_a_fraction_of_one(exponent, scale):
    m = largest()
    huge, shift, own, masked = exponent(m, scale, -np.inf)
    assert np.abs(shift).max() <= 0.125
    assert np.array_equal(own, shift)             # the largest logit's own term is 2^shift
    assert (masked == -np.inf).all()
    # logits of a usual size take the shorter way (where scale log2(e) is a number)
    assert scale > 2.3e38 or not huge[np.abs(m.astype(np.float64) * scale) < 1e6].any()


@pytest.mark.parametrize("scale", SCALES, ids=lambda s: f"{s:g}")
def test_the_exponent_of_another_logit(exponent, scale):
    """y - shift against 64 bits: three roundings, or the smallest numbers' absolute error."""
    rng = np.random.default_rng(1)
    m = largest()
    m = m[np.abs(m) >= 2.0 ** -100]
    with np.errstate(over="ignore"):
        x = (m - np.abs(m) * rng.choice([0.0, 1e-6, 1e-3, 0.5, 2.0], m.size)
             - rng.random(m.size) * rng.choice([0.0, 1.0 / scale], m.size)).astype(np.float32)
    x = np.where(np.isfinite(x), np.minimum(x, m), np.float32(-3.4e38)).astype(np.float32)
    _, shift, _, y = exponent(m, scale, x)
    want = (x.astype(np.float64) - m.astype(np.float64)) * float(scale) * np.log2(np.e)
    near = want > -1e4        # where 2^y is a number at all
    # the rounding of y, which holds the shift; the difference's, the constants' and the products';
    # a product below the smallest normal number is off by 2^-150
    bound = 2.0 ** -24 * (0.25 + 5 * np.abs(want)) + 2.0 ** -149
    # the constant scale log2(e) of a scale near the smallest number is itself off by 2^-150
    bound = bound + np.abs(want) * (2.0 ** -149 / (float(scale) * 1.44))
    err = np.abs(y.astype(np.float64) - shift.astype(np.float64) - want)
    assert (err[near] <= bound[near]).all(), (m[near][np.argmax((err - bound)[near])])
    assert (y[~near] < -9000).all()
