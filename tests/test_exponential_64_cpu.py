"""The sampler's 64-bit exponential (csrc/k_exp.h), built for the CPU, against the library's in 64 bits."""
import os
import subprocess

import numpy as np

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_18489_amd", "csrc")
MAIN = r"""
#include <math.h>
#include <stdio.h>
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_exp2f exp2f
#include "k_exp.h"
int main() {
  double t;
  while (fread(&t, 8, 1, stdin) == 1) {
    const double e = ec::exp2_times_2to46(t);
    const unsigned long long w = ec::exp2_fixed46(t);
    fwrite(&e, 8, 1, stdout);
    fwrite(&w, 8, 1, stdout);
  }
}
"""


def test_formula(tmp_path):
    """3.7e-14 relative from the polynomial, up to a dozen roundings of 2^-53 (1.3e-15) and, of the argument t + 46 that the library's 2^t is
    given here, 2^-48 ln 2 (2.5e-15): 4.1e-14.  The whole number is off by at most 1/2 more."""
    (tmp_path / "main.cpp").write_text(MAIN)
    subprocess.check_call(["g++", "-O1", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "exp")])
    rng = np.random.default_rng(7)
    t = np.concatenate((-rng.uniform(0, 60, 50000), -rng.uniform(0, 1, 50000), [0.0, -0.5, -1.0, -46.0, -47.0, -48.0, -200.0, -1e9, -np.inf]))
    out = subprocess.run([str(tmp_path / "exp")], input=t.tobytes(), stdout=subprocess.PIPE, check=True).stdout
    e, w = np.frombuffer(out, dtype=np.float64)[::2], np.frombuffer(out, dtype=np.uint64)[1::2].astype(np.float64)
    want = np.exp2(t + 46)
    seen = t > -200
    assert np.abs(e[seen] / want[seen] - 1).max() < 4.1e-14
    assert (np.abs(w - want) <= 0.5 + 4.1e-14 * want).all()
    assert w[100000] == 2.0 ** 46 and w[100002] == 2.0 ** 45 and (w[-3:] == 0).all()
