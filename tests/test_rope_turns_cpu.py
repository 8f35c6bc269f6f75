"""Frequencies of the rotary positions as 64-bit fractions of a turn, and cosines and sines at the far ends of the positions
(functions of the CUDA sources that also compile for the host), against exact fractions (CPU only; needs nvcc)."""
import decimal
import math
import random
import subprocess
from fractions import Fraction as F

import pytest

from paper_2609_29029_gb300 import build

PI = F("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")

PROGRAM = r"""
#include <cstdio>
#include "rope_angle.cuh"
int main() {
  rift_rope_spec s = {};
  int n;
  s.scaling = RIFT_ROPE_LINEAR;
  while (scanf("%d %lf %lf %d", &s.rot_dim, &s.theta, &s.factor, &n) == 4) {
    double w[RIFT_ROPE_MAX_HEAD_DIM / 2];
    rift::rope_frequencies(s, w);
    for (int j = 0; j < s.rot_dim / 2; ++j) {
      const uint64_t f = rift::turns_of(w[j]);
      printf("%a %llu", w[j], (unsigned long long)f);
      for (long long p : {(long long)n, 2147483647LL, -2147483648LL, 1073741825LL}) {
        const float2 v = rift::cos_sin_of_turns((uint64_t)p * f, {1.f, 0.f});
        printf(" %a %a", v.x, v.y);
      }
      printf("\n");
    }
  }
}
"""


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    """(rot_dim, theta, factor, p, j, w, f, [(cos, sin) at p, 2^31 - 1, -2^31, 2^30 + 1])"""
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("turns")
    (d / "turns.cu").write_text(PROGRAM)
    subprocess.run([nvcc, "-std=c++17", "-O2", "--expt-relaxed-constexpr", "-I", str(build.ROOT / "include"), "-I",
                    str(build.CSRC), *build.ARCH, str(d / "turns.cu"), "-o", str(d / "turns")], check=True, capture_output=True)
    rng = random.Random(3)
    specs = [(rot, theta, factor, rng.randrange(-2 ** 31, 2 ** 31)) for rot in (256, 128, 96, 58, 2)
             for theta in (1e4, 5e5, 1e7, 3.7e11) for factor in (1.0, 40.0)]
    specs += [(128, 1.0, 1.0, 77), (64, 1e-3, 1.0, -5), (128, 1e-9, 1.0, 9), (128, 1e300, 1.0, 1 << 30), (128, 1e4, 1e-5, 12345)]
    text = "".join("%d %r %r %d\n" % s for s in specs)
    lines = iter(subprocess.run([str(d / "turns")], input=text, check=True, capture_output=True, text=True).stdout.splitlines())
    out = []
    for rot, theta, factor, p in specs:
        for j in range(rot // 2):
            x = next(lines).split()
            v = [float.fromhex(y) for y in x[2:]]
            out.append((rot, theta, factor, p, j, float.fromhex(x[0]), int(x[1]), list(zip(v[::2], v[1::2]))))
    return out


def test_frequencies(rows):
    """theta^(-2j / rot_dim) / factor to (8 + |ln theta|) 2^-53 of itself."""
    with decimal.localcontext() as c:
        c.prec = 60
        for rot, theta, factor, _, j, w, _, _ in rows:
            want = (decimal.Decimal(theta).ln() * (-2 * j) / rot).exp() / decimal.Decimal(factor)
            assert abs(decimal.Decimal(w) - want) <= want * decimal.Decimal((8 + abs(math.log(theta))) * 2.0 ** -53), (rot, theta, j)


def test_turns_are_the_nearest(rows):
    """2^64 w / 2 pi (mod 2^64), rounded once: half a unit, and what two doubles leave of 1 / 2 pi."""
    for rot, theta, factor, _, j, w, f, _ in rows:
        off = (F(w) * 2 ** 64 / (2 * PI) - f) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= F(1, 2) + F(1, 2 ** 10), (rot, theta, j)


def test_cos_sin_at_far_positions(rows):
    """Any int32 position: |got - want| <= half an fp32 step + 2^-34 + |p| 2^-62."""
    for rot, theta, factor, n, j, w, _, got in rows:
        for p, (c, s) in zip((n, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1), got):
            a = 2 * math.pi * float((F(w) * p / (2 * PI) + F(1, 2)) % 1 - F(1, 2))
            for have, want in ((c, math.cos(a)), (s, math.sin(a))):
                step = 2.0 ** max(math.frexp(want)[1] - 24, -149)
                assert abs(have - want) <= step / 2 + 2.0 ** -34 + abs(p) * 2.0 ** -62 + 1e-15, (rot, theta, j, p)
