"""min-p's border of a row (the least float whose distance from the largest
logit is within T ln(min_p)), compiled for the host: the definition at pairs
that cancel, at the type's ends and at random ones, within a bounded number of
steps (no GPU)."""
import os
import subprocess

import pytest

from paper_2010_03166_amd import build

# 2,000 pairs of whole numbers (a border next to 0), each of which takes some
# 6e8 steps, seconds, where every float on the way is looked at; then others.
SOURCE = r"""
#include <cstdio>
#include <random>
#include "choose.hpp"
using gnnprop::least_near;

static long wrong = 0, done = 0;
static void check(float top, double cut) {
  const float z = least_near(top, cut);
  const float below = nextafterf(z, -INFINITY);
  const bool ok = z <= top && (double)z - top >= cut && !((double)below - top >= cut);
  if (!ok && wrong++ < 10) printf("top %a cut %a: %a\n", top, cut, z);
  ++done;
}

int main() {
  for (int k = 1; k <= 2000; ++k) check((float)k, -(double)k);
  for (double T : {0.25, 0.5, 1.0, 2.0, 3.0})
    for (int k = 1; k <= 100; ++k) check((float)(T * k), T * std::log(std::exp(-(double)k)));
  const float ends[] = {3.4028234e38f, -3.4028234e38f, 1e-45f, -1e-45f, 0.f, -0.f, 1.1754944e-38f};
  for (float top : ends)
    for (double cut : {0.0, -1e-300, -1e-50, -1.4e-45, -1.0, -7e8, -3.4028234663852886e38})
      check(top, cut);
  std::mt19937_64 r(1);
  std::uniform_real_distribution<double> unit(0.0, 1.0);
  for (int k = 0; k < 2000000; ++k) {
    const float top = (float)((unit(r) - 0.5) * std::pow(10.0, 12 * unit(r) - 6));
    check(top, std::pow(10.0, 4 * unit(r) - 2) * std::log(unit(r) + 1e-18));
    check(top, -(double)top < 0 ? -(double)top : (double)top);
    check(top, -std::fabs((double)top) * (1 + (unit(r) - 0.5) * 1e-15));
  }
  printf("%ld pairs, %ld wrong\n", done, wrong);
  return wrong != 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("border")
    src, exe = str(at / "border.hip"), str(at / "border")
    with open(src, "w") as f:
        f.write(SOURCE)
    r = subprocess.run([build.hipcc(), "--offload-host-only", "-O2", "-std=c++17",
                        "-I", build.INCLUDE, "-I", build.CSRC, src, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return exe


def test_border_of_min_p_is_the_definitions_and_found_in_few_steps(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=60,
                       env=dict(os.environ, HIP_VISIBLE_DEVICES=""))
    assert r.returncode == 0, r.stdout + r.stderr
