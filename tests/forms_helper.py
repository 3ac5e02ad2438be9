"""Which form of a kernel a call takes (csrc/forms.h), asked on the host at the sizes of the device's 152 SMs."""
from __future__ import annotations

import functools
import os
import subprocess
import tempfile
from collections import namedtuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SMS = 152

Linear = namedtuple("Linear", "tokens channels bn pair split")
Norm = namedtuple("Norm", "stream vectors warps teams two rows smem")
Rope = namedtuple("Rope", "stream full stages warps teams vectors tokens smem")

_PROGRAM = r"""
#include <stdio.h>
#include "forms.h"
using namespace ispa;
int main() {
  char kind;
  while (scanf(" %c", &kind) == 1) {
    long long a[11];
    for (int i = 0; i < 11; ++i)
      if (scanf("%lld", a + i) != 1) return 1;
    if (kind == 'L') {
      const LinearForm f = linear_i8_form(a[0], a[1], a[2], a[3]);
      printf("%d %d %d %d %d\n", f.tokens, f.channels, f.bn, f.pair, f.split);
    } else if (kind == 'N') {
      const NormForm f = norm_form(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
      printf("%d %d %d %d %d %lld %d\n", f.stream, f.vectors, f.warps, f.teams, f.two, (long long)f.rows, f.smem);
    } else {
      const int heads[2] = {(int)a[2], (int)a[3]}, norms[2] = {(int)a[4], (int)a[5]};
      const RopeForm f = rope_form(a[0], a[1], heads, norms, a[6], a[7], a[8], a[9], a[10]);
      printf("%d %d %d %d %d %d %lld %d\n", f.stream, f.full, f.stages, f.warps, f.teams, f.vectors, (long long)f.tokens,
             f.smem);
    }
  }
  return 0;
}
"""


_dir = None


@functools.cache
def _program() -> str:
    global _dir
    _dir = tempfile.TemporaryDirectory()      # as long as the module lives
    src, exe = os.path.join(_dir.name, "forms.cc"), os.path.join(_dir.name, "forms")
    with open(src, "w") as f:
        f.write(_PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2607_00712_gb300", "csrc"), src, "-o", exe], check=True)
    return exe


def _ask(kind, rows, as_type):
    lines = "\n".join(" ".join([kind] + [str(int(v)) for v in r] + ["0"] * (11 - len(r))) for r in rows)
    out = subprocess.run([_program()], input=lines, capture_output=True, text=True, check=True).stdout.splitlines()
    return [as_type(*map(int, line.split())) for line in out]


def linear(sizes):
    """sizes: (T, D, D_out)."""
    return _ask("L", [(*s, SMS) for s in sizes], Linear)


def norm(calls):
    """calls: (rows, dim, x_fp32, residual, post_bias, modulated, rows_per_group)."""
    return _ask("N", [(*c, SMS) for c in calls], Norm)


def rope(calls):
    """calls: (n, heads of each tensor, norms of each, head_dim, pairs, half)."""
    rows = []
    for n, heads, norms, d, pairs, half in calls:
        lanes = 1
        while 8 * lanes < d:
            lanes *= 2
        rows.append((n, len(heads), heads[0], heads[-1], norms[0], norms[-1], d, pairs, lanes, half, SMS))
    return _ask("R", rows, Rope)
