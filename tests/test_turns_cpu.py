"""Frequencies as turns (csrc/turns.h), compiled for the host, against whole numbers of any size."""
import math
import subprocess

import numpy as np

from tests.test_cache_index_cpu import CSRC


def arctan_of_one_over(n, one):
    t, s, k = one // n, one // n, 1
    while t:
        t //= n * n
        k += 2
        s += -(t // k) if k % 4 == 3 else t // k
    return s


BITS = 2600  # places that are kept: 2^1024 turns and some more
ONE = 1 << BITS
PI = 4 * (4 * arctan_of_one_over(5, ONE) - arctan_of_one_over(239, ONE))  # (Machin)


def test_pi():
    assert PI / ONE == math.pi and abs(PI / ONE - math.pi) < 1e-15


def test_turns_are_the_nearest(tmp_path):
    """Small, usual and huge frequencies of either sign, those of half a turn and more among them: never more than half a unit of
    2^-64 turns off."""
    g = np.random.default_rng(0)
    f = np.concatenate([10000.0 ** -(np.arange(128) / 128), g.uniform(0, 2 * np.pi, 2000), g.uniform(np.pi, 1e3, 1000), np.exp(g.uniform(-745, 709, 2000)),
                        2.0 ** np.arange(-1074, 1024), 2 * np.pi * np.arange(1, 20), 5e-324 * np.arange(4), [1.7976931348623157e308]])
    f = np.concatenate([f, -f, -np.exp(g.uniform(-45, -25, 2000))])
    (tmp_path / "f").write_bytes(f.tobytes())
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include <cstdio>\n#include "turns.h"\nint main() {\n  double f;\n  while (std::fread(&f, 8, 1, stdin) == 1) '
                   'std::printf("%llu\\n", (unsigned long long)palq::turns_of(f));\n}\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error", "-I",
                    CSRC, str(src), "-o", str(exe)], check=True)
    with open(tmp_path / "f", "rb") as stdin:
        got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True, stdin=stdin).stdout.split()]
    assert len(got) == len(f)
    for x, t in zip(f, got):
        n, d = float(x).as_integer_ratio()
        exact = (n * ONE * ONE << 64) // (d * 2 * PI)       # turns in 2^-64, with BITS places
        off = (exact - (t << BITS)) % (ONE << 64)
        off = min(off, (ONE << 64) - off)
        assert off <= ONE // 2 + (ONE >> 60), (x, t, off / ONE)
