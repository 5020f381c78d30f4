"""The cache kernels' index arithmetic (csrc/cache_index.h), compiled for the host
and evaluated for every page and head size that the library takes."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2208_01944_amd", "csrc")
PAIRS = [(page, dim) for page in (16, 32, 64, 128) for dim in (64, 96, 128, 256)]


def evaluate(tmp_path, body):
    """The lines that a host program with `body` in its main prints, as lists of whole numbers."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(f'#include <cstdio>\n#include "cache_index.h"\nusing namespace palq;\nint main() {{\n{body}\nreturn 0;\n}}\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    return [[int(v) for v in line.split()] for line in out.splitlines()]


@pytest.fixture(scope="module")
def append_shapes(tmp_path_factory):
    rows = evaluate(tmp_path_factory.mktemp("append"), """
  for (int page : kPages)
    for (int dim : kDims) {
      const int n = append_rounds(page, dim);
      std::printf("%d %d %d %d %d %d %d\\n", page, dim, kAppendThreads, append_items(page, dim), n, turned_stride(page), turned_words(n));
    }""")
    assert [(r[0], r[1]) for r in rows] == PAIRS
    return {(r[0], r[1]): r[2:] for r in rows}


@pytest.mark.parametrize("page,dim", PAIRS)
def test_append_takes_every_value_of_a_block(append_shapes, page, dim):
    """Items of 4 tokens x 8 channels, thread by thread: every value of a block once, every word that is turned inside LDS."""
    threads, items, rounds, stride, words = append_shapes[page, dim]
    assert rounds in (1, 2, 4)
    seen, groups = set(), dim // 8
    for thread in range(threads):
        for i in range(rounds):
            p = thread + i * threads
            if p < items:
                tokens, channels = p // groups * 4, p % groups * 8
                seen |= {(t, c) for t in range(tokens, tokens + 4) for c in range(channels, channels + 8)}
                assert all(0 <= (channels + j) * stride + tokens // 4 < words for j in range(8))
    assert seen == {(t, c) for t in range(page) for c in range(dim)}
    assert (dim - 1) * stride + (page - 1) // 4 < words  # the last word read back
