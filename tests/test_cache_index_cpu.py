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


@pytest.fixture(scope="module")
def tile_shapes(tmp_path_factory):
    """{dim: pieces} and {(page, dim): offsets} of attend_tile_kernel's loads, thread after thread, for every tile of a page."""
    rows = evaluate(tmp_path_factory.mktemp("tile"), """
  for (int shift = 4; shift <= 7; ++shift)
    for (int dim : kDims)
      for (int tile = 0; tile == 0 || tile < 1 << shift; tile += 64)
        for (int n = 0; n < (4 * dim + kTileThreads - 1) / kTileThreads * kTileThreads; ++n) {
          const int page = 1 << shift, mask = page < 64 ? page - 1 : 63;
          const TilePiece p = tile_piece(n, dim);
          std::printf("%d %d %d %d %u %u %d %d %d %d %d\\n", page, dim, n, tile_piece_past(n, dim), tile_key_at(p, tile, mask, dim),
                      tile_value_at(p, tile, mask, shift), p.tok, p.s, p.kr, p.d, p.vt);
        }""")
    out = {}
    for r in rows:
        out.setdefault((r[0], r[1]), []).append(r[2:])
    assert sorted(out) == PAIRS
    return out


@pytest.mark.parametrize("page,dim", PAIRS)
def test_tile_loads_stay_inside_a_block(tile_shapes, page, dim):
    """Loads of every thread, those without a piece among them, lie in the block of page x dim bytes; the pieces that count
    are the whole tile, each once, and each key piece has a place of its own."""
    block = page * dim
    for n, past, key, value, *_ in tile_shapes[page, dim]:
        assert 0 <= key <= block - 16 and 0 <= value <= block - 16, n
    tiles = max(1, page // 64)
    real = [r for r in tile_shapes[page, dim] if not r[1]]
    assert len(real) == 4 * dim * tiles
    real = real[:4 * dim]
    assert {(tok, s) for *_, tok, s, kr, d, vt in real} == {(t, s) for t in range(64) for s in range(dim // 16)}
    assert {(kr, s) for *_, tok, s, kr, d, vt in real} == {(t, s) for t in range(64) for s in range(dim // 16)}
    assert {(d, vt) for *_, tok, s, kr, d, vt in real} == {(d, t) for d in range(dim) for t in range(0, 64, 16)}
