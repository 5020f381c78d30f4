"""The tiles of an attention's rows with sinks (csrc/cache_index.h), compiled for the host,
against the set of the tokens that the rows see."""
import pytest

from tests.test_cache_index_cpu import evaluate

TOP = 2 ** 31 - 1024  # the most tokens of a request


@pytest.mark.parametrize("hi", [0, 1, 40, 63, 64, 65, 90, 128, 129, 700])
def test_tiles_hold_what_is_seen(tmp_path, hi):
    """Every tile with a token j that a row of range [lo, hi) and some first tokens sees (lo <= j < hi or j < min(sinks, hi)),
    once and in order, and no other; also where the window begins behind the last token."""
    cases = [(lo, sinks) for lo in (0, 1, 39, 40, 50, 63, 64, 90, 100, 128, 130, 200, 699, 700, 701, 2 ** 31 - 1)
             for sinks in (0, 1, 4, 64, 65, 100, 200, 2 ** 31 - 1)]
    lines = evaluate(tmp_path, "".join(f"""
  {{ const TileOrder t = tiles_seen({lo}, {hi}, {sinks});
    for (int i = 0; i < t.count; ++i) std::printf("%d ", t.at(i));
    std::printf("\\n"); }}""" for lo, sinks in cases))
    for (lo, sinks), got in zip(cases, lines):
        assert got == sorted({j // 64 for j in range(hi) if j >= lo or j < min(sinks, hi)}), (lo, hi, sinks)


@pytest.mark.parametrize("hi", [1, 65, TOP - 1, TOP])
def test_places_past_the_last_tile(tmp_path, hi):
    """Tiles that are asked for ahead, eight past the last, have 32-bit places."""
    cases = [(lo, sinks) for lo in (0, 64, hi - 1, hi, TOP, 2 ** 31 - 1) for sinks in (0, 1, 65, TOP, 2 ** 31 - 1)]
    for (lo, sinks), (count, place) in zip(cases, evaluate(tmp_path, "".join(f"""
  {{ const TileOrder t = tiles_seen({lo}, {hi}, {sinks});
    const long long i = t.count + 8LL;
    std::printf("%d %lld\\n", t.count, i < t.sink ? i : i + t.gap); }}""" for lo, sinks in cases))):
        assert 0 <= place * 64 and place * 64 + 63 < 2 ** 31, (lo, hi, sinks)
