"""The order of an attention's tiles with sinks (csrc/cache_index.h), compiled for the host."""
import pytest

from tests.test_cache_index_cpu import evaluate

TOP = 2 ** 31 - 1024  # the most tokens of a request


@pytest.mark.parametrize("hi", [0, 1, 63, 64, 65, 700, TOP])
@pytest.mark.parametrize("sinks", [0, 1, 64, 65, 2 ** 31 - 1])
def test_tiles_with_sinks(tmp_path, hi, sinks):
    """Every tile that holds a seen token once and in rising order, none other; the places that are asked for, eight past the
    last among them, are 32-bit ones, also where the range begins behind the last token."""
    los = [lo for lo in (0, 1, 64, 130, hi - 65, hi - 1, hi, hi + 1, 2 ** 31 - 1) if 0 <= lo < 2 ** 31]
    body = "".join(f"""
  {{ const TileOrder t = tile_order({lo}, {hi}, {sinks});
    std::printf("%d %d %lld\\n", t.count, t.sink, (long long)t.gap);
    for (long long i = 0; i < t.count + 9LL; i += (i < 20 || i > t.count - 20) ? 1 : 100003)
      std::printf("%lld %lld\\n", i, i < t.sink ? i : i + (long long)t.gap);
  }}""" for lo in los)
    lines, at = evaluate(tmp_path, body), 0
    for lo in los:
        count, sink, gap = lines[at]
        at += 1
        first = -(-min(sinks, hi) // 64) if hi > 0 else 0  # tiles of the first tokens
        rest = range(lo // 64, -(-hi // 64)) if hi > lo else range(0)
        assert count == min(first, lo // 64) + len(rest)
        if hi <= 700:
            assert [lines[at + i][1] for i in range(count)] == list(range(min(first, lo // 64))) + list(rest), (lo, hi, sinks)
        while at < len(lines) and len(lines[at]) == 2:
            i, place = lines[at]
            assert 0 <= place * 64 and place * 64 + 63 < 2 ** 31, (lo, hi, sinks, i)
            at += 1
