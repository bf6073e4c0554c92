"""The waits of the wide attention kernels' loop, on a model of a wave's copies."""

import pytest

from test_gpu_short_parts import waits


@pytest.mark.parametrize("wave", [0, 1])
def test_every_copy_has_landed(wave):
    for tiles in range(1, 40):
        for plain in range(tiles + 1):
            assert waits(tiles, plain, wave, True) == [], (tiles, plain)


@pytest.mark.parametrize("wave", [0, 1])
def test_without_the_rule_short_items_miss_v(wave):
    found = {t for t in range(1, 40) for plain in range(t + 1) if waits(t, plain, wave, False)}
    assert found == {2, 3}
    assert set(waits(3, 3, wave, False)) == {("V", 1)}
