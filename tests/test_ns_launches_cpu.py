"""The sizes that the GPU tests run reach every launch that the plans reach (host code only)."""
import pytest

import ns_launches


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    exe = ns_launches.compiled(str(tmp_path_factory.mktemp("plans")))
    if exe is None:
        pytest.skip("g++ not found")
    return exe


def test_tested_sizes_reach_every_launch(exe):
    """400000 sizes over the range: a class that only they reach wants a size in the list."""
    tested = set()
    for batch, m, n, f32 in ns_launches.SIZES:
        got = ns_launches.classes(exe, batch, m, n, int(f32))
        assert got and got == ns_launches.classes(exe, batch, n, m, int(f32))
        tested |= got
    assert len(tested) >= 80
    for seed in (1, 2):
        missing = ns_launches.classes(exe, seed, 200000) - tested
        assert not missing, sorted(missing)


def test_every_tile_is_tested_with_and_without_running_on(exe):
    tested = set()
    for batch, m, n, f32 in ns_launches.SIZES:
        tested |= ns_launches.classes(exe, batch, m, n, int(f32))
    for product in range(3):
        # one part: all five (256 x 128 of B X behind larger ones only); two parts: up to 128 x 128
        assert {c[3] for c in tested if c[0] == product and c[1] == 1} == {0, 1, 2, 3, 4}
        assert {c[3] for c in tested if c[0] == product and c[1] == 2} == {0, 1, 2}
        assert {c[4] for c in tested if c[0] == product and c[1] == 1} == {0, 1, 2}
        for tile in (0, 2, 4):
            assert {c[5] for c in tested if c[0] == product and c[3] == tile} == {0, 1}
