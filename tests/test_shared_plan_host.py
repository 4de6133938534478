"""The shapes that the GPU tests of large row tiles use take those kernels (the plan, compiled for the CPU)."""
import pytest

import shared_harness as P


@pytest.mark.parametrize("kind", P.KINDS)
def test_shapes_of_large_tiles_take_their_kernels(kind):
    dtype, d, waves = kind
    for G, H, groups in P.shapes(kind):
        for behind in (0, 2) if len(groups) > 1 else (0,):
            for counts in ([0], [70000]):        # with as few entries as the tests have, and with many
                got = P.kernel(dtype, d, G, H, sum(groups) + behind, len(groups), P.rows_of(G, groups, counts))
                assert got == ("many", waves), (kind, G, H, groups)


@pytest.mark.parametrize("kind", P.KINDS)
def test_shapes_cover_what_they_say(kind):
    assert len(P.many_units(kind)[2]) * P.many_units(kind)[0] > 64
    G, H, groups, counts = P.deep(kind)
    # row tiles times key tiles, against the places that the grid has for them
    R, keys, places = (128, 128, 256) if kind[2] == 8 else (64, 128, 256) if kind[0] == "bf16" else (64, 32, 512)
    tiles = [-(-m * (H // G) // R) for m in groups]
    assert sum(t * -(-n // keys) for t, n in zip(tiles, counts)) > places - sum(tiles)       # chunks of several key tiles
    assert len(groups) * G <= 64
