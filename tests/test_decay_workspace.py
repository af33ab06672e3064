"""Workspace of linear attention with a decay for each head: a few machines full of segments' states, however long the sequences are."""
import pytest


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("backward", [0, 1])
def test_states_of_a_bounded_number_of_segments(dtype, backward):
    from paper_2405_18428_b200 import build, dig
    build.build()
    assert (dig.DIG_F32, dig.DIG_BF16) == (0, 1)
    tile, passes = (128 if dtype == dig.DIG_BF16 else 64), 3 if backward else 1
    far_below_the_finest = 0
    for B, H in ((1, 1), (1, 6), (1, 16), (4, 12), (5, 16), (40, 16)):
        for L in (1, 64, 129, 1000, 4096, 1 << 14, 1 << 17, 1 << 20, 1 << 24):
            for d in (64, 72, 128):
                # cuts are tried until three rounds of two CTAs on 148 SMs are full; from one number of tiles for each segment to the next the number of
                # segments at most doubles; a sequence more or less on top
                segments = 2 * (3 * 2 * 148 // passes + B * H)
                # entering states of one or two passes, final states
                most = 3 * (segments * d * d * 4 + 256)
                got = dig.dig_decay_workspace_bytes(B, H, H, 1, L, d, d, dtype, backward)
                assert 0 < got <= most, (B, H, L, d, got, most)
                far_below_the_finest += most < B * H * (L // tile) * d * d * 4
    assert far_below_the_finest > 40         # cuts of a tile each would not pass
