"""Sizes that the library's 31 bits do not hold are refused, not cut to what is left of them."""
import pytest
import torch

LONG = 2 ** 32 + 8


def test_rows_longer_than_31_bits_are_refused():
    from paper_2405_18428_b200 import build, dig
    build.build()
    x = torch.zeros(1, 1).expand(1, LONG)
    for call in (lambda: dig.dig_layernorm_fwd(x), lambda: dig.dig_layernorm_bwd(x, x), lambda: dig.dig_gla_outgate_fwd(x, x, None, None, 1e-5),
                 lambda: dig.dig_gla_outgate_bwd(x, x, x, None, None, 1e-5)):
        with pytest.raises(ValueError, match="too large"):
            call()


@pytest.mark.gpu
def test_batches_beyond_31_bits_are_refused():
    from paper_2405_18428_b200 import dig
    z = torch.zeros(1, 2, 2, 8, device="cuda")
    many = z.expand(2 ** 32 + 1, 2, 2, 8)
    pos = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    for call in (lambda: dig.dig_decay_fwd(many, many, many, [0.0, 0.0], 1, 2), lambda: dig.dig_rope(many, None, pos, [1.0], [0]),
                 lambda: dig.dig_layernorm_fwd(z, torch.zeros(1, 8, device="cuda").expand(2 ** 32 + 1, 8))):
        with pytest.raises(ValueError, match="too large"):
            call()
