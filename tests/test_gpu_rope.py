"""Rotary positions with several axes on the GPU against complex products in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def turned(x, positions, freqs, axes, interleaved, inverse):
    x = x.double().cpu()
    n = len(freqs)
    angle = positions.cpu().double()[..., list(axes)] * torch.tensor(freqs, dtype=torch.float64)
    z = torch.polar(torch.ones_like(angle), -angle if inverse else angle).unsqueeze(-2)
    y = x.clone()
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    r = torch.complex(a.contiguous(), b.contiguous()) * z
    if interleaved:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = r.real, r.imag
    else:
        y[..., :n], y[..., n:2 * n] = r.real, r.imag
    return y


def close(got, ref, x, dtype):
    # angles are within 2e-7 (fp32 of a turn's fraction, sine and cosine), then two products and a sum, and the result's rounding
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    size = x.double().abs().cpu().amax(-1, keepdim=True) * 2
    lim = half * ref.abs() + 1e-6 * size
    assert ((got.double().cpu() - ref).abs() <= lim).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs", [(64, (16, 16)), (72, (18, 18)), (72, (6, 15, 15)), (128, (64,)), (8, (2, 2)), (8, (1, 1)), (40, (5, 4, 7)), (16, (1, 1)), (24, (3, 3)), (128, (10, 20, 20))])
def test_layouts(dtype, interleaved, d, pairs):
    from paper_2405_18428_b200 import dig
    freqs, axes = dig.dig_rope_freqs(pairs)
    gen = torch.Generator(device="cuda").manual_seed(d)
    B, L, H, Hk = 3, 37, 4, 2
    q, k = (torch.randn(B, L, h, d, generator=gen, device="cuda").to(dtype) for h in (H, Hk))
    pos = torch.randint(-50, 2000, (B, L, len(pairs)), generator=gen, device="cuda", dtype=torch.int32)
    for p in (pos, pos[0].contiguous()):
        for inverse in (False, True):
            a, b = dig.dig_rope(q, k, p, freqs, axes, interleaved=interleaved, inverse=inverse)
            assert a.dtype == dtype and a.shape == q.shape and b.shape == k.shape
            close(a, turned(q, p, freqs, axes, interleaved, inverse), q, dtype)
            close(b, turned(k, p, freqs, axes, interleaved, inverse), k, dtype)
    only, none = dig.dig_rope(q, None, pos, freqs, axes, interleaved=interleaved)
    assert none is None and torch.equal(only, dig.dig_rope(q, k, pos, freqs, axes, interleaved=interleaved)[0])


def test_far_positions_keep_their_angles():
    from paper_2405_18428_b200 import dig
    freqs, axes = dig.dig_rope_freqs((16, 16))
    q = torch.randn(1, 64, 2, 64, device="cuda")
    pos = torch.randint(2 ** 30, 2 ** 31 - 1, (64, 2), device="cuda", dtype=torch.int32)
    pos[0] = -2 ** 31
    a, _ = dig.dig_rope(q, None, pos, freqs, axes)
    close(a, turned(q, pos, freqs, axes, False, False), q, torch.float32)


@pytest.mark.parametrize("B,L,H,Hk", [(1, 1, 1, 1), (1, 5000, 3, 1), (9, 1, 16, 16), (2, 16384, 2, 2)])
def test_sizes_strides_and_in_place(B, L, H, Hk):
    from paper_2405_18428_b200 import dig
    freqs, axes = dig.dig_rope_freqs((16, 16))
    both = torch.randn(B, L, (H + 2 * Hk) * 64, device="cuda").to(torch.bfloat16)
    q, k, _ = both.split([H * 64, Hk * 64, Hk * 64], 2)
    q, k = q.unflatten(2, (H, 64)), k.unflatten(2, (Hk, 64))
    t = torch.arange(L, device="cuda", dtype=torch.int32)
    pos = torch.stack([t // 64, t % 64], 1).contiguous()
    a, b = dig.dig_rope(q, k, pos, freqs, axes)
    assert a.is_contiguous()
    close(a, turned(q, pos, freqs, axes, False, False), q, torch.bfloat16)
    was = both.clone()
    a2, b2 = dig.dig_rope(q, k, pos, freqs, axes, inplace=True)
    assert a2.data_ptr() == q.data_ptr() and torch.equal(a2, a) and torch.equal(b2, b)
    assert torch.equal(both[..., (H + Hk) * 64:], was[..., (H + Hk) * 64:])


def test_the_inverse_is_the_gradient():
    from paper_2405_18428_b200 import dig
    freqs, axes = dig.dig_rope_freqs((9, 9))
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, g = (torch.randn(2, 50, 3, 40, generator=gen, device="cuda") for _ in range(2))
    pos = torch.randint(0, 999, (50, 2), generator=gen, device="cuda", dtype=torch.int32)
    y, _ = dig.dig_rope(x, None, pos, freqs, axes, interleaved=True)
    dx, _ = dig.dig_rope(g, None, pos, freqs, axes, interleaved=True, inverse=True)
    a, b = (float((s.double() * t.double()).sum()) for s, t in ((y, g), (x, dx)))
    assert abs(a - b) <= 12000 * 1e-6
