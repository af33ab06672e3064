"""Rotary positions in place: tensors whose rows coincide are refused, all others give what dense results hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def turn(q, k, positions, inplace):
    from paper_2405_18428_b200 import dig
    return dig.dig_rope(q, k, positions, *dig.dig_rope_freqs((32,)), inplace=inplace)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_batch_broadcast_from_one_sequence_is_refused(dtype):
    def refused(q, k=None):
        was = [None if t is None else t.clone() for t in (q, k)]
        pos = torch.arange(q.shape[1], dtype=torch.int32, device="cuda")[:, None].contiguous()
        with pytest.raises(ValueError, match="overlap"):
            turn(q, k, pos, True)
        assert all(a is None or torch.equal(a, b) for a, b in zip((q, k), was))

    x = torch.randn(1, 6, 4, 64, device="cuda").to(dtype)
    ok = torch.randn(3, 6, 4, 64, device="cuda").to(dtype)
    one = torch.randn(3, 1, 4, 64, device="cuda").to(dtype)
    refused(x.expand(3, 6, 4, 64))
    refused(x[:, :1].expand(3, 1, 4, 64))
    refused(x[:, :1].expand(1, 6, 4, 64))
    refused(ok, x.expand(3, 6, 4, 64))
    refused(one, x[:, :1].expand(3, 1, 4, 64))
    # sequences, then tokens, that overlap by half a row
    flat = torch.randn(5000, device="cuda").to(dtype)
    refused(flat.as_strided((3, 6, 4, 64), (128, 512, 64, 1)))
    refused(flat.as_strided((3, 1, 4, 64), (128, 256, 64, 1)))
    refused(flat.as_strided((1, 6, 4, 64), (0, 128, 64, 1)))


def test_keys_that_are_queries_are_refused():
    from paper_2405_18428_b200 import dig
    x = torch.randn(2, 6, 6, 64, device="cuda")
    pos = torch.arange(5, dtype=torch.int32, device="cuda")[:, None].contiguous()
    for q, k in ((x[:, :5, :4], x[:, :5, 2:]), (x[:, :5], x[:, 1:]), (x[:, :5, :4], x[:, 1:, 3:])):
        with pytest.raises(dig.DigError):
            turn(q, k, pos, True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_any_distinct_layout(dtype):
    B, L, H, Hk, d = 3, 7, 4, 2, 64
    pos = torch.arange(L, dtype=torch.int32, device="cuda")[:, None].contiguous()
    new = lambda *s: torch.randn(*s, device="cuda").to(dtype)
    fused, by_token, block, rows = new(B, L, (H + 2 * Hk) * d), new(L, B, (H + Hk) * d), new(B, L * (H + Hk) * d), new(B, 2 * L, H, d)
    flat = new(4000)
    layouts = [
        (fused[..., :H * d].unflatten(2, (H, d)), fused[..., H * d:(H + Hk) * d].unflatten(2, (Hk, d))),
        (fused[..., Hk * d:(H + Hk) * d].unflatten(2, (H, d)), fused[..., :Hk * d].unflatten(2, (Hk, d))),
        (by_token[..., :H * d].unflatten(2, (H, d)).transpose(0, 1), by_token[..., H * d:].unflatten(2, (Hk, d)).transpose(0, 1)),
        (block[:, :L * H * d].view(B, L, H, d), block[:, L * H * d:].view(B, L, Hk, d)),
        (rows[:, :L], rows[:, L:]),
        (rows[:, 0::2], rows[:, 1::2]),
        (rows[:, :L], None),
        # sequences two rows apart, tokens three: no order of whole sequences or tokens, yet no two meet
        (flat.as_strided((3, 2, 1, 64), (128, 192, 64, 1)), None),
    ]
    for q, k in layouts:
        p = pos[:q.shape[1]]
        want = turn(q, k, p, False)
        got = turn(q, k, p, True)
        assert got[0].data_ptr() == q.data_ptr() and torch.equal(got[0], want[0])
        assert k is None or (got[1].data_ptr() == k.data_ptr() and torch.equal(got[1], want[1]))
