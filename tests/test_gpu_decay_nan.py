"""A NaN or an infinity stays in the state of linear attention with a decay for each head, as in the recurrence (0 times a NaN is a NaN): the same
channels are finite whether a sequence is cut or not, in fp32 and bf16 storage, and token by token."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("log_decay", [-0.002, -0.5, -5.0, -1e5])
@pytest.mark.parametrize("B,d", [(1, 64), (80, 64), (1, 72), (1, 128), (80, 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_it_stays_however_far_the_decay_has_gone(dtype, log_decay, B, d, bad):
    from paper_2405_18428_b200 import dig
    L, at, c = 1400, 70, 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(B, L, 2, d, generator=gen, device="cuda").to(dtype) for _ in range(3))
    lam = [log_decay] * 2
    for name, t in (("k", k), ("v", v)):
        was = t[0, at, 1, c].item()
        t[0, at, 1, c] = bad
        out, s = dig.dig_decay_fwd(q, k, v, lam, 1, L, want_s_out=True)
        t[0, at, 1, c] = was
        lost = torch.zeros(d, d, dtype=torch.bool, device="cuda")
        lost[(c, slice(None)) if name == "k" else (slice(None), c)] = True
        assert not torch.isfinite(s[0, 1][lost]).any() and torch.isfinite(s[0, 1][~lost]).all()
        rows = out[0, at:, 1]
        assert not torch.isfinite(rows if name == "k" else rows[:, c]).any()
        if name == "v":
            assert torch.isfinite(rows[:, :c]).all() and torch.isfinite(rows[:, c + 1:]).all()
        assert torch.isfinite(out[0, :at // 32 * 32]).all() and torch.isfinite(out[0, :, 0]).all() and torch.isfinite(s[0, 0]).all()
        if B > 1:
            assert torch.isfinite(out[1:]).all() and torch.isfinite(s[1:]).all()
        # one more token
        dig.dig_decay_step(*(x[:, 0].contiguous() for x in (q, k, v)), lam, s)
        assert not torch.isfinite(s[0, 1][lost]).any() and torch.isfinite(s[0, 1][~lost]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("log_decay", [-0.5, -1e5])
def test_gradients_keep_it_too(dtype, log_decay):
    from paper_2405_18428_b200 import dig
    L, d, at, c = 1400, 64, 1300, 5
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, g = (torch.randn(1, L, 2, d, generator=gen, device="cuda").to(dtype) for _ in range(4))
    g[0, at, 1, c] = float("nan")
    dq, dk, dv, ds = dig.dig_decay_bwd(q, k, v, [log_decay] * 2, g, 1, L, want_ds_in=True)
    # dv = (K Q^T . W^T) dO: channel c of all tokens up to `at`; dk = (V dO^T . W^T) Q and ds_in likewise
    assert not torch.isfinite(dv[0, :at + 1, 1, c]).any() and not torch.isfinite(dk[0, :at + 1, 1]).any() and not torch.isfinite(ds[0, 1][:, c]).any()
    assert torch.isfinite(dv[0, (at + 32) // 32 * 32:]).all() and torch.isfinite(dk[0, at + 32:]).all() and torch.isfinite(ds[0, 0]).all()
    assert not torch.isfinite(dq[0, at, 1]).any() and torch.isfinite(dq[0, :at]).all() and torch.isfinite(dq[0, at + 1:]).all()
