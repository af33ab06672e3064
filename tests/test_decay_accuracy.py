"""Accuracy of linear attention with a decay for each head as a whole: the error's norm against the result's, head by head.  Elementwise bounds have to
allow for the worst element; these show a result that is a little off throughout, and states with fewer bits than their 24."""
import numpy as np
import pytest
import torch

import decay_ref as ref

# bf16 storage: decayed scores and keys are rounded to bf16, and so is the result.  A rounding is off by up to 2^-8 of its value, in the mean of
# squares by 2^-8 / sqrt(3) at most; what is summed has random signs, so that the two stand beside one another: sqrt(2) times as much.
BF16 = 2.0 ** -8 * (2 / 3) ** 0.5
# fp32: a power of the decay is 2^x, x = c n rounded twice, off by 2 |x| ln 2 2^-24 (tokens that count have |x| < 8: 6.6e-7), and the approximate
# exponential by 2^-22; products and sums of up to 128 terms in a tile and 30 tiles 2^-25 sqrt(128 + 30) each way, 3.8e-7.
F32 = 2 * 8 * np.log(2) * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -25 * 158 ** 0.5
DECAYS = [-0.02, 0.0, -0.3, -1e-4]


def head_errors(got, want, heads):
    """Relative L2 error of each head."""
    got, want = (np.moveaxis(np.asarray(a, dtype=np.float64), heads, 0).reshape(a.shape[heads], -1) for a in (got, want))
    return np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)


def state_of_parts(k, v, lam, parts):
    """The final state from decayed keys in so many bf16 parts, all else exact."""
    n = len(k)
    w = np.exp2((lam * np.log2(np.e) * np.arange(n - 1, -1, -1)).astype(np.float32)).astype(np.float32)
    rest, keys = torch.from_numpy(k * w[:, None]), torch.zeros(k.shape, dtype=torch.float64)
    for _ in range(parts):
        part = rest.to(torch.bfloat16).float()
        keys += part.double()
        rest = rest - part
    return keys.numpy().T @ v.astype(np.float64)


@pytest.mark.parametrize("lam", [0.0, -1e-4, -0.02])
def test_the_bound_tells_two_parts_from_three(lam):
    x = ref.make(1, 3000, 1, 1, 72, 72, "bf16", 3)
    k, v = x["k"][0, :, 0], x["v"][0, :, 0]
    want = (k.astype(np.float64) * np.exp(lam * np.arange(2999, -1, -1))[:, None]).T @ v.astype(np.float64)
    err = [float(np.linalg.norm(state_of_parts(k, v, lam, p) - want) / np.linalg.norm(want)) for p in (1, 2, 3)]
    # with a decay of one the keys are bf16 as they come
    assert err[2] <= F32 and (lam == 0.0 or (err[0] > F32 and err[1] > F32)), err


def test_the_bound_tells_a_scaled_result():
    rng = np.random.default_rng(5)
    exact = rng.standard_normal((1, 4000, 2, 64))
    twice = torch.from_numpy(exact * (1 + 2.0 ** -8 / 3 ** 0.5 * rng.uniform(-1, 1, exact.shape))).to(torch.bfloat16).double().numpy()
    assert (head_errors(twice, exact, 2) <= BF16).all()
    assert (head_errors(exact * 1.004, exact, 2) > BF16).all()


CASES = [(1, 4, 4, 50, 61, 72, 72, 0, None), (2, 4, 2, 40, 45, 64, 64, 3, None), (2, 4, 4, 24, 30, 128, 128, 1, None), (40, 4, 4, 16, 16, 64, 64, 2, None),
         (6, 4, 1, 1, 700, 128, 64, 0, [700, 1, 350, 129, 699, 512]), (3, 4, 4, 1, 900, 80, 96, 1, [900, 128, 301]), (1, 4, 4, 37, 29, 64, 40, 1, None)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hk,gh,gw,dk,dv,direction,lengths", CASES)
def test_errors_of_heads(dtype, B, H, Hk, gh, gw, dk, dv, direction, lengths):
    from paper_2405_18428_b200 import dig
    x = ref.make(B, gh * gw, H, Hk, dk, dv, dtype, 17, True)
    if lengths is not None:
        for b, n in enumerate(lengths):
            for t in ("q", "k", "v", "d_out"):
                x[t][b, n:] = 0
    q, k, v, d_out = (ref.dev(x[n], dtype) for n in ("q", "k", "v", "d_out"))
    s_in, ds_out = (ref.dev(x[n], "f32") for n in ("s_in", "ds_out"))
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, s_out = dig.dig_decay_fwd(q, k, v, DECAYS, gh, gw, direction, s_in=s_in, lengths=n, want_s_out=True)
    dq, dk_, dv_, ds_in = dig.dig_decay_bwd(q, k, v, DECAYS, d_out, gh, gw, direction, s_in=s_in, ds_out=ds_out, lengths=n, want_ds_in=True)
    want = [*ref.fwd(x, DECAYS, gh, gw, direction, lengths), *ref.bwd(x, DECAYS, gh, gw, direction, lengths)]
    bound = F32 if dtype == "f32" else BF16
    for name, got, w, heads, lim in (("out", out, want[0], 2, bound), ("s_out", s_out, want[1], 1, F32), ("dq", dq, want[2], 2, bound), ("dk", dk_, want[3], 2, bound),
                                     ("dv", dv_, want[4], 2, bound), ("ds_in", ds_in, want[5], 1, F32)):
        err = head_errors(got.float().cpu().numpy(), w, heads)
        assert (err <= lim).all(), (name, err, lim)
