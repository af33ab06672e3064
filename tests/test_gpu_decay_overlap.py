"""Results that a caller gives: refused where they overlap an input or one another, taken where they only stand between its rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_results_that_overlap_are_refused(dtype):
    from paper_2405_18428_b200 import dig
    B, L, H, d = 2, 12, 4, 64
    new = lambda *s: torch.randn(*s, device="cuda").to(dtype)
    q, k, v, g = (new(B, L, H, d) for _ in range(4))
    lam = [-0.1] * H
    state = torch.randn(B, H, d, d, device="cuda")
    both = new(B, L, 3 * H * d)
    fused = [t.unflatten(2, (H, d)) for t in both.split(H * d, 2)]
    part = both.flatten()[H * d:H * d + B * L * H * d].view(B, L, H, d)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    given = lambda at, n: ws[at:at + 2 * n if dtype == torch.bfloat16 else at + 4 * n].view(dtype)
    n = B * L * H * d
    cases = [lambda: dig.dig_decay_fwd(q, k, v, lam, 3, 4, out=q), lambda: dig.dig_decay_fwd(q, k, v, lam, 3, 4, out=v), lambda: dig.dig_decay_fwd(*fused, lam, 3, 4, out=part),
             lambda: dig.dig_decay_fwd(q, k, v, lam, 3, 4, s_in=state, workspace=state), lambda: dig.dig_decay_fwd(q, k, v, lam, 3, 4, out=given(256, n).view(B, L, H, d), workspace=ws),
             lambda: dig.dig_decay_bwd(q, k, v, lam, g, 3, 4, grads=(q, torch.empty_like(k), torch.empty_like(v))),
             lambda: dig.dig_decay_bwd(q, k, v, lam, g, 3, 4, grads=(torch.empty_like(q), torch.empty_like(k), g))]
    a, b = torch.empty_like(q), torch.empty_like(q)
    cases += [lambda: dig.dig_decay_bwd(q, k, v, lam, g, 3, 4, grads=(a, b, a)), lambda: dig.dig_decay_bwd(q, k, v, lam, g, 3, 4, grads=(a, a, b))]
    t = [x[:, 0].contiguous() for x in (q, k, v)]
    cases += [lambda i=i: dig.dig_decay_step(*t, lam, state, out=t[i]) for i in range(3)]
    if dtype == torch.float32:
        cases += [lambda: dig.dig_decay_step(*t, lam, state, out=state.flatten()[64:64 + B * H * d].view(B, H, d)),
                  lambda: dig.dig_decay_step(state.flatten()[64:64 + B * H * d].view(B, H, d), *t[1:], lam, state)]
    was = [x.clone() for x in (q, k, v, g, state, both)]
    for i, call in enumerate(cases):
        with pytest.raises(ValueError, match="overlaps"):
            call()
            pytest.fail(f"case {i} was taken")
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((q, k, v, g, state, both), was))


def test_results_between_the_rows_of_an_input_are_taken():
    from paper_2405_18428_b200 import dig
    # two sequences far apart in one buffer, results between them
    L, H, d = 5, 2, 64
    row = H * d
    buf = torch.randn(40 * L * row, device="cuda").to(torch.bfloat16)
    q, k, v = (buf.as_strided((2, L, H, d), (20 * L * row, row, d, 1), i * L * row) for i in range(3))
    out = buf[4 * L * row:6 * L * row].view(2, L, H, d)
    want = dig.dig_decay_fwd(q, k, v, [-0.1, -0.2], 1, L)[0]
    got = dig.dig_decay_fwd(q, k, v, [-0.1, -0.2], 1, L, out=out)[0]
    assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
    grads = [buf[i * L * row:(i + 2) * L * row].view(2, L, H, d) for i in (6, 8, 10)]
    g = torch.randn(2, L, H, d, device="cuda").to(torch.bfloat16)
    want = dig.dig_decay_bwd(q, k, v, [-0.1, -0.2], g, 1, L)[:3]
    got = dig.dig_decay_bwd(q, k, v, [-0.1, -0.2], g, 1, L, grads=grads)[:3]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a token's result beside its queries
    both = torch.randn(4, 3, 64, device="cuda").to(torch.bfloat16)
    q, out = both[:2], both[2:]
    k = torch.randn(2, 3, 64, device="cuda").to(torch.bfloat16)
    s = torch.randn(2, 3, 64, 64, device="cuda")
    want = dig.dig_decay_step(q, k, k, [-0.1] * 3, s.clone())
    assert torch.equal(dig.dig_decay_step(q, k, k, [-0.1] * 3, s, out=out), want)
