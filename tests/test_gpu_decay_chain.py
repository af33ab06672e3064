"""Layer norm, rotary positions, linear attention with a decay for each head and the output gate in a row, as a mixer block has them, forward
and backward, against the same block in 64 bits; then tokens one by one from the state that a prompt left."""
import numpy as np
import pytest
import torch

import decay_ref as ref

pytestmark = pytest.mark.gpu


def reference(x, scale, shift, wq, wk, wv, wr, ln_w, ln_b, lam, pos, freqs, axes, order, H, Hk, d, dz):
    leaves = [t.double().detach().requires_grad_() for t in (x, scale, shift, wq, wk, wv, wr, ln_w, ln_b)]
    x, scale, shift, wq, wk, wv, wr, ln_w, ln_b = leaves
    B, L, D = x.shape
    norm = lambda t, eps=1e-5: (t - t.mean(-1, keepdim=True)) / (t.var(-1, unbiased=False, keepdim=True) + eps).sqrt()
    y = norm(x) * scale[:, None] + shift[:, None]
    heads = lambda w, n: (y @ w).view(B, L, n, d)
    angle = pos.double()[:, axes] * torch.tensor(freqs, dtype=torch.float64, device=pos.device)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turn(t):
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    q, k, v, r = turn(heads(wq, H)), turn(heads(wk, Hk)), heads(wv, Hk), heads(wr, H)
    each = torch.arange(H, device=x.device) // (H // Hk)
    q, k, v = q[:, order], k[:, order][:, :, each], v[:, order][:, :, each]
    gap = torch.arange(L, device=x.device, dtype=torch.float64)
    gap = gap[:, None] - gap[None]
    w = torch.where(gap >= 0, (torch.tensor(lam, dtype=torch.float64, device=x.device)[:, None, None] * gap.clamp(min=0)).exp(), 0.0)
    o = torch.einsum("blhc,bmhc,hlm,bmhe->blhe", q, k, w, v)
    o = o[:, torch.argsort(order)]
    z = torch.nn.functional.silu(r) * (norm(o) * ln_w + ln_b)
    z.backward(dz.double())
    return z.detach(), [t.grad for t in leaves]


@pytest.mark.parametrize("dtype,direction,Hk", [(torch.float32, 0, 4), (torch.float32, 3, 2), (torch.bfloat16, 2, 4), (torch.bfloat16, 1, 1)])
def test_a_block_and_its_gradients(dtype, direction, Hk):
    from paper_2405_18428_b200 import dig
    B, gh, gw, H, d = 2, 12, 17, 4, 64
    L, D = gh * gw, H * d
    gen = torch.Generator(device="cuda").manual_seed(7)
    mk = lambda *s, scale=1.0: torch.randn(s, generator=gen, device="cuda") * scale
    store = lambda t: t.to(dtype)
    x, dz = store(mk(B, L, D)), store(mk(B, L, H, d))
    scale, shift = 1 + mk(B, D, scale=0.2), mk(B, D, scale=0.2)
    wq, wk, wv, wr = mk(D, H * d, scale=D ** -0.5), mk(D, Hk * d, scale=D ** -0.5 * d ** -0.5), mk(D, Hk * d, scale=D ** -0.5), mk(D, H * d, scale=D ** -0.5)
    ln_w, ln_b = 1 + mk(d, scale=0.1), mk(d, scale=0.1)
    lam = [-0.3, -0.02, -0.1, -0.005]
    t = torch.arange(L, device="cuda")
    pos = torch.stack([t // gw, t % gw], 1).int()
    freqs, axes = dig.dig_rope_freqs((16, 16))
    grid = t.view(gh, gw).t().reshape(-1) if direction & 2 else t
    order = grid.flip(0) if direction & 1 else grid

    # forward
    y = dig.dig_layernorm_fwd(x.view(B * L, D), scale, shift).view(B, L, D).float()
    heads = lambda w, n: store(y @ w).view(B, L, n, d)
    q0, k0, v, r = heads(wq, H), heads(wk, Hk), heads(wv, Hk), heads(wr, H)
    q, k = dig.dig_rope(q0, k0, pos, freqs, axes)
    o, _ = dig.dig_decay_fwd(q, k, v, lam, gh, gw, direction)
    z = dig.dig_gla_outgate_fwd(o, r, ln_w, ln_b, 1e-5)
    # backward
    d_o, d_r, dln_w, dln_b = dig.dig_gla_outgate_bwd(o, r, dz, ln_w, ln_b, 1e-5)
    dq, dk, dv, _ = dig.dig_decay_bwd(q, k, v, lam, d_o, gh, gw, direction)
    dq, dk = dig.dig_rope(dq, dk, pos, freqs, axes, inverse=True)
    flat = [g.reshape(B * L, -1).float() for g in (dq, dk, dv, d_r)]
    ws = (wq, wk, wv, wr)
    dws = [y.view(B * L, D).t() @ g for g in flat]
    dy = store(sum(g @ w.t() for g, w in zip(flat, ws)))
    dx, dscale, dshift = dig.dig_layernorm_bwd(x.view(B * L, D), dy, scale)
    got = [dx.view(B, L, D), dscale, dshift, *dws, dln_w, dln_b]
    zr, want = reference(x, scale, shift, *ws, ln_w, ln_b, lam, pos, freqs, axes, order, H, Hk, d, dz)
    # Eight operators and six products in a row, each off by up to 1e-5 in fp32 (hundreds of roundings of 2^-24) or 2.5e-3 in bf16 (a rounding
    # of its own, 2^-8 at most and 1.7e-3 on average, and those of its operands), the norms in between with a factor of up to 3.
    tol = 14 * 3 * (1e-5 if dtype == torch.float32 else 2.5e-3)
    for i, (a, b) in enumerate(zip([z] + got, [zr] + want)):
        err = float((a.double() - b).norm() / b.norm())
        assert err <= tol, (i, err)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_one_by_one_from_the_state_of_a_prompt(dtype):
    from paper_2405_18428_b200 import dig
    B, H, Hk, d, n, more = 3, 4, 2, 72, 200, 4
    x = ref.make(B, n + more, H, Hk, d, d, dtype, 21)
    lam = [-0.4, -0.01, 0.0, -0.1]
    q, k, v = (ref.dev(x[s], dtype) for s in ("q", "k", "v"))
    freqs, axes = dig.dig_rope_freqs((d // 2,))
    pos = torch.arange(n + more, device="cuda", dtype=torch.int32)[:, None].contiguous()
    tq, tk = dig.dig_rope(q, k, pos, freqs, axes)
    whole, _ = dig.dig_decay_fwd(tq, tk, v, lam, 1, n + more)
    _, state = dig.dig_decay_fwd(tq[:, :n], tk[:, :n], v[:, :n], lam, 1, n, want_s_out=True)
    turned = dict(x, q=tq.float().cpu().numpy(), k=tk.float().cpu().numpy())
    o, _ = ref.fwd(turned, lam, 1, n + more, 0)
    size, _ = ref.fwd(ref.magnitude(turned), lam, 1, n + more, 0)
    for t in range(n, n + more):
        # the token's own rotation is that of the whole sequence's
        sq, sk = dig.dig_rope(q[:, t:t + 1], k[:, t:t + 1], pos[t:t + 1], freqs, axes)
        assert torch.equal(sq[:, 0], tq[:, t]) and torch.equal(sk[:, 0], tk[:, t])
        out = dig.dig_decay_step(sq[:, 0].contiguous(), sk[:, 0].contiguous(), v[:, t].contiguous(), lam, state)
        ref.close("step", out, o[:, t], size[:, t], dtype, n + d)
        ref.close("whole", whole[:, t], o[:, t], size[:, t], dtype, n + d)
