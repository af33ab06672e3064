"""What the Python functions of linear attention with a decay for each head, rotary positions and layer norm refuse, on CUDA tensors."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def test_decay_refuses():
    from paper_2405_18428_b200 import dig
    q, k, v, lam = z(2, 12, 4, 64), z(2, 12, 2, 64), z(2, 12, 2, 72), [-0.1] * 4
    fwd = lambda q=q, k=k, v=v, lam=lam, gh=3, gw=4, dir=0, **kw: dig.dig_decay_fwd(q, k, v, lam, gh, gw, dir, **kw)
    assert fwd()[0].shape == (2, 12, 4, 72)
    for bad in (dict(q=z(2, 12, 4, 64, dtype=torch.float32)), dict(k=z(2, 12, 3, 64)), dict(k=z(2, 11, 2, 64)), dict(v=z(2, 12, 4, 72)), dict(q=q[0]), dict(gw=5), dict(lam=[-0.1] * 3),
                dict(q=z(2, 12, 64, 4).transpose(2, 3)), dict(q=z(2, 12, 4, 66)[..., :64]), dict(q=z(2, 12, 4 * 64 + 4)[..., 4:].unflatten(2, (4, 64))),
                dict(s_in=z(2, 4, 64, 64, dtype=torch.float32)), dict(s_in=z(2, 4, 64, 72)), dict(lengths=torch.zeros(2, device="cuda")), dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(lengths=torch.zeros(2, dtype=torch.int32)), dict(out=z(2, 12, 4, 64)), dict(q=z(0, 12, 4, 64), k=z(0, 12, 2, 64), v=z(0, 12, 2, 72)), dict(workspace=torch.zeros(1 << 20))):
        with pytest.raises(ValueError):
            fwd(**bad)
    with pytest.raises(TypeError):
        fwd(q=q.half())
    for bad, status in ((dict(lam=[0.1] * 4), dig.DIG_ERR_INVALID_ARG), (dict(lam=[float("nan")] * 4), dig.DIG_ERR_INVALID_ARG), (dict(dir=4), dig.DIG_ERR_INVALID_ARG),
                        (dict(dir=2, lengths=torch.ones(2, dtype=torch.int32, device="cuda")), dig.DIG_ERR_UNSUPPORTED), (dict(workspace=z(8)), dig.DIG_ERR_WORKSPACE),
                        (dict(q=z(2, 12, 4, 136), k=z(2, 12, 2, 136)), dig.DIG_ERR_INVALID_ARG)):
        with pytest.raises(dig.DigError) as e:
            fwd(**bad)
        assert e.value.status == status, bad
    g = z(2, 12, 4, 72)
    assert dig.dig_decay_bwd(q, k, v, lam, g, 3, 4)[1].shape == k.shape
    for bad in (dict(grads=(z(2, 12, 4, 64),)), dict(grads=(z(2, 12, 4, 64), z(2, 12, 4, 64), z(2, 12, 2, 72))), dict(ds_out=z(2, 4, 64, 72))):
        with pytest.raises(ValueError):
            dig.dig_decay_bwd(q, k, v, lam, g, 3, 4, **bad)
    with pytest.raises(ValueError):
        dig.dig_decay_bwd(q, k, v, lam, z(2, 12, 4, 64), 3, 4)
    state = z(2, 4, 64, 72, dtype=torch.float32)
    step = lambda q=z(2, 4, 64), k=z(2, 2, 64), v=z(2, 2, 72), lam=lam, state=state: dig.dig_decay_step(q, k, v, lam, state)
    assert step().shape == (2, 4, 72)
    for bad in (dict(q=z(2, 4, 1, 64)), dict(k=z(2, 3, 64)), dict(v=z(2, 4, 72)), dict(state=z(2, 4, 72, 64, dtype=torch.float32)), dict(state=z(2, 4, 64, 72)), dict(lam=[0.0]),
                dict(state=z(2, 4, 72, 64, dtype=torch.float32).transpose(2, 3))):
        with pytest.raises(ValueError):
            step(**bad)


def test_rope_and_norm_refuse():
    from paper_2405_18428_b200 import dig
    q, pos = z(2, 6, 4, 64), torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    freqs, axes = dig.dig_rope_freqs((16, 16))
    rope = lambda q=q, k=None, pos=pos, freqs=freqs, axes=axes, **kw: dig.dig_rope(q, k, pos, freqs, axes, **kw)
    rope()
    for bad in (dict(k=z(2, 6, 4, 72)), dict(k=z(1, 6, 4, 64)), dict(pos=pos[:5].contiguous()), dict(pos=pos.long()), dict(pos=pos.cpu()), dict(axes=axes[:-1]), dict(pos=pos.expand(3, 6, 2).contiguous()),
                dict(q=z(1, 1, 4, 64).expand(2, 6, 4, 64), inplace=True)):
        with pytest.raises(ValueError):
            rope(**bad)
    for bad in (dict(axes=[2] * 32), dict(axes=[-1] * 32), dict(freqs=freqs + [1.0], axes=axes + [0]), dict(freqs=[float("inf")] * 32)):
        with pytest.raises(dig.DigError):
            rope(**bad)
    x, w = z(6, 64), torch.ones(64, device="cuda")
    dig.dig_layernorm_fwd(x, w, w)
    f32 = torch.float32
    for bad in ((z(0, 64), None, None), (x, w.bfloat16(), None), (x, w[:63], None), (x, z(4, 64, dtype=f32), None), (x, w, z(2, 64, dtype=f32)), (x.t(), None, None), (x, w.cpu(), None)):
        with pytest.raises(ValueError):
            dig.dig_layernorm_fwd(*bad)
    with pytest.raises(ValueError):
        dig.dig_layernorm_bwd(x, x.float(), w)
    with pytest.raises(ValueError):
        dig.dig_layernorm_bwd(x, x[:5], w)
    with pytest.raises(dig.DigError):
        dig.dig_layernorm_fwd(z(2, 9000))
    with pytest.raises(dig.DigError):
        dig.dig_layernorm_fwd(x, w, w, -1.0)
    with pytest.raises(dig.DigError):
        dig.dig_layernorm_bwd(x, x, w, workspace=z(8))


def test_broadcast_inputs_are_read_as_they_are():
    # the same keys and values for all sequences, and a projection with larger strides
    from paper_2405_18428_b200 import dig
    gen = torch.Generator(device="cuda").manual_seed(2)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = mk(3, 150, 2, 64), mk(1, 150, 2, 64), mk(1, 150, 2, 64)
    a, _ = dig.dig_decay_fwd(q, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), [-0.1, -0.2], 10, 15, 2)
    b, _ = dig.dig_decay_fwd(q, k.repeat(3, 1, 1, 1), v.repeat(3, 1, 1, 1), [-0.1, -0.2], 10, 15, 2)
    assert torch.equal(a, b)
    big = mk(3, 400, 5, 64)
    part = big[:, 7:157, 1:3]
    assert not part.is_contiguous()
    a, _ = dig.dig_decay_fwd(part, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), [-0.1, -0.2], 10, 15, 1)
    b, _ = dig.dig_decay_fwd(part.contiguous(), k.repeat(3, 1, 1, 1), v.repeat(3, 1, 1, 1), [-0.1, -0.2], 10, 15, 1)
    assert torch.equal(a, b)
