"""Layer norm and its backward pass on the GPU against 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(x, w, b, dy, eps):
    """y, dx, dw, db in fp64, through autograd of the definition; w, b: [groups, D]."""
    x = x.double().detach().requires_grad_()
    w, b = w.double().detach().requires_grad_(), b.double().detach().requires_grad_()
    xg = x.view(w.shape[0], -1, x.shape[-1])
    m = xg.mean(-1, keepdim=True)
    y = (xg - m) / ((xg - m).square().mean(-1, keepdim=True) + eps).sqrt() * w[:, None] + b[:, None]
    y.backward(dy.double().view_as(y))
    return y.detach().view_as(x), x.grad, w.grad, b.grad


def check(rows, D, groups, dtype, *, affine=True, seed=0, eps=1e-5, offset=1.0):
    from paper_2405_18428_b200 import dig
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")
    x = (mk(rows, D) * 2 + offset).to(dtype)
    dy = mk(rows, D).to(dtype)
    shape = (D,) if groups == 1 else (groups, D)
    w, b = (1 + 0.3 * mk(*shape), 0.3 * mk(*shape)) if affine else (None, None)
    one = torch.ones(groups, D, device="cuda")
    y, dx, dw, db = reference(x, one if w is None else w.view(groups, D), 0 * one if b is None else b.view(groups, D), dy, eps)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    # sums of D terms by a tree of D / 32 adds at most per thread; the mean's error counts against the spread of the row
    off = (D / 32 + 32) * 2.0 ** -24 * (1 + abs(offset))
    got = dig.dig_layernorm_fwd(x, w, b, eps)
    assert got.dtype == dtype and got.shape == x.shape
    wmax = 1.0 if w is None else float(w.abs().max())
    size = y.abs() + wmax
    assert ((got.double() - y).abs() <= half * y.abs() + off * size * 8).all()
    gx, gw, gb = dig.dig_layernorm_bwd(x, dy, w, eps)
    # 1 / sqrt(var) is the scale of dx; xh reaches 6 or the like
    scale = (1 / (x.double().var(-1, unbiased=False, keepdim=True) + eps).sqrt()) * wmax * dy.double().abs().amax(-1, keepdim=True) * 8
    assert ((gx.double() - dx).abs() <= half * dx.abs() + off * scale * 8).all()
    # at most 1 / 148 of the rows one after the other, or all of them
    n = (rows // groups + 64) * 2.0 ** -24
    xh = (x.double() - x.double().mean(-1, keepdim=True)).abs() / (x.double().var(-1, unbiased=False, keepdim=True) + eps).sqrt()
    of = lambda t: t.view(groups, -1, D).sum(1)
    assert gw.shape == gb.shape == shape and gw.dtype == torch.float32
    assert ((gw.double().view(groups, D) - dw).abs() <= (n + off * 8) * of(dy.double().abs() * (xh + 1))).all()
    assert ((gb.double().view(groups, D) - db).abs() <= n * of(dy.double().abs())).all()
    gx2, none, none2 = dig.dig_layernorm_bwd(x, dy, w, eps, affine_grads=False)
    assert none is None and none2 is None and torch.equal(gx2, gx)
    again = dig.dig_layernorm_bwd(x, dy, w, eps)
    assert torch.equal(again[1], gw) and torch.equal(again[2], gb)          # a fixed order


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [1, 2, 7, 8, 33, 64, 255, 256, 384, 520, 766, 768, 1001, 1002, 1024, 1152, 2048, 2056, 4094, 4095, 4096, 5000, 6002, 8191, 8192])
def test_row_lengths(dtype, D):
    check(37, D, 1, dtype, seed=D)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,groups", [(1, 1), (3000, 1), (700, 7), (64, 64), (12800, 128), (6000, 3)])
@pytest.mark.parametrize("D", [384, 99])
def test_rows_and_groups(dtype, rows, groups, D):
    check(rows, D, groups, dtype, seed=rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_without_affine_parameters(dtype):
    check(100, 640, 1, dtype, affine=False)


def test_constant_rows_give_the_bias_and_no_infinity():
    from paper_2405_18428_b200 import dig
    x = torch.full((4, 384), 3.0, device="cuda")
    b = torch.randn(384, device="cuda")
    assert torch.equal(dig.dig_layernorm_fwd(x, None, b), b.expand(4, -1))
    dx, dw, db = dig.dig_layernorm_bwd(x, torch.ones_like(x))
    assert torch.isfinite(dx).all() and (dw == 0).all() and (db == 4).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_constant_rows_and_a_small_eps(dtype):
    from paper_2405_18428_b200 import dig
    x, dy = torch.full((4, 384), 3.0, device="cuda", dtype=dtype), torch.zeros(4, 384, device="cuda", dtype=dtype)
    dy[:, 0], dy[:, 1] = 1, -1                               # mean(g) = 0: dx = r dy, and r = 2^50
    dx, dw, db = dig.dig_layernorm_bwd(x, dy, None, 2.0 ** -100)
    # 1 / sqrt(eps) to two units in the last place of fp32, and a rounding to the type
    assert ((dx.double() - dy.double() * 2.0 ** 50).abs() <= 2.0 ** 50 * (torch.finfo(dtype).eps / 2 + 2.0 ** -22) * dy.double().abs()).all()
    assert (dw == 0).all() and torch.equal(db, 4 * dy[0].float())


def test_a_nan_stays_in_its_row():
    from paper_2405_18428_b200 import dig
    x = torch.randn(300, 1152, device="cuda").to(torch.bfloat16)
    y = dig.dig_layernorm_fwd(x)
    z = x.clone()
    z[77, 5] = float("nan")
    out = dig.dig_layernorm_fwd(z)
    assert torch.isnan(out[77]).all()
    out[77] = y[77]
    assert torch.equal(out, y)


def test_graph_and_stream():
    from paper_2405_18428_b200 import dig
    x, dy = (torch.randn(4096, 768, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randn(768, device="cuda")
    run = lambda: (dig.dig_layernorm_fwd(x, w), *dig.dig_layernorm_bwd(x, dy, w))
    want = run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for t in got:
        t.fill_(float("nan"))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        g.replay()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
