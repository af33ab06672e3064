"""Performance cases of the operators around linear attention with a decay for each head: the attention itself (whole
sequences, training, single tokens), rotary positions with several axes in front of it, and the layer norm of the block.

Sizes are those of the repository's workloads (grids of 16 x 16 to 128 x 128 tokens, 6, 12 or 16 heads of 64 or 72
channels, hidden sizes 384, 768 and 1152), and heads of 128 channels with shared key/value heads.

`op` of a case:
  prompt     forward pass over whole sequences, with the state that single tokens go on from
  train      forward and backward pass, from a start state where `state` is set
  step       one token for every sequence, the state updated in place
  rope       rotation of queries and keys (`inverse`: the gradient's direction)
  norm       layer norm
  norm_train layer norm and its backward pass with the gradients of the affine parameters
"""
import math

import torch

own = False

_EPS = 1e-5


def _attn(name, op, dtype, B, H, Hk, grid_h, grid_w, dk, dv, direction=0, decay="retention", state=False, lengths=False, fused=False):
    c = dict(op=op, dtype=dtype, B=B, H=H, Hk=Hk, grid_h=grid_h, grid_w=grid_w, dk=dk, dv=dv, direction=direction, decay=decay, state=state,
             lengths=lengths, fused=fused)
    return c if name is None else dict(name=name, **c)


def _rope(name, dtype, B, T, grid_h, grid_w, H, Hk, d, interleaved=False, inverse=False):
    c = dict(op="rope", dtype=dtype, B=B, T=T, grid_h=grid_h, grid_w=grid_w, H=H, Hk=Hk, d=d, interleaved=interleaved, inverse=inverse)
    return c if name is None else dict(name=name, **c)


def _norm(name, op, dtype, groups, rows, D):
    c = dict(op=op, dtype=dtype, groups=groups, rows=rows, D=D)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # the next token of one sequence through an S-size block: the smallest call, all latency
        _attn("step_1_s", "step", "bf16", 1, 6, 6, 1, 1, 64, 64),
        # the next token of 192 sequences of an XL block being served together
        _attn("step_192_xl", "step", "bf16", 192, 16, 16, 1, 1, 72, 72),
        # one 256 x 256 image through an S-size block
        _attn("prompt_256px_s", "prompt", "bf16", 1, 6, 6, 16, 16, 64, 64),
        # a padded batch of prompts of different lengths, wide heads whose keys and values four queries share, q, k and v
        # as one projection wrote them, from a start state
        _attn("prompt_padded_shared", "prompt", "bf16", 5, 16, 4, 1, 2500, 128, 128, decay="slopes", state=True, lengths=True, fused=True),
        # one 2048 x 2048 image through an XL block in a reversed column scan
        _attn("prompt_2048px_xl", "prompt", "bf16", 1, 16, 16, 128, 128, 72, 72, direction=3),
        # training at 1024 x 1024, B size
        _attn("train_1024px_b", "train", "bf16", 4, 12, 12, 64, 64, 64, 64, direction=2),
        # training in fp32 storage on an odd grid, key and value channels of different number, from a start state
        _attn("train_odd_f32", "train", "f32", 2, 6, 6, 37, 29, 64, 40, direction=1, decay="slopes", state=True),
        # queries and keys of one 256 x 256 image, two axes
        _rope("rope_256px_s", "bf16", 1, 1, 16, 16, 6, 6, 64),
        # the gradient's rotation for a clip of 8 frames of 512 x 512 in a batch of two, XL size, three axes
        _rope("rope_video_xl", "bf16", 2, 8, 32, 32, 16, 16, 72, interleaved=True, inverse=True),
        # the norm in front of a block for one 256 x 256 image
        _norm("norm_256px_s", "norm", "bf16", 1, 256, 384),
        # training at 2048 x 2048, XL size
        _norm("norm_train_2048px_xl", "norm_train", "bf16", 1, 16384, 1152),
        # training on 128 images of 256 x 256, each with its own scale and shift, fp32 storage
        _norm("norm_train_modulated", "norm_train", "f32", 128, 128 * 256, 768),
    ]


# Work of the largest listed cases: state elements of a step, elements of q.
_MOST_STEP = 192 * 16 * 72 * 72
_MOST = 128 * 128 * 16 * 72
_MOST_NORM = 128 * 256 * 768


def draw(rng):
    """One more case: an op with its share of use, then sizes spread over their logarithm."""
    spread = lambda lo, hi: max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))
    op = rng.choices(["prompt", "train", "step", "rope", "norm", "norm_train"], [25, 25, 15, 15, 8, 12])[0]
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if op in ("norm", "norm_train"):
        D = rng.choice([384, 768, 1152, spread(100, 4096), 8 * spread(8, 512)])
        groups = 1 if rng.random() < 0.6 else spread(2, 128)
        each = spread(1, min(_MOST_NORM // (D * groups), 32768))
        return _norm(None, op, dtype, groups, groups * each, D)
    H, d = rng.choice([(6, 64), (12, 64), (16, 72), (16, 128), (8, 96), (4, 80)])
    Hk = H if rng.random() < 0.7 else H // 2
    if op == "step":
        return _attn(None, op, dtype, spread(1, min(512, _MOST_STEP // (H * d * d))), H, Hk, 1, 1, d, rng.choice([d, d, 64]), decay=rng.choice(["retention", "slopes"]))
    if op == "rope":
        T, gh, gw = rng.choice([1, 1, 1, spread(2, 16)]), spread(1, 64), spread(1, 64)
        return _rope(None, dtype, spread(1, max(1, min(64, _MOST // (T * gh * gw * H * d)))), T, gh, gw, H, Hk, d, rng.random() < 0.5, rng.random() < 0.5)
    most = _MOST // (8 if dtype == "f32" else 2 if op == "train" else 1)
    while True:
        gh, gw = spread(1, 128), spread(8, 128)
        if gh * gw * H * d <= most:
            break
    direction = rng.randrange(4)
    return _attn(None, op, dtype, spread(1, min(128, most // (gh * gw * H * d))), H, Hk, gh, gw, d, rng.choice([d, d, 64]), direction,
                 rng.choice(["retention", "slopes"]), rng.random() < 0.4, op == "prompt" and direction < 2 and rng.random() < 0.4, rng.random() < 0.3)


def _log_decay(case):
    """One log decay for each head: 1 - 2^-5 ... 1 - 2^-9 (slow decays), or slopes 2^(-8/H) ... 2^-8."""
    H = case["H"]
    if case["decay"] == "retention":
        return [math.log(1 - 2.0 ** (-5 - 4 * h / H)) for h in range(H)]
    return [-(2.0 ** (-8 * (h + 1) / H)) for h in range(H)]


def _freqs(pairs, theta=10000.0):
    """A ladder of frequencies for each axis, as long as its share of the pairs, and the axis of each pair."""
    freqs, axes = [], []
    for a, n in enumerate(pairs):
        freqs += [theta ** (-i / n) for i in range(n)]
        axes += [a] * n
    return freqs, axes


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    op = case["op"]

    def normal(*shape, scale=1.0, dtype=st):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    s = dict(case=case)
    if op in ("norm", "norm_train"):
        rows, D, G = case["rows"], case["D"], case["groups"]
        shape = (D,) if G == 1 else (G, D)
        # token vectors have means and scales of their own
        s["x"] = (torch.randn((rows, D), generator=gen, device="cuda") * (0.5 + torch.rand((rows, 1), generator=gen, device="cuda")) +
                  torch.randn((rows, 1), generator=gen, device="cuda")).to(st)
        s["w"] = 1 + normal(*shape, scale=0.1, dtype=torch.float32)
        s["b"] = normal(*shape, scale=0.1, dtype=torch.float32)
        if op == "norm_train":
            s["dy"] = normal(rows, D)
        return s
    B, H, Hk = case["B"], case["H"], case["Hk"]
    if op == "rope":
        T, gh, gw, d = case["T"], case["grid_h"], case["grid_w"], case["d"]
        L = T * gh * gw
        s["q"], s["k"] = normal(B, L, H, d), normal(B, L, Hk, d)
        t = torch.arange(L, device="cuda")
        cols = [t // gw % gh, t % gw]
        n = d // 2
        share = [n // 2, n - n // 2]
        if T > 1:
            # a clip starts anywhere in its video
            cols = [t // (gh * gw) + int(torch.randint(0, 100000, (1,), generator=gen, device="cuda"))] + cols
            share = [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2]
        s["positions"] = torch.stack(cols, 1).to(torch.int32)
        s["freqs"], s["axes"] = _freqs(share)
        return s
    dk, dv = case["dk"], case["dv"]
    s["log_decay"] = _log_decay(case)
    if op == "step":
        s["q"], s["k"], s["v"] = normal(B, H, dk), normal(B, Hk, dk, scale=dk ** -0.5), normal(B, Hk, dv)
        s["state"] = normal(B, H, dk, dv, dtype=torch.float32)
        return s
    L = case["grid_h"] * case["grid_w"]
    if case["fused"]:
        # one projection wrote q, k and v of a token side by side
        both = normal(B, L, H * dk + Hk * (dk + dv))
        both[..., H * dk:(H + Hk) * dk] *= dk ** -0.5
        q, k, v = both.split([H * dk, Hk * dk, Hk * dv], 2)
        s["q"], s["k"], s["v"] = q.unflatten(2, (H, dk)), k.unflatten(2, (Hk, dk)), v.unflatten(2, (Hk, dv))
    else:
        s["q"], s["k"], s["v"] = normal(B, L, H, dk), normal(B, L, Hk, dk, scale=dk ** -0.5), normal(B, L, Hk, dv)
    s["s_in"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
    s["lengths"] = torch.randint(0, L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if case["lengths"] else None
    if op == "train":
        s["d_out"] = normal(B, L, H, dv)
        s["ds_out"] = normal(B, H, dk, dv, dtype=torch.float32) if case["state"] else None
    return s


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _own(c, s):
    from paper_2405_18428_b200 import dig
    op = c["op"]
    if op == "norm":
        return dig.dig_layernorm_fwd(s["x"], s["w"], s["b"], _EPS)
    if op == "norm_train":
        return dig.dig_layernorm_fwd(s["x"], s["w"], s["b"], _EPS), dig.dig_layernorm_bwd(s["x"], s["dy"], s["w"], _EPS)
    if op == "rope":
        return dig.dig_rope(s["q"], s["k"], s["positions"], s["freqs"], s["axes"], interleaved=c["interleaved"], inverse=c["inverse"])
    if op == "step":
        return dig.dig_decay_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"]), s["state"]
    if op == "prompt":
        return dig.dig_decay_fwd(s["q"], s["k"], s["v"], s["log_decay"], c["grid_h"], c["grid_w"], c["direction"], s_in=s["s_in"], lengths=s["lengths"],
                                 want_s_out=True)
    out, _ = dig.dig_decay_fwd(s["q"], s["k"], s["v"], s["log_decay"], c["grid_h"], c["grid_w"], c["direction"], s_in=s["s_in"])
    return out, dig.dig_decay_bwd(s["q"], s["k"], s["v"], s["log_decay"], s["d_out"], c["grid_h"], c["grid_w"], c["direction"], s_in=s["s_in"],
                                  ds_out=s["ds_out"], want_ds_in=c["state"])


# ---- the plain forms: elementary torch operations in 32 bits, powers of the decay in 64 --------------------------------
def _powers(case, n, device):
    """The decays of all heads to the powers `n`: [H, ...], fp32."""
    lam = torch.tensor(_log_decay(case), dtype=torch.float64, device=device).view(-1, *[1] * n.dim())
    return (lam * n.double()).exp().float()


def _order(case, device):
    """The tokens in scan order."""
    t = torch.arange(case["grid_h"] * case["grid_w"], device=device)
    if case["direction"] & 2:
        t = t.view(case["grid_h"], case["grid_w"]).t().reshape(-1)
    return t.flip(0) if case["direction"] & 1 else t


def _scan(case, q, k, v, start, first):
    """Outputs [B, H, L, dv] of linear attention with a decay for each head over q, k, v [B, H, L, d]; the start state counts
    with the power `first` of the decay at the first token.  Chunks of 64 tokens: within a chunk as masked products, between them
    through the chunks' states, which a triangular matrix of decays joins."""
    B, H, L, dk = q.shape
    C, dv = 64, v.shape[-1]
    N = -(-L // C)
    fill = lambda x: torch.cat([x, x.new_zeros(B, H, N * C - L, x.shape[-1])], 2).view(B, H, N, C, x.shape[-1])
    qc, kc, vc = fill(q), fill(k), fill(v)
    i = torch.arange(C, device=q.device)
    w = _powers(case, (i[:, None] - i[None, :]).clamp(min=0), q.device) * (i[:, None] >= i[None, :])
    out = ((qc @ kc.transpose(-1, -2)) * w[:, None]) @ vc
    own_state = (kc * _powers(case, C - 1 - i, q.device)[:, None, :, None]).transpose(-1, -2) @ vc
    n = torch.arange(N, device=q.device)
    ahead = n[:, None] - 1 - n[None, :]
    join = _powers(case, (ahead * C).clamp(min=0), q.device) * (ahead >= 0)
    entering = (join @ own_state.view(B, H, N, dk * dv)).view(B, H, N, dk, dv)
    out = out + (qc @ entering) * _powers(case, i + 1, q.device)[:, None, :, None]
    out = out.reshape(B, H, N * C, dv)[:, :, :L]
    if start is not None:
        out = out + (q @ start) * _powers(case, torch.arange(L, device=q.device) + first, q.device)[:, :, None]
    return out


def _plain_attn(c, s):
    order = _order(c, s["q"].device)
    B, L, H, Hk = c["B"], c["grid_h"] * c["grid_w"], c["H"], c["Hk"]
    lengths = s["lengths"]
    if lengths is not None:
        # the tokens of each sequence in scan order, those behind its end after them
        p = torch.arange(L, device=order.device)[None].expand(B, L)
        there = p < lengths[:, None]
        order = torch.where(there, lengths[:, None] - 1 - p, p) if c["direction"] == 1 else p
    else:
        order = order[None].expand(B, L)
        there = None
    back = torch.argsort(order, 1)

    def rows(x):
        x = x.float().transpose(1, 2).repeat_interleave(H // x.shape[2], 1)
        x = x.gather(2, order[:, None, :, None].expand_as(x))
        return x if there is None else torch.where(there[:, None, :, None], x, 0)

    def tokens(x, heads, dtype):
        x = x.gather(2, back[:, None, :, None].expand_as(x))
        return x.view(B, heads, H // heads, L, -1).sum(2).transpose(1, 2).to(dtype).contiguous()

    q, k, v, st = rows(s["q"]), rows(s["k"]), rows(s["v"]), s["q"].dtype
    out = tokens(_scan(c, q, k, v, s["s_in"], 1), H, st)
    n = torch.full((B,), L, device=q.device) if lengths is None else lengths.long()
    p = torch.arange(L, device=q.device)
    if c["op"] == "prompt":
        left = (n[:, None] - 1 - p).clamp(min=0)
        s_out = (k * _powers(c, left, q.device).transpose(0, 1)[..., None]).transpose(-1, -2) @ v
        if s["s_in"] is not None:
            s_out = s_out + s["s_in"] * _powers(c, n, q.device).t()[..., None, None]
        return out, s_out
    d_out = rows(s["d_out"])
    turned = lambda x: None if x is None else x.transpose(-1, -2)
    flip = lambda x: x.flip(2)
    dq = _scan(c, d_out, v, k, turned(s["s_in"]), 1)
    dk = flip(_scan(c, flip(v), flip(d_out), flip(q), turned(s["ds_out"]), 0))
    dv = flip(_scan(c, flip(k), flip(q), flip(d_out), s["ds_out"], 0))
    ds_in = None
    if c["state"]:
        ds_in = (q * _powers(c, p + 1, q.device)[:, :, None]).transpose(-1, -2) @ d_out + s["ds_out"] * _powers(c, n, q.device).t()[..., None, None]
    return out, (tokens(dq, H, st), tokens(dk, Hk, st), tokens(dv, Hk, st), ds_in)


def _plain_step(c, s):
    each = c["H"] // c["Hk"]
    q, k, v = s["q"].float(), s["k"].float().repeat_interleave(each, 1), s["v"].float().repeat_interleave(each, 1)
    s["state"].mul_(_powers(c, torch.ones(1, device=q.device), q.device)[:, :, None]).add_(k[..., :, None] * v[..., None, :])
    return (q[..., None, :] @ s["state"])[..., 0, :].to(s["q"].dtype), s["state"]


def _plain_rope(c, s):
    freqs = torch.tensor(s["freqs"], dtype=torch.float64, device="cuda")
    angle = s["positions"][:, torch.tensor(s["axes"], device="cuda")].double() * freqs * (-1 if c["inverse"] else 1)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x):
        f = x.float()
        if c["interleaved"]:
            a, b = f[..., 0::2], f[..., 1::2]
            return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).to(x.dtype)
        a, b = f.chunk(2, -1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).to(x.dtype)

    return turn(s["q"]), turn(s["k"])


def _plain_norm(c, s):
    G, D = c["groups"], c["D"]
    x, w, b = s["x"].float().view(G, -1, D), s["w"].view(G, 1, D), s["b"].view(G, 1, D)
    mean = x.mean(-1, keepdim=True)
    r = 1 / ((x - mean).square().mean(-1, keepdim=True) + _EPS).sqrt()
    xh = (x - mean) * r
    y = (xh * w + b).view(-1, D).to(s["x"].dtype)
    if c["op"] == "norm":
        return y
    dy = s["dy"].float().view(G, -1, D)
    g = dy * w
    dx = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    # sums over up to 32768 rows in 64 bits
    return y, (dx.view(-1, D).to(s["x"].dtype), (dy * xh).sum(1, dtype=torch.float64).float().view_as(s["w"]),
               dy.sum(1, dtype=torch.float64).float().view_as(s["b"]))


def run(state):
    c = state["case"]
    if own:
        return _own(c, state)
    if c["op"] in ("norm", "norm_train"):
        return _plain_norm(c, state)
    if c["op"] == "rope":
        return _plain_rope(c, state)
    if c["op"] == "step":
        return _plain_step(c, state)
    return _plain_attn(c, state)


# ---- 64 bits, from the definitions ------------------------------------------------------------------------------------
def _exact_attn(c, s):
    """Sums over all pairs of tokens, a block of rows at a time, without chunk states."""
    B, H, Hk, L, dk, dv = c["B"], c["H"], c["Hk"], c["grid_h"] * c["grid_w"], c["dk"], c["dv"]
    lam = torch.tensor(_log_decay(c), dtype=torch.float64, device="cuda")
    train = c["op"] == "train"
    heads = torch.arange(H, device="cuda") // (H // Hk)
    out = torch.zeros(B, L, H, dv, dtype=torch.float64, device="cuda")
    dq = torch.zeros(B, L, H, dk, dtype=torch.float64, device="cuda")
    dk_, dv_ = torch.zeros(B, L, Hk, dk, dtype=torch.float64, device="cuda"), torch.zeros(B, L, Hk, dv, dtype=torch.float64, device="cuda")
    s_out = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda")
    ds_in = torch.zeros_like(s_out)
    grid = [y * c["grid_w"] + x for x in range(c["grid_w"]) for y in range(c["grid_h"])] if c["direction"] & 2 else list(range(L))
    for b in range(B):
        n = L if s["lengths"] is None else int(s["lengths"][b])
        seen = grid[:n] if s["lengths"] is not None else grid
        at = torch.tensor(seen[::-1] if c["direction"] & 1 else seen, dtype=torch.long, device="cuda")
        p = torch.arange(n, device="cuda", dtype=torch.float64)
        for h in range(H):
            q, k, v = s["q"][b, at, h].double(), s["k"][b, at, heads[h]].double(), s["v"][b, at, heads[h]].double()
            s0 = s["s_in"][b, h].double() if s["s_in"] is not None else None
            g = s["d_out"][b, at, h].double() if train else None
            for lo in range(0, n, 2048):
                i = slice(lo, min(n, lo + 2048))
                gap = p[i, None] - p[None, :i.stop]
                w = torch.where(gap >= 0, (lam[h] * gap).exp(), 0.0)
                a = (q[i] @ k[:i.stop].t()) * w
                o = a @ v[:i.stop]
                if s0 is not None:
                    o = o + (lam[h] * (p[i, None] + 1)).exp() * (q[i] @ s0)
                out[b, at[i], h] = o
                if train:
                    e = (g[i] @ v[:i.stop].t()) * w
                    d = e @ k[:i.stop]
                    if s0 is not None:
                        d = d + (lam[h] * (p[i, None] + 1)).exp() * (g[i] @ s0.t())
                    dq[b, at[i], h] = d
                    dk_[b, at[:i.stop], heads[h]] += e.t() @ q[i]
                    dv_[b, at[:i.stop], heads[h]] += a.t() @ g[i]
            left = (lam[h] * (n - 1 - p)).exp()[:, None]
            s_out[b, h] = (k * left).t() @ v
            if s0 is not None:
                s_out[b, h] += (lam[h] * n).exp() * s0
            if train and c["state"]:
                d1 = s["ds_out"][b, h].double()
                dk_[b, at, heads[h]] += left * (v @ d1.t())
                dv_[b, at, heads[h]] += left * (k @ d1)
                ds_in[b, h] = (q * (lam[h] * (p + 1)).exp()[:, None]).t() @ g + (lam[h] * n).exp() * d1
    if not train:
        return out, s_out
    return out, (dq, dk_, dv_, ds_in if c["state"] else None)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op = c["op"]
    if op in ("prompt", "train"):
        L = c["grid_h"] * c["grid_w"]
        if c["B"] * c["H"] * max(1, L // 2048) > 6000:
            return None
        return _exact_attn(c, s)
    if op == "step":
        each = torch.arange(c["H"], device="cuda") // (c["H"] // c["Hk"])
        g = torch.tensor([math.exp(x) for x in s["log_decay"]], dtype=torch.float64, device="cuda")
        state = torch.einsum("h,bhij->bhij", g, s["state"].double()) + torch.einsum("bhi,bhj->bhij", s["k"][:, each].double(), s["v"][:, each].double())
        return torch.einsum("bhi,bhij->bhj", s["q"].double(), state), state
    if op == "rope":
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                        s["positions"].double()[:, s["axes"]] * torch.tensor(s["freqs"], dtype=torch.float64, device="cuda"))
        z = (z.conj() if c["inverse"] else z)[:, None]

        def turn(x):
            x = x.double()
            half = x.shape[-1] // 2
            y = torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous()) if c["interleaved"] else torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous())
            y = y * z
            return torch.view_as_real(y).flatten(-2) if c["interleaved"] else torch.cat([y.real, y.imag], -1)

        return turn(s["q"]), turn(s["k"])
    x = s["x"].double()
    each = c["rows"] // c["groups"]
    wide = lambda t: t.double().view(c["groups"], -1).repeat_interleave(each, 0)
    var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
    xh = (x - mean) * torch.rsqrt(var + _EPS)
    y = xh * wide(s["w"]) + wide(s["b"])
    if op == "norm":
        return y
    dy = s["dy"].double()
    # through the norm's Jacobian: the part of w dy across the mean and across xh
    g = wide(s["w"]) * dy
    g = g - g.sum(1, keepdim=True) / c["D"]
    dx = torch.rsqrt(var + _EPS) * (g - xh * ((g * xh).sum(1, keepdim=True) / c["D"]))
    of = lambda t: t.view(c["groups"], each, c["D"]).sum(1)
    return y, (dx, of(dy * xh).view_as(s["w"]), of(dy).view_as(s["b"]))


def work(case):
    """Each input read once and each output written once; affine parameters, positions and lengths are left out as small.
    Attention flops: the recurrence token by token (decay, update and readout of a state of dk x dv), and for the gradients the
    state again and twice as much."""
    w, op = 4 if case["dtype"] == "f32" else 2, case["op"]
    if op in ("norm", "norm_train"):
        n = case["rows"] * case["D"]
        return {"bytes": n * w * (2 if op == "norm" else 5), "flops": n * (8 if op == "norm" else 24)}
    B, H, Hk = case["B"], case["H"], case["Hk"]
    if op == "rope":
        n = B * case["T"] * case["grid_h"] * case["grid_w"] * (H + Hk) * case["d"]
        return {"bytes": 2 * n * w, "flops": 3 * n}
    dk, dv = case["dk"], case["dv"]
    n = B * case["grid_h"] * case["grid_w"]
    states = B * H * dk * dv * 4
    first = n * (H * (dk + dv) + Hk * (dk + dv)) * w
    flops = 5 * n * H * dk * dv
    if op == "step":
        return {"bytes": first + 2 * states, "flops": flops}
    if op == "prompt":
        return {"bytes": first + states * (2 if case["state"] else 1), "flops": flops}
    # the forward pass's inputs are the backward pass's too: in q k v d_out, out the output and the three gradients
    return {"bytes": first + n * (H * (dk + dv) + Hk * (dk + dv)) * w + states * (3 if case["state"] else 0), "flops": 3 * flops + 4 * n * H * dk * dv}
