"""Linear attention with a decay for each head in 64 bits: the oracle's recurrence with a constant gate, heads that share keys and
values repeated, padded sequences cut, and elementwise bounds on the error of the GPU results."""
from __future__ import annotations

import numpy as np
import torch

import oracle

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def make(B, L, H, Hk, dk, dv, dtype, seed, state=False):
    rng = np.random.default_rng(seed)

    def values(*shape, scale=1.0):
        t = torch.from_numpy(rng.standard_normal(shape) * scale).float()
        return (t.to(torch.bfloat16).float() if dtype == "bf16" else t).numpy()

    x = dict(q=values(B, L, H, dk), k=values(B, L, Hk, dk, scale=dk ** -0.5), v=values(B, L, Hk, dv), d_out=values(B, L, H, dv), s_in=None, ds_out=None)
    if state:
        x["s_in"], x["ds_out"] = (rng.standard_normal((B, H, dk, dv)).astype(np.float32) for _ in range(2))
    return x


def decays(H, kind="mixed"):
    if kind == "mixed":              # from none to one that forgets a token within two, over the heads
        return [[0.0, -0.01, -0.3, -1e-4, -2.5, -0.05][h % 6] for h in range(H)]
    return [kind] * H


def _gate(q, log_decay):
    return np.broadcast_to(np.asarray(log_decay, dtype=np.float32).astype(np.float64)[None, None, :, None], q.shape)


def fwd(x, log_decay, gh, gw, direction, lengths=None):
    """out and s_out in fp64."""
    q = x["q"]
    B, L, H, dk = q.shape
    share = H // x["k"].shape[2]
    k, v = (np.repeat(x[n], share, 2) for n in ("k", "v"))
    s_in = x["s_in"]
    if lengths is None:
        return oracle.gla_fwd_state(q, k, v, _gate(q, log_decay), s_in, gh, gw, direction)
    out = np.zeros(q.shape[:3] + (v.shape[-1],))
    s = np.zeros((B, H, dk, v.shape[-1])) if s_in is None else s_in.astype(np.float64).copy()
    for b in range(B):
        n = min(max(int(lengths[b]), 0), L)
        if n:
            o, s1 = oracle.gla_fwd_state(q[b:b + 1, :n], k[b:b + 1, :n], v[b:b + 1, :n], _gate(q[b:b + 1, :n], log_decay),
                                         None if s_in is None else s_in[b:b + 1], 1, n, direction)
            out[b, :n], s[b] = o[0], s1[0]
    return out, s


def bwd(x, log_decay, gh, gw, direction, lengths=None):
    """dq, dk, dv, ds_in in fp64."""
    q = x["q"]
    B, L, H, dk = q.shape
    Hk = x["k"].shape[2]
    share = H // Hk
    k, v = (np.repeat(x[n], share, 2) for n in ("k", "v"))
    dv = v.shape[-1]
    grads = [np.zeros(q.shape), np.zeros(q.shape), np.zeros(v.shape)]
    ds = np.zeros((B, H, dk, dv)) if x["ds_out"] is None else x["ds_out"].astype(np.float64).copy()
    for b in range(B):
        n = L if lengths is None else min(max(int(lengths[b]), 0), L)
        if n == 0:
            continue
        at = slice(b, b + 1)
        r = oracle.gla_bwd_state(q[at, :n], k[at, :n], v[at, :n], _gate(q[at, :n], log_decay), x["d_out"][at, :n],
                                 None if x["s_in"] is None else x["s_in"][at], None if x["ds_out"] is None else x["ds_out"][at],
                                 *((gh, gw) if lengths is None else (1, n)), direction)
        for g, y in zip(grads, (r[0], r[1], r[2])):
            g[b, :n] = y[0]
        ds[b] = r[4][0]
    summed = lambda g: g.reshape(B, L, Hk, share, -1).sum(3)
    return grads[0], summed(grads[1]), summed(grads[2]), ds


def magnitude(x):
    """The same inputs by their absolute values: the results are the sums of the terms' magnitudes."""
    return {n: None if a is None else np.abs(a) for n, a in x.items()}


def tolerance(ref, size, dtype, terms, state=False):
    """Elementwise bound on |result - ref|, `size` the sum of the magnitudes of the terms.
    A power of the decay is 2^(c n) with c and the product rounded to fp32 and |c n| <= 126 (smaller ones are zeros), so off by at most
    2 * 126 ln 2 * 2^-24 < 2^-16 of itself, and an approximate exponential 2^-21; powers of two factors at most occur in a product of two.
    fp32: sums of `terms` products, 2^-24 each, twice for what a tensor core may drop; bf16 storage: decayed scores, or decayed keys and
    the state they add up to (each 2^-8 of its terms), and the rounding of the result.  A state's decayed keys come in two bf16 parts: 2^-16."""
    t = 2 * (2.0 ** -16 + 2.0 ** -21) + 2 * terms * 2.0 ** -24
    if dtype == "bf16":
        t += 2.0 ** -16 if state else 2 * 2.0 ** -8 + 2.0 ** -16
    return t * size + (0.0 if state else (HALF[dtype] * (1 + t)) * np.abs(ref)) + 1e-30


def dev(a, dtype):
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def close(name, got, ref, size, dtype, terms, state=False):
    got = got.float().cpu().numpy().astype(np.float64)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) / tolerance(ref, size, dtype, terms, state)
    assert over.max() <= 1, f"{name}: {over.max():.2f} times the bound at {np.unravel_index(over.argmax(), over.shape)}"
