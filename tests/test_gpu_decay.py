"""Linear attention with a decay for each head on the GPU against the fp64 recurrence: forward, backward, single tokens."""
import numpy as np
import pytest
import torch

import decay_ref as ref

pytestmark = pytest.mark.gpu


def check(B, H, Hk, gh, gw, dk, dv, dtype, direction, *, log_decay=None, state=False, lengths=None, seed=1, backward=True, fused=False):
    from paper_2405_18428_b200 import dig
    L = gh * gw
    x = ref.make(B, L, H, Hk, dk, dv, dtype, seed, state)
    log_decay = ref.decays(H) if log_decay is None else log_decay
    q, k, v, d_out = (ref.dev(x[n], dtype) for n in ("q", "k", "v", "d_out"))
    s_in, ds_out = (ref.dev(x[n], "f32") for n in ("s_in", "ds_out"))
    if fused:
        both = torch.cat([q.flatten(2), k.flatten(2), v.flatten(2)], 2)
        q, k, v = both.split([H * dk, Hk * dk, Hk * dv], 2)
        q, k, v = q.unflatten(2, (H, dk)), k.unflatten(2, (Hk, dk)), v.unflatten(2, (Hk, dv))
        assert not k.is_contiguous() or L == 1
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if lengths is not None:
        # what stands behind the end of a sequence does not count
        for b, m in enumerate(lengths):
            for t in (q, k, v, d_out):
                t[b, max(m, 0):] = float("nan")
    big = ref.magnitude(x)
    out, s_out = dig.dig_decay_fwd(q, k, v, log_decay, gh, gw, direction, s_in=s_in, lengths=n, want_s_out=True)
    o, s = ref.fwd(x, log_decay, gh, gw, direction, lengths)
    om, sm = ref.fwd(big, log_decay, gh, gw, direction, lengths)
    terms = L + dk + dv + 64
    ref.close("out", out, o, om, dtype, terms)
    ref.close("s_out", s_out, s, sm, dtype, terms, state=True)
    plain, none = dig.dig_decay_fwd(q, k, v, log_decay, gh, gw, direction, s_in=s_in, lengths=n)
    assert none is None and torch.equal(plain, out)
    if not backward:
        return
    got = dig.dig_decay_bwd(q, k, v, log_decay, d_out, gh, gw, direction, s_in=s_in, ds_out=ds_out, lengths=n, want_ds_in=True)
    want, size = ref.bwd(x, log_decay, gh, gw, direction, lengths), ref.bwd(big, log_decay, gh, gw, direction, lengths)
    for name, a, b, m in zip(("dq", "dk", "dv"), got, want, size):
        ref.close(name, a, b, m, dtype, terms * (H // Hk))
    ref.close("ds_in", got[3], want[3], size[3], dtype, terms, state=True)
    assert dig.dig_last_device_status() == dig.DIG_OK
    again = dig.dig_decay_bwd(q, k, v, log_decay, d_out, gh, gw, direction, s_in=s_in, ds_out=ds_out, lengths=n)
    assert again[3] is None and all(torch.equal(a, b) for a, b in zip(again[:3], got[:3]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("direction", [0, 1, 2, 3])
@pytest.mark.parametrize("gh,gw", [(1, 1), (1, 7), (3, 21), (8, 8), (5, 13), (16, 8), (7, 19), (24, 16)])
def test_orders_and_lengths(dtype, direction, gh, gw):
    check(2, 3, 3, gh, gw, 64, 64, dtype, direction, seed=gh * gw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(8, 8), (16, 64), (72, 72), (64, 128), (128, 128), (24, 40), (128, 8), (80, 96), (120, 88)])
def test_head_sizes(dtype, dk, dv):
    check(1, 2, 2, 9, 31, dk, dv, dtype, 1, state=True, seed=dk + dv)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,fused", [(4, 2, False), (6, 1, True), (3, 3, True)])
def test_shared_heads_and_fused_projections(dtype, H, Hk, fused):
    check(2, H, Hk, 11, 17, 64, 64, dtype, 2, state=True, fused=fused, seed=H)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("direction", [0, 1])
@pytest.mark.parametrize("state", [False, True])
def test_padded_batches(dtype, direction, state):
    check(7, 2, 1, 1, 300, 64, 72, dtype, direction, state=state, lengths=[300, 0, 1, 128, 129, 257, 64], seed=3)


def test_lengths_outside_the_range_count_as_the_nearest():
    from paper_2405_18428_b200 import dig
    x = ref.make(3, 40, 2, 2, 64, 64, "bf16", 5)
    q, k, v = (ref.dev(x[n], "bf16") for n in ("q", "k", "v"))
    run = lambda n: dig.dig_decay_fwd(q, k, v, ref.decays(2), 1, 40, lengths=torch.tensor(n, dtype=torch.int32, device="cuda"), want_s_out=True)
    for a, b in zip(run([-7, 41, 2 ** 31 - 1]), run([0, 40, 40])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("log_decay", [0.0, -1e-6, -0.7, -20.0, -88.0, -1e5, -3e38])
def test_decays_from_none_to_all(dtype, log_decay):
    check(1, 2, 2, 6, 50, 64, 64, dtype, 0, log_decay=[log_decay] * 2, state=True, seed=9)


@pytest.mark.parametrize("dtype,B,H,gh,gw,d", [("bf16", 1, 4, 50, 61, 72), ("bf16", 2, 3, 64, 40, 64), ("f32", 1, 4, 41, 47, 64), ("bf16", 1, 2, 33, 64, 128)])
@pytest.mark.parametrize("direction", [0, 3])
def test_long_sequences_are_cut(dtype, B, H, gh, gw, d, direction):
    check(B, H, H, gh, gw, d, d, dtype, direction, log_decay=[-2.0 ** -(3 + 2 * h) for h in range(H)], state=True, seed=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_short_sequences(dtype):
    check(70, 6, 6, 5, 5, 64, 64, dtype, 1, backward=True, seed=4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_sequence_in_pieces(dtype):
    # cut at odd places and chained through the state: the whole
    from paper_2405_18428_b200 import dig
    x = ref.make(2, 500, 2, 2, 64, 64, dtype, 8, True)
    lam = [-0.004, -0.2]
    q, k, v = (ref.dev(x[n], dtype) for n in ("q", "k", "v"))
    s, outs = ref.dev(x["s_in"], "f32"), []
    for lo, hi in ((0, 1), (1, 130), (130, 131), (131, 500)):
        o, s = dig.dig_decay_fwd(q[:, lo:hi], k[:, lo:hi], v[:, lo:hi], lam, 1, hi - lo, s_in=s, want_s_out=True)
        outs.append(o)
    o, s_ref = ref.fwd(x, lam, 1, 500, 0)
    om, sm = ref.fwd(ref.magnitude(x), lam, 1, 500, 0)
    ref.close("out", torch.cat(outs, 1), o, om, dtype, 700)
    # four states in a row, each with its own rounding
    ref.close("s_out", s, s_ref, 4 * sm, dtype, 700, state=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hk,dk,dv", [(1, 1, 1, 8, 8), (3, 6, 6, 64, 64), (2, 4, 2, 72, 128), (5, 6, 1, 128, 40), (64, 16, 16, 72, 72)])
def test_steps(dtype, B, H, Hk, dk, dv):
    from paper_2405_18428_b200 import dig
    T, lam = 5, ref.decays(H)
    x = ref.make(B, T, H, Hk, dk, dv, dtype, 6, True)
    q, k, v = (ref.dev(x[n], dtype) for n in ("q", "k", "v"))
    state = ref.dev(x["s_in"], "f32")
    o, s = ref.fwd(x, lam, 1, T, 0)
    om, sm = ref.fwd(ref.magnitude(x), lam, 1, T, 0)
    for t in range(T):
        out = dig.dig_decay_step(*(a[:, t].contiguous() for a in (q, k, v)), lam, state)
        # fp32 arithmetic whatever the storage: the result's rounding, and that of its terms in fp32
        got = out.float().cpu().numpy()
        lim = ref.HALF[dtype] * np.abs(o[:, t]) + (T * 2.0 ** -20 + (dk + 8) * 2.0 ** -24) * om[:, t] + 1e-30
        assert (np.abs(got - o[:, t]) <= lim).all()
    assert (np.abs(state.cpu().numpy() - s) <= (T * 2.0 ** -20) * sm + 1e-30).all()


def test_a_nan_reaches_no_row_of_earlier_positions():
    from paper_2405_18428_b200 import dig
    x = ref.make(1, 300, 1, 1, 64, 64, "bf16", 2)
    q, k, v = (ref.dev(x[n], "bf16") for n in ("q", "k", "v"))
    clean, _ = dig.dig_decay_fwd(q, k, v, [-0.1], 1, 300)
    for at in (0, 31, 32, 100, 128, 255, 299):
        for which in range(3):
            for bad in (float("nan"), float("inf")):
                p = [t.clone() for t in (q, k, v)]
                p[which][0, at, 0, 5] = bad
                out, _ = dig.dig_decay_fwd(*p, [-0.1], 1, 300)
                keep = at // 32 * 32 if which == 2 else at
                assert torch.equal(out[:, :keep], clean[:, :keep])
                if which == 0:
                    assert torch.equal(out[:, at + 1:], clean[:, at + 1:])
                assert not torch.isfinite(out[0, at]).all()


def test_streams_graphs_and_given_results():
    from paper_2405_18428_b200 import dig
    x = ref.make(2, 600, 3, 3, 64, 64, "bf16", 7, True)
    q, k, v, d_out = (ref.dev(x[n], "bf16") for n in ("q", "k", "v", "d_out"))
    s_in, ds_out = (ref.dev(x[n], "f32") for n in ("s_in", "ds_out"))
    lam = ref.decays(3)

    def both(out=None, grads=None):
        o = dig.dig_decay_fwd(q, k, v, lam, 20, 30, 2, s_in=s_in, want_s_out=True, out=out)
        return o + dig.dig_decay_bwd(q, k, v, lam, d_out, 20, 30, 2, s_in=s_in, ds_out=ds_out, want_ds_in=True, grads=grads)

    want = [t.clone() for t in both()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    given = torch.empty_like(want[0]), [torch.empty_like(t) for t in want[2:5]]
    got = both(*given)
    assert got[0].data_ptr() == given[0].data_ptr() and all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, outs = [], []
    for _ in range(2):               # two graphs, replayed side by side
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both())
        graphs.append(g)
    for t in outs:
        for y in t:
            y.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    for t in outs:
        assert all(torch.equal(a, b) for a, b in zip(t, want))


def test_gradient_against_differences():
    # fp32 storage, a loss linear in q: a step of any size gives its derivative exactly up to rounding; k and v likewise
    from paper_2405_18428_b200 import dig
    x = ref.make(1, 70, 2, 1, 16, 24, "f32", 12, True)
    t = {n: ref.dev(a, "f32") for n, a in x.items()}
    lam = [-0.05, -0.5]

    def loss(q, k, v, s):
        out, s_out = dig.dig_decay_fwd(q, k, v, lam, 10, 7, 3, s_in=s, want_s_out=True)
        return float((out.double() * t["d_out"].double()).sum() + (s_out.double() * t["ds_out"].double()).sum())

    grads = dig.dig_decay_bwd(t["q"], t["k"], t["v"], lam, t["d_out"], 10, 7, 3, s_in=t["s_in"], ds_out=t["ds_out"], want_ds_in=True)
    base = [t["q"], t["k"], t["v"], t["s_in"]]
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i, g in enumerate(grads):
        step = torch.randn(base[i].shape, generator=gen, device="cuda")
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + step, base[i] - step
        slope = (loss(*up) - loss(*down)) / 2
        want = float((g.double() * step.double()).sum())
        # each loss is a sum of about 4000 values of size 10 known to about 1e-6
        assert abs(slope - want) <= 4e3 * 10 * 1e-6 + 1e-6 * abs(want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_further_apart_than_32_bits_count(dtype):
    from paper_2405_18428_b200 import dig
    L, H, d, apart = 1100, 2, 64, 1 << 22                    # the last row starts at 4.6e9 elements
    storage = torch.bfloat16 if dtype == "bf16" else torch.float32
    far = torch.empty(1, L, apart, dtype=storage, device="cuda")
    near = torch.randn(1, L, 2 * H * d, device="cuda").to(storage)
    far[:, :, :2 * H * d] = near
    cut = lambda t: [x.unflatten(2, (-1, d)) for x in (t[:, :, :H * d], t[:, :, H * d:(H + 1) * d], t[:, :, (H + 1) * d:2 * H * d])]
    d_out = torch.randn(1, L, H, d, device="cuda").to(storage)
    lam = [-0.01, -0.5]
    for direction in (1, 2):
        runs = []
        for t in (far, near):
            q, k, v = cut(t)
            runs.append((*dig.dig_decay_fwd(q, k, v, lam, 20, 55, direction, want_s_out=True), *dig.dig_decay_bwd(q, k, v, lam, d_out, 20, 55, direction, want_ds_in=True)))
        assert all(torch.equal(a, b) for a, b in zip(*runs))
    freqs, axes = dig.dig_rope_freqs((32,))
    pos = torch.arange(L, device="cuda", dtype=torch.int32).view(L, 1)
    want = dig.dig_rope(*cut(near)[:2], pos, freqs, axes)
    assert all(torch.equal(a, b) for a, b in zip(dig.dig_rope(*cut(far)[:2], pos, freqs, axes), want))
    turned = dig.dig_rope(*cut(far)[:2], pos, freqs, axes, inplace=True)
    assert all(torch.equal(a, b) for a, b in zip(turned, want))
    del far, turned, q, k, v, t
    torch.cuda.empty_cache()


def test_a_turn_in_place_needs_tensors_of_its_own():
    from paper_2405_18428_b200 import dig
    x = torch.randn(1, 16, 2, 64, device="cuda")
    pos = torch.zeros(16, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(dig.DigError):
        dig.dig_rope(x, x, pos, *dig.dig_rope_freqs((32,)), inplace=True)
    a, b = dig.dig_rope(x, x, pos, *dig.dig_rope_freqs((32,)))
    assert torch.equal(a, x) and torch.equal(b, x)


@pytest.mark.parametrize("B,H,Hk,L,d", [(1, 6, 6, 256, 64), (5, 16, 4, 2500, 128), (128, 6, 6, 256, 64)])
def test_the_final_state_is_there_for_what_follows(B, H, Hk, L, d):
    """Uncut sequences: their final state is summed beside the passes.  On two streams at once, and as a replayed graph."""
    from paper_2405_18428_b200 import dig
    mk = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)
    q, k, v, d_out = mk(B, L, H, d), mk(B, L, Hk, d), mk(B, L, Hk, d), mk(B, L, H, d)
    s_in, ds_out = torch.randn(B, H, d, d, device="cuda"), torch.randn(B, H, d, d, device="cuda")
    lam = [-0.002 * (h + 1) for h in range(H)]
    token = q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous()

    def run():
        out, s = dig.dig_decay_fwd(q, k, v, lam, 1, L, s_in=s_in, want_s_out=True)
        kept = s.clone()
        step = dig.dig_decay_step(*token, lam, s)
        grads = dig.dig_decay_bwd(q, k, v, lam, d_out, 1, L, s_in=s_in, ds_out=ds_out, want_ds_in=True)
        return out.clone(), kept, s, step, *(g.clone() for g in grads)

    want = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(8):
        for stream in streams:
            with torch.cuda.stream(stream):
                got.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = run()
    for t in kept:
        t.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, want))
    assert dig.dig_last_device_status() == dig.DIG_OK
