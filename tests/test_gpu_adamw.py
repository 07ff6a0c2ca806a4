"""AdamW on the GPU against the fp64 oracle, and a whole training step with it: Muon on the matrices of a model, AdamW on the rest.

Tolerances: m takes three roundings to fp32, v four (2^-24 each, relative to its terms, all of one sign in v); x takes its own
rounding and that of the update, whose square root, reciprocal and products are a unit in the last place each: 16 * 2^-24."""
import math

import numpy as np
import pytest

from oracle.optimizers_oracle import adamw_step, muon_step
from paper_2605_16341_amd import binding

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


def types(torch, name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def flat(torch, rng, lengths, dtype, scale, lead=0, positive=False):
    """Tensors packed one behind the other in one buffer that starts with `lead` elements and ends with 8, all 7."""
    total = sum(lengths)
    buf = torch.full((lead + total + 8,), 7.0, device="cuda:0", dtype=dtype)
    a = scale * rng.standard_normal(total)
    buf[lead:lead + total].copy_(torch.from_numpy(np.abs(a) if positive else a))
    at, out = lead, []
    for n in lengths:
        out.append(buf[at:at + n])
        at += n
    return buf, out


def host(seq):
    return [t.double().cpu().numpy() for t in seq]


def check(state, before, g, t, lr, b1, b2, eps, wd, x_name):
    for x, m, v, x0, m0, v0, g0, lr_i, wd_i in zip(*map(host, state), *before, g, lr, wd):
        wx, wm, wv = adamw_step(x0, g0, m0, v0, t, lr_i, b1, b2, eps, wd_i)
        assert np.all(np.abs(m - wm) <= 4 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * g0)) + 1e-44)
        assert np.all(np.abs(v - wv) <= 6 * U * wv + 1e-44)
        # the update's own error: that of m over m-hat's terms, and 16 units of the update
        terms = (np.abs(b1 * m0) + np.abs((1 - b1) * g0)) / (1 - b1 ** t) / (np.sqrt(wv / (1 - b2 ** t)) + eps)
        room = HALF[x_name] * np.abs(wx) + 4 * U * np.abs(x0) + 16 * U * lr_i * terms + 1e-44
        assert np.all(np.abs(x - wx) <= room), np.max(np.abs(x - wx) / room)


@pytest.mark.parametrize("lengths", [[1], [7], [8], [0], [0, 5, 0], [4096], [4095, 4097], [12289], [1000] * 3 + [8192] * 2, [3] * 200,
                                     [65536, 1, 0, 333]])
@pytest.mark.parametrize("x,g", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("lead", [0, 1])
def test_steps(lengths, x, g, lead):
    """Lengths around the work of a thread and a workgroup, more tensors than a launch takes, packed so that most start off a
    16-byte boundary; three steps on the same state."""
    import torch
    rng = np.random.default_rng(sum(lengths) + len(lengths))
    b1, b2, eps, lr = 0.9, 0.95, 1e-8, 0.01
    wd = [0.1 * (i % 3) for i in range(len(lengths))]
    scales = [1.0 + (i % 2) for i in range(len(lengths))]
    opt = binding.AdamW(lengths, x_dtype=x, g_dtype=g, lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd, lr_scale=scales)
    bufs = [flat(torch, rng, lengths, types(torch, x), 0.1, lead), flat(torch, rng, lengths, torch.float32, 0.0, lead),
            flat(torch, rng, lengths, torch.float32, 0.0, lead)]
    X, M, V = (b[1] for b in bufs)
    counter = torch.zeros(2, device="cuda:0", dtype=torch.int32)
    # lr and the decays reach the kernel as floats, 1 - lr wd as one
    lr_i = [float(np.float32(lr)) * s for s in scales]
    wd_i = [float(np.float32(w)) for w in wd]
    for t in range(1, 4):
        _, G = flat(torch, rng, lengths, types(torch, g), 1e-2, lead)
        before, grads = [host(s) for s in (X, M, V)], host(G)
        opt.step(X, G, M, V, counter)
        torch.cuda.synchronize()
        assert counter.tolist() == [t, 0]
        check((X, M, V), before, grads, t, lr_i, b1, b2, float(np.float32(eps)), wd_i, x)
        for buf, views in bufs:
            n = sum(lengths)
            assert bool((buf[:lead] == 7).all()) and bool((buf[lead + n:] == 7).all())


@pytest.mark.parametrize("t0", [0, 1, 999, 100000])
def test_bias_correction_from_the_counter(t0):
    import torch
    rng = np.random.default_rng(t0)
    lengths = [300]
    opt = binding.AdamW(lengths, x_dtype="f32", lr=0.1, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
    X, G, M = (flat(torch, rng, lengths, torch.float32, s)[1] for s in (1.0, 1e-2, 1e-3))
    V = flat(torch, rng, lengths, torch.float32, 1e-5, positive=True)[1]
    counter = torch.tensor([t0, 0], device="cuda:0", dtype=torch.int32)
    before, grads = [host(s) for s in (X, M, V)], host(G)
    opt.step(X, G, M, V, counter)
    f = lambda v: float(np.float32(v))
    check((X, M, V), before, grads, t0 + 1, [f(0.1)], 0.9, 0.999, f(1e-8), [f(0.01)], "f32")
    assert counter.tolist() == [t0 + 1, 0]


def test_zero_gradients_and_non_finite_ones_stay_where_they_are():
    import torch
    opt = binding.AdamW([16], x_dtype="f32", lr=0.1, eps=1e-8)
    X, G, M, V = (torch.zeros(16, device="cuda:0") for _ in range(4))
    X += 1.0
    G[3], G[7] = float("nan"), float("inf")
    counter = torch.zeros(2, device="cuda:0", dtype=torch.int32)
    opt.step([X], [G], [M], [V], counter)
    bad = torch.zeros(16, dtype=torch.bool, device="cuda:0")
    bad[3] = bad[7] = True
    assert bool((X[~bad] == 1.0).all()) and bool(X[bad].isnan().all())
    assert bool((M[~bad] == 0).all()) and bool((V[~bad] == 0).all())


def test_captured_step_counts_its_replays():
    import torch
    rng = np.random.default_rng(1)
    lengths = [513, 40, 70000] + [11] * 80
    opt = binding.AdamW(lengths, x_dtype="bf16", lr=0.01, weight_decay=0.1)

    def state():
        r = np.random.default_rng(2)
        return [flat(torch, r, lengths, dt, s)[1] for dt, s in ((torch.bfloat16, 0.1), (torch.bfloat16, 1e-2), (torch.float32, 0.0), (torch.float32, 0.0))] + \
               [torch.zeros(2, device="cuda:0", dtype=torch.int32)]

    eager, graphed = state(), state()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        opt.step(*graphed)
    for t in range(1, 6):
        for n, a, b in zip(lengths, eager[1], graphed[1]):
            g = torch.from_numpy(1e-2 * rng.standard_normal(n))
            a.copy_(g)
            b.copy_(g)
        graph.replay()
        torch.cuda.synchronize()
        opt.step(*eager)
        torch.cuda.synchronize()
        assert eager[4].tolist() == graphed[4].tolist() == [t, 0]
        for k in (0, 2, 3):
            assert all(torch.equal(a, b) for a, b in zip(eager[k], graphed[k]))


def test_training_step_of_a_small_model_in_one_graph():
    """The two optimizers as they are used together: a two-layer model's matrices by Muon, its embedding, gains and biases by
    AdamW, one captured graph, six replays against the oracle with gradients of a regression loss."""
    import torch
    rng = np.random.default_rng(3)
    d, f, vocab = 48, 80, 37
    names = ["up", "down"]
    shapes = [(f, d), (d, f)]
    lengths = [vocab * d, d, f]                # embedding, gain, bias
    muon = binding.Muon(shapes, x_dtype="f32", lr=0.02, weight_decay=0.05, mu=0.9)
    adam = binding.AdamW(lengths, x_dtype="f32", lr=0.01, betas=(0.9, 0.95), weight_decay=[0.1, 0.0, 0.0])
    dev = torch.device("cuda:0")
    put = lambda a: torch.from_numpy(a).to(dev, torch.float32)
    W = [put(0.1 * rng.standard_normal(s)) for s in shapes]
    E, gain, bias = put(0.1 * rng.standard_normal((vocab, d))), torch.ones(d, device=dev), torch.zeros(f, device=dev)
    tokens, target = torch.from_numpy(rng.integers(0, vocab, 64)).to(dev), put(rng.standard_normal((64, d)))
    params = W + [E, gain, bias]
    grads = [torch.zeros_like(p) for p in params]
    state = [torch.zeros_like(p) for p in params]
    second = [torch.zeros_like(p) for p in params[2:]]
    counter = torch.zeros(2, device=dev, dtype=torch.int32)

    def backward():
        """Gradients of 0.5 mean (y - target)^2, y = W_down relu(W_up (gain * E[tokens]) + bias), by hand."""
        e = E[tokens]
        h = (e * gain) @ W[0].t() + bias
        a = h.clamp_min(0)
        dy = (a @ W[1].t() - target) / target.numel()
        dh = (dy @ W[1]) * (h > 0)
        de = dh @ W[0]
        grads[0].copy_(dh.t() @ (e * gain))
        grads[1].copy_(dy.t() @ a)
        grads[2].zero_().index_add_(0, tokens, de * gain)
        grads[3].copy_((de * e).sum(0))
        grads[4].copy_(dh.sum(0))

    def optimise():
        muon.step(W, grads[:2], state[:2])
        adam.step([E.view(-1), gain, bias], [g.view(-1) for g in grads[2:]], [s.view(-1) for s in state[2:]], [s.view(-1) for s in second], counter)

    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        optimise()
    f32 = lambda v: float(np.float32(v))
    for t in range(1, 7):
        backward()
        p0, g0, s0, v0 = (host(seq) for seq in (params, grads, state, second))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in range(2):
            scale = math.sqrt(max(1.0, shapes[k][0] / shapes[k][1]))
            wx, wm, _ = muon_step(p0[k], g0[k], s0[k], binding.MUON_COEFFS, f32(0.9), f32(0.02), f32(0.05), f32(scale))
            # 5 steps of rounding to 22 bits, each multiplied by at most 3.4445^5 (see the tolerance of the Muon tests)
            assert np.linalg.norm(host([W[k]])[0] - wx) <= 0.02 * scale * 15 * 2.0 ** -22 * 3.4445 ** 5 + 4 * U * np.linalg.norm(wx), (names[k], t)
            assert np.allclose(host([state[k]])[0], wm, rtol=4 * U, atol=4 * U * np.abs(wm).max())
        for k in range(3):
            wx, wm, wv = adamw_step(p0[2 + k], g0[2 + k], s0[2 + k], v0[k], t, f32(0.01), 0.9, 0.95, f32(1e-8), f32([0.1, 0.0, 0.0][k]))
            assert np.allclose(host([params[2 + k]])[0], wx, rtol=32 * U, atol=32 * U * 0.1)
            assert np.allclose(host([second[k]])[0], wv, rtol=8 * U, atol=1e-44)
        assert counter.tolist() == [t, 0]


def test_a_tensor_beyond_32_bit_offsets():
    import torch
    n = 2 ** 31 + 4099
    gen = torch.Generator(device="cuda:0").manual_seed(0)
    X, G = (torch.empty(n, device="cuda:0", dtype=torch.bfloat16).normal_(0, 0.1, generator=gen) for _ in range(2))
    M, V = (torch.zeros(n, device="cuda:0") for _ in range(2))
    spots = [slice(0, 64), slice(2 ** 30 - 32, 2 ** 30 + 32), slice(2 ** 31 - 32, 2 ** 31 + 32), slice(n - 64, n)]
    before = [[host([t[s]])[0] for t in (X, M, V)] for s in spots]
    grads = [host([G[s]])[0] for s in spots]
    counter = torch.zeros(2, device="cuda:0", dtype=torch.int32)
    binding.AdamW([n], x_dtype="bf16", lr=0.01).step([X], [G], [M], [V], counter)
    f = lambda v: float(np.float32(v))
    for s, b, g in zip(spots, before, grads):
        check(([X[s]], [M[s]], [V[s]]), [[b[0]], [b[1]], [b[2]]], [g], 1, [f(0.01)], 0.9, 0.999, f(1e-8), [0.0], "bf16")
    assert bool(((V > 0) == (G != 0)).all())          # no element was left out
